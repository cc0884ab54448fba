"""Host threads that share a cache and a stream: a call of the attention is several launches, and its workspace is one call's at a time.  The
library is stood in for by one that says when two calls are in it at once."""
import threading
import time

import torch

from paper_2503_09387_b200 import binding


def test_attend_from_two_threads_on_one_stream(monkeypatch):
    binding._need_torch()
    inside, met, lock = [], [], threading.Lock()

    class Library:
        @staticmethod
        def vs_cache_attention_bytes(head_dim, out):
            out._obj.value = 512
            return 0

        @staticmethod
        def vs_cache_attention(cache, block, stream):
            workspace = binding.VS_CACHE_QUERIES.unpack(block)[10]
            with lock:
                met.extend(w for w in inside if w == workspace)
                inside.append(workspace)
            time.sleep(0.002)
            with lock:
                inside.remove(workspace)
            return 0

    monkeypatch.setattr(binding, "load_library", lambda path=None: Library)
    monkeypatch.setattr(binding, "_raw_stream", lambda index: 7)
    monkeypatch.setattr(binding, "_capturing", lambda index: False)
    monkeypatch.setattr(binding, "_on_gpu", lambda t, what: t.get_device())                  # (-1, as all of these tensors)
    codes = torch.zeros((2, 1, 64, 64), dtype=torch.uint8).view(torch.float8_e4m3fn)
    cache = binding.PageCache(codes, codes, torch.ones(2, 1), torch.ones(2, 1))
    table, lengths, q = torch.zeros((1, 1), dtype=torch.int32), torch.ones(1, dtype=torch.int32), torch.zeros((1, 4, 64), dtype=torch.bfloat16)
    threads = [threading.Thread(target=lambda: [cache.attend(table, lengths, q) for _ in range(10)]) for _ in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not met and not inside
