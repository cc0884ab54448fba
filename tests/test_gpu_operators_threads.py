"""Calls of several host threads at once: what one thread asks for changes nothing for another."""
import threading

import pytest
import torch

from paper_2503_09387_b200 import binding
from tests.test_gpu_operators import gen, ints, normal, pool, same_bits, tables

pytestmark = pytest.mark.gpu


def run_threads(work):
    """work: functions, each called in a thread of its own, all begun together; an error of any is this test's."""
    errors, start = [], threading.Barrier(len(work))

    def body(f):
        try:
            start.wait()
            f()
        except BaseException as e:                        # (handed on)
            errors.append(e)
    threads = [threading.Thread(target=body, args=(f,)) for f in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if errors:
        raise errors[0]


@pytest.mark.parametrize("rows", [1, 40])
def test_attend_of_few_and_of_most_sequences_in_two_threads(rows):
    """The shared memory that a call asks for goes by its sequences; the limit that it sets is the same for all."""
    calls = []
    for n_seqs in (1, binding.VS_CACHE_MAX_SEQS):
        g = gen(n_seqs)
        cache = pool(g, 40, 1, 64, junk=False)
        table = torch.randint(0, 40, (n_seqs, 30), device="cuda", generator=g, dtype=torch.int32)
        lengths = torch.full((n_seqs,), 70, dtype=torch.int32, device="cuda")
        q = normal(g, n_seqs * rows, 8, 64)
        calls.append((cache, table, lengths, q, cache.attend(table, lengths, q)))
    torch.cuda.synchronize()

    def many(cache, table, lengths, q, want):
        def f():
            # (the C call itself, time after time: what a program without an interpreter in between does)
            with torch.cuda.stream(torch.cuda.Stream()):
                out, lse, ws, stream = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda"), cache.workspace(), torch.cuda.current_stream()
                block = binding.VS_CACHE_QUERIES.pack(table.data_ptr(), lengths.data_ptr(), 0, table.shape[0], table.shape[1], q.shape[0], 0, q.data_ptr(),
                                                      out.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.nbytes, 512, 64, 512, 64, 8, 1, 0, 0, 0.125, 0)
                call, codes = binding.load_library().vs_cache_attention, []
                for _ in range(4000):
                    codes.append(call(cache._cache, block, stream.cuda_stream))
                stream.synchronize()
                assert set(codes) == {binding.VS_OK}
                assert same_bits(out, want[0]) and same_bits(lse, want[1])
        return f
    run_threads([many(*c) for c in calls for _ in range(2)])


@pytest.mark.parametrize("rows", [(1, 3), (40, 70), (1, 40)])
def test_attend_from_two_threads_on_one_stream(rows):
    """One cache, one stream and so one workspace: the launches of two calls do not mix."""
    g = gen(9)
    cache = pool(g, 200, 4, 128, junk=False)
    calls = []
    for n, length in zip(rows, (6000, 2900)):
        table, q = tables(g, [length], 200), normal(g, n, 28, 128)
        calls.append((table, ints([length]), q, cache.attend(table, ints([length]), q)))
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()

    def many(table, lengths, q, want):
        def f():
            with torch.cuda.stream(stream):
                got = [cache.attend(table, lengths, q) for _ in range(200)]
                stream.synchronize()
                for out, lse in got:
                    assert same_bits(out, want[0]) and same_bits(lse, want[1])
        return f
    run_threads([many(*c) for c in calls])
    assert cache.attend_status() == 0
