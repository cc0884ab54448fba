// vs_token_logprobs: what a row of logits says about a given token -- its log probability and its place in the order -- with the
// entropy of the row and its best alternatives.
//
//   lse = log sum_j e^{x_j},   logprob = x_t - lse,   entropy = lse - sum_j p_j x_j,   p_j = e^{x_j - lse}
//   rank = how many tokens come before t in the order "larger logit, else lower index"; alternatives: the first `top` of that order.
//
// One pass over the row.  A thread keeps the largest logit that it has met apart and sums the others, each new one or the largest that it takes
// the place of:  s = sum of e^{y - ref},  u = sum of (y - ref) e^{y - ref};  ref is its first logits' maximum, moved only when the largest is far above it.
// With M the row's largest and s, u relative to it,  log sum = log1p(s)  and  entropy = that - u / (1 + s):  a row that is all but certain
// keeps the few bits that its entropy has, and nothing in the loop branches on a new maximum.
// Alternatives: the k-th largest of the threads' own maxima is a bound that at least k logits reach, so only threads whose maximum reaches
// it hold any of the best k.  Their logits -- a few dozen threads' -- are read once more (they lie in L2), those that reach the bound collected and put in
// order by counting.
//
// What bounds it: the logits' bytes, once from HBM; a row or two: the chain of loads, maxima and the two small sorts.  Few rows: the
// CTAs of a cluster share a row, and the first one joins their parts through shared memory; many: a CTA a row.
#include "vs_operators.cuh"
#include "vs_ptx.cuh"

namespace vs {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kTop = VS_MAX_TOP, kMaxCluster = 8;
constexpr int kAbove = 1024, kEqual = 256;             // candidates above the bound, and equal to it, that are kept
constexpr uint32_t kLeastNumber = 0x00800000u;         // the most negative finite logit, as ordered() has it; -inf is one less, NaN 0
constexpr float kLog2e = 1.4426950408889634f;

struct ScoreArgs {
  const void* logits;
  const int32_t* tokens;
  float *logprob, *entropy, *top_logprob;
  int32_t *rank, *top_index;
  long long row_stride;
  int rows, vocab, top, cluster;
};

// what is known of a stretch of a row: its largest logit, and sums over the others relative to it
struct Part {
  float m, s, u;                       // (m = -inf: nothing but -inf, or nothing, so far; s = u = 0 then)
  uint32_t pad;
  __device__ __forceinline__ void join(const Part& o) {
    const float M = fmaxf(m, o.m), low = fminf(m, o.m);
    if (low == -INFINITY) { if (m != M) *this = o; return; }
    // the smaller of the largest joins the others
    const float d = fmaxf(low - M, -1000.f), r = ex2_approx(d * kLog2e);
    const float ls = m == M ? o.s : s, lu = m == M ? o.u : u, hs = m == M ? s : o.s, hu = m == M ? u : o.u;
    s = hs + r * (1.f + ls);
    u = hu + (r > 0.f ? r * (lu + d * (1.f + ls)) : 0.f);
    m = M;
  }
  // over the lanes of every aligned group of `n`
  __device__ __forceinline__ void join_lanes(int n) {
    for (int o = n >> 1; o > 0; o >>= 1) {
      Part q;
      q.m = __shfl_xor_sync(0xffffffffu, m, o);
      q.s = __shfl_xor_sync(0xffffffffu, s, o);
      q.u = __shfl_xor_sync(0xffffffffu, u, o);
      join(q);
    }
  }
};

__device__ __forceinline__ float of_ordered(uint32_t o) {               // (NaN of 0)
  return o == 0u ? __int_as_float(0x7fc00000) : __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint32_t ordered(float v) {                 // ascending with v; NaN below every number, -0 = 0
  if (v != v) return 0u;
  const uint32_t b = __float_as_uint(v + 0.f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
// (larger logit, else lower index) as one word; 0 is nobody's
__device__ __forceinline__ unsigned long long key_of(uint32_t o, int i) { return ((unsigned long long)o << 32) | (uint32_t)(0x7fffffff - i); }

template <typename T>
struct Vec { static constexpr int n = 16 / (int)sizeof(T); };

// the logits of vector i of a row: those behind its end as -inf
template <typename T, bool kVector>
__device__ __forceinline__ uint4 fetch(const T* row, int i, int vocab) {
  constexpr int V = Vec<T>::n;
  if (kVector && (i + 1) * V <= vocab) return __ldg(reinterpret_cast<const uint4*>(row) + i);
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(T) == 4) {
      w[j] = i * V + j < vocab ? __float_as_uint(row[i * V + j]) : 0xff800000u;
    } else {
      const uint16_t* r = reinterpret_cast<const uint16_t*>(row);
      const uint32_t lo = i * V + 2 * j < vocab ? r[i * V + 2 * j] : 0xff80u, hi = i * V + 2 * j + 1 < vocab ? r[i * V + 2 * j + 1] : 0xff80u;
      w[j] = lo | (hi << 16);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ float element(const uint4& v, int j) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(word(v, j));
  else return (j & 1) ? __uint_as_float(word(v, j >> 1) & 0xffff0000u) : __uint_as_float(word(v, j >> 1) << 16);
}

__device__ __forceinline__ unsigned long long ld_peer_u64(uint32_t addr) {
  unsigned long long v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}

struct Shared {
  unsigned long long above[kAbove], equal[kEqual + kTop], best[kMaxCluster * kTop];
  Part part[kWarps];
  int before[kWarps], odd[kWarps];     // logits that come before the token; whether a NaN or +inf was met
  Part whole;                          // this CTA's part of the row, for the cluster's first
  int n_before, n_odd, n_above, n_equal;
  uint32_t bound;
};

template <typename T, bool kVector>
__global__ void __launch_bounds__(kThreads, 2) token_logprobs_kernel(const __grid_constant__ ScoreArgs a) {
  __shared__ Shared sm;
  constexpr int V = Vec<T>::n, E = 16, U = E / V;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int C = a.cluster, row_i = (int)blockIdx.x / C, rank = (int)blockIdx.x - row_i * C;
  const T* row = static_cast<const T*>(a.logits) + (long long)row_i * a.row_stride;
  const int nv = (a.vocab + V - 1) / V;
  const int v0 = (int)((long long)nv * rank / C), v1 = (int)((long long)nv * (rank + 1) / C);
  const int token = a.tokens != nullptr ? a.tokens[row_i] : -1;
  const bool has_token = token >= 0 && token < a.vocab;
  const uint4 nothing = sizeof(T) == 4 ? make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u) : make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
  uint4 next[U];
#pragma unroll
  for (int j = 0; j < U; ++j) next[j] = v0 + tid + j * kThreads < v1 ? fetch<T, kVector>(row, v0 + tid + j * kThreads, a.vocab) : nothing;
  float xt = INFINITY;                 // (no token: nothing comes before it)
  if (has_token) {
    if constexpr (sizeof(T) == 4) xt = row[token];
    else xt = __bfloat162float(row[token]);
  }
  const bool xt_nan = xt != xt;

  // ---- one pass: largest, sums of the others, place of the token -----------------------------------------------
  float best_x = -INFINITY, ref = 0.f, sum = 0.f, sum_u = 0.f;         // ref: the thread's reference
  int n_before = 0;
  bool odd = false;
  float zero = 0.f;
  for (int v = v0 + tid; v < v1; v += U * kThreads) {
    uint4 now[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      now[j] = next[j];
      const int w = v + (U + j) * kThreads;
      next[j] = w < v1 ? fetch<T, kVector>(row, w, a.vocab) : nothing;
    }
    const float was = best_x;
    bool ties = false;
    float y[E];                                                         // what is summed: the logit, or the largest so far that it replaces
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float x = element<T>(now[i / V], i % V);
      y[i] = fminf(best_x, x);
      best_x = fmaxf(best_x, x);
      n_before += x > xt ? 1 : 0;
      ties = ties || x == xt;
      zero = fmaf(x, 0.f, zero);                                        // (NaN by a NaN or an infinity)
    }
    if (!(zero == 0.f)) {                                              // rarely, but for masked rows: NaN or +inf?
      zero = 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) odd = odd || !(element<T>(now[i / V], i % V) <= 3.402823466e38f);
    }
    if (ties) {                                                        // equal ones of a lower index
#pragma unroll
      for (int i = 0; i < E; ++i) n_before += element<T>(now[i / V], i % V) == xt && (v + (i / V) * kThreads) * V + i % V < token ? 1 : 0;
    }
    if (xt_nan) {                                                      // behind every number, and NaN of a lower index
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int w = v + (i / V) * kThreads, at = w * V + i % V;
        const float x = element<T>(now[i / V], i % V);
        n_before += w < v1 && at < a.vocab && (x == x || at < token) ? 1 : 0;
      }
    }
    if (best_x > -INFINITY && (was == -INFINITY || best_x - ref > 40.f)) {
      const float d = fmaxf(ref - best_x, -1000.f), r = was == -INFINITY ? 0.f : exp2f(d * kLog2e);
      sum_u = r > 0.f ? r * (sum_u + d * sum) : 0.f;
      sum *= r;
      ref = best_x;
    }
    float s = 0.f, u = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float d = fmaxf(y[i] - ref, -1000.f), e = ex2_approx(d * kLog2e);           // (-inf: 0, and 0 in u)
      s += e;
      u = fmaf(d, e, u);
    }
    sum += s;
    sum_u += u;
  }
  Part p = {best_x, 0.f, 0.f, 0u};
  if (best_x > -INFINITY) {
    const float d = ref - best_x, r = exp2f(d * kLog2e);               // (e^{-40} at least)
    p.s = sum * r;
    p.u = r * (sum_u + d * sum);
  }
  const uint32_t own_max = ordered(p.m);
  p.join_lanes(32);
  n_before = __reduce_add_sync(0xffffffffu, n_before);
  odd = __any_sync(0xffffffffu, odd);
  if (lane == 0) { sm.part[warp] = p; sm.before[warp] = n_before; sm.odd[warp] = odd; }
  if (tid == 0) { sm.n_above = 0; sm.n_equal = 0; }
  __syncthreads();
  if (warp == 0) {
    Part w = sm.part[lane & (kWarps - 1)];
    w.join_lanes(kWarps);
    const int b = __reduce_add_sync(0xffffffffu, lane < kWarps ? sm.before[lane] : 0);
    const bool o = __any_sync(0xffffffffu, lane < kWarps && sm.odd[lane & (kWarps - 1)] != 0);
    if (lane == 0) { sm.whole = w; sm.n_before = b; sm.n_odd = o; }
  }

  // ---- the best of this CTA's part -----------------------------------------------------------------------------
  const int k = a.top;
  if (k > 0) {
    // a bound that at least k of the threads' maxima reach, bit by bit from the top (the last 14 bits would sharpen it little)
    uint32_t bound = 0u;
    for (int bit = 31; bit >= 14; --bit) {
      const uint32_t higher = bound | (1u << bit);
      if (__syncthreads_count(own_max >= higher) >= k) bound = higher;
    }
    bound = max(bound, kLeastNumber);
    for (;;) {
      // a warp reads a thread's logits again, its lanes side by side
      for (unsigned left = __ballot_sync(0xffffffffu, own_max >= bound); left != 0u; left &= left - 1u) {
        const int t = warp * 32 + __ffs(left) - 1;
        for (int v = v0 + t + lane * kThreads; v < v1; v += 32 * kThreads) {
          const uint4 w = fetch<T, kVector>(row, v, a.vocab);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const uint32_t o = ordered(element<T>(w, e));
            const int i = v * V + e;
            if (o < bound || i >= a.vocab) continue;
            if (o > bound) { const int at = atomicAdd(&sm.n_above, 1); if (at < kAbove) sm.above[at] = key_of(o, i); }
            else { const int at = atomicAdd(&sm.n_equal, 1); if (at < kEqual) sm.equal[at] = key_of(o, i); }
          }
        }
      }
      __syncthreads();
      if (sm.n_above <= kAbove) break;
      // more than are kept: the k-th of those kept is a higher bound that k logits reach
      for (int c = tid; c < kAbove; c += kThreads) {
        const unsigned long long mine = sm.above[c];
        int place = 0;
        for (int i = 0; i < kAbove; ++i) place += sm.above[i] > mine ? 1 : 0;
        if (place == k - 1) sm.bound = (uint32_t)(mine >> 32);
      }
      __syncthreads();
      bound = sm.bound;
      if (tid == 0) { sm.n_above = 0; sm.n_equal = 0; }
      __syncthreads();
    }
    const int n_above = sm.n_above, n_found = sm.n_equal;
    int n_equal = min(n_found, kEqual);
    if (n_above + n_equal < k || (n_found > kEqual && n_above < k)) {
      // a great many equal to the bound, or fewer numbers than asked for (a masked vocabulary, a short part): the first ones in order of
      // their index that equal the bound, then -inf, then NaN, by one warp
      __syncthreads();
      if (warp == 0) {
        int have = n_found > kEqual ? 0 : n_equal;
        for (int round = n_found > kEqual ? 0 : 1; round < 3; ++round) {
          const uint32_t wanted = round == 0 ? bound : (round == 1 ? kLeastNumber - 1u : 0u);
          for (int v = v0; v < v1 && have < k - n_above; v += 32) {
            const uint4 w = v + lane < v1 ? fetch<T, kVector>(row, v + lane, a.vocab) : nothing;
            uint32_t hits = 0u;
#pragma unroll
            for (int e = 0; e < V; ++e)
              hits |= (v + lane < v1 && (v + lane) * V + e < a.vocab && ordered(element<T>(w, e)) == wanted) ? 1u << e : 0u;
            int sum = __popc(hits);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += t; }
            int at = have + sum - __popc(hits);
#pragma unroll
            for (int e = 0; e < V; ++e)
              if ((hits >> e) & 1u) { if (at < k) sm.equal[at] = key_of(wanted, (v + lane) * V + e); ++at; }
            have += __shfl_sync(0xffffffffu, sum, 31);
          }
        }
        if (lane == 0) sm.n_equal = min(have, k - n_above);
      }
      __syncthreads();
      n_equal = sm.n_equal;
    }
    const int n = n_above + (n_above < k ? n_equal : 0);
    // in order, by counting; a part of few logits may hold fewer than k
    if (tid >= n && tid < k) sm.best[tid] = 0ull;
    for (int c = tid; c < n; c += kThreads) {
      const unsigned long long mine = c < n_above ? sm.above[c] : sm.equal[c - n_above];
      int place = 0;
      for (int i = 0; i < n; ++i) place += (i < n_above ? sm.above[i] : sm.equal[i - n_above]) > mine ? 1 : 0;
      if (place < k) sm.best[place] = mine;
    }
  }
  __syncthreads();

  // ---- the row ------------------------------------------------------------------------------------------------
  if (C > 1) {
    cluster_arrive_release();
    cluster_wait_acquire();
    if (rank == 0) {
      if (warp == 0) {
        if (lane < C) {
          const uint32_t at = map_shared_rank(smem_u32(&sm.whole), (uint32_t)lane), counts = map_shared_rank(smem_u32(&sm.n_before), (uint32_t)lane);
          const unsigned long long w0 = ld_peer_u64(at), w1 = ld_peer_u64(at + 8), w2 = ld_peer_u64(counts);
          sm.part[lane] = {__uint_as_float((uint32_t)w0), __uint_as_float((uint32_t)(w0 >> 32)), __uint_as_float((uint32_t)w1), 0u};
          sm.before[lane] = (int)(uint32_t)w2;
          sm.odd[lane] = (int)(w2 >> 32);
        }
      } else if (warp < C && lane < k) {
        sm.best[warp * kTop + lane] = ld_peer_u64(map_shared_rank(smem_u32(&sm.best[lane]), (uint32_t)warp));
      }
      __syncthreads();
      // every part's best are in order: a key's place is its own there and, by halving, how many of the other parts' come before it
      const int c = tid / kTop, j = tid - c * kTop;
      if (c < C && j < k) {
        const unsigned long long mine = sm.best[c * kTop + j];
        int place = j;
        for (int q = 0; q < C; ++q) {
          if (q == c) continue;
          int lo = 0, hi = k;
          while (lo < hi) { const int mid = (lo + hi) >> 1; if (sm.best[q * kTop + mid] > mine) lo = mid + 1; else hi = mid; }
          place += lo;
        }
        if (mine != 0ull && place < k) sm.above[place] = mine;
      }
      __syncthreads();
    }
    cluster_arrive_release();          // (a peer's shared memory is read: it stays until then)
    cluster_wait_acquire();
    if (rank != 0) return;
  }
  if (warp != 0) return;
  const unsigned long long* best = C > 1 ? sm.above : sm.best;
  Part whole = sm.whole;
  int all_before = sm.n_before;
  bool bad = sm.n_odd != 0;
  if (C > 1) {
    whole = sm.part[lane & (C - 1)];
    whole.join_lanes(C);
    all_before = __reduce_add_sync(0xffffffffu, lane < C ? sm.before[lane] : 0);
    bad = __any_sync(0xffffffffu, sm.odd[lane & (C - 1)] != 0);
  }
  const float nan = __int_as_float(0x7fc00000);
  const float log_sum = log1pf(whole.s);                                // of e^{x - m}
  const bool empty = whole.m == -INFINITY;                              // nothing but -inf (and NaN)
  auto logprob_of = [&](float x) { return bad ? nan : (empty ? -INFINITY : (x - whole.m) - log_sum); };
  if (tid == 0) {
    if (a.logprob != nullptr) a.logprob[row_i] = has_token ? logprob_of(xt) : (token < 0 ? 0.f : nan);
    if (a.rank != nullptr) a.rank[row_i] = has_token ? all_before : -1;
    if (a.entropy != nullptr) a.entropy[row_i] = bad ? nan : (empty ? 0.f : fmaxf(log_sum - whole.u / (1.f + whole.s), 0.f));
  }
  if (tid < k) {
    const unsigned long long key = best[tid];
    if (a.top_index != nullptr) a.top_index[(long long)row_i * k + tid] = 0x7fffffff - (int)(uint32_t)key;
    if (a.top_logprob != nullptr) a.top_logprob[(long long)row_i * k + tid] = logprob_of(of_ordered((uint32_t)(key >> 32)));
  }
}

template <typename T, bool kVector>
int launch(const ScoreArgs& a, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.rows * a.cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = (unsigned)a.cluster; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = a.cluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, kVector>, a) == cudaSuccess ? launched() : VS_ERR_CUDA;
}

}  // namespace

}  // namespace vs

extern "C" int vs_token_logprobs(const vs_scores* x, void* cuda_stream) {
  using namespace vs;
  if (x == nullptr || x->rows < 0 || x->vocab < 1 || x->dtype < 0 || x->dtype > 1 || x->top < 0) return VS_ERR_INVALID_ARG;
  if (x->vocab > (1 << 30) || x->rows > (1 << 27)) return VS_ERR_UNSUPPORTED;
  if (x->top > VS_MAX_TOP) return VS_ERR_CAPACITY;
  if (x->top > x->vocab || (x->top > 0 && x->top_index == nullptr)) return VS_ERR_INVALID_ARG;
  if (x->rows == 0) return VS_OK;
  if ((x->logprob != nullptr || x->rank != nullptr) && x->tokens == nullptr) return VS_ERR_INVALID_ARG;
  const size_t el = x->dtype == 1 ? 4 : 2;
  if (x->logits == nullptr || !aligned(x->logits, el)) return VS_ERR_INVALID_ARG;
  const void* words[6] = {x->tokens, x->logprob, x->entropy, x->rank, x->top_index, x->top_logprob};
  for (const void* w : words) if (!aligned(w, 4)) return VS_ERR_INVALID_ARG;
  OnDevice on(x->device);
  if (!on.ok) return VS_ERR_CUDA;
  ScoreArgs a = {x->logits, x->tokens, x->logprob, x->entropy, x->top_logprob, x->rank, x->top_index, x->row_stride, x->rows, x->vocab, x->top, 1};
  // CTAs of a row, measured for rows of 5000 to 152064 logits (fp32, top 0 to 20).  A part of at least 4096 vectors keeps a CTA busy for longer than joining
  // the parts takes (one row of 32000: 9.2 us in one part, 8.9 in four; 64 rows 10.2, 11.3).  Eight parts up to eight rows (one row of 152064: 26.6 us in one,
  // 13.7 in four, 13.3 in eight; sixteen rows 28.2, 14.5, 17.1: clusters of eight wait for one another's places), four up to 74 (40 rows
  // 29.3, 20.5), then as many CTAs as there are SMs are at work anyway: two where the last round over the SMs would be less than half full
  // (197 rows 42.3, 39.8; 148 rows 27.9, 28.4; 256 rows 42.9, 50.6).
  const int vectors = (int)((x->vocab + 16 / el - 1) / (16 / el)), last = x->rows % 148;
  const int most = x->rows <= 8 ? 8 : (x->rows <= 74 ? 4 : (x->rows > 148 && last != 0 && last <= 74 ? 2 : 1));
  while (a.cluster < most && vectors >= 8192 * a.cluster) a.cluster *= 2;
  const bool vector = aligned(x->logits, 16) && (x->row_stride * (int64_t)el) % 16 == 0;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (x->dtype == 1) return vector ? launch<float, true>(a, st) : launch<float, false>(a, st);
  return vector ? launch<bf16, true>(a, st) : launch<bf16, false>(a, st);
}
