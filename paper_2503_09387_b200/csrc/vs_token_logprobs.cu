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
// order by counting.  (The bound by bisection, a barrier a bit, took 2 us more.)
//
// What bounds it: many rows, the SMs that have two of them (two rows of 152064 take one 25 us in fp32 as in bf16, 16 of them issue slots, some thirteen
// instructions a logit; of 197 rows 49 SMs have two); a row or two, the chain of loads, maxima and the small sorts.  Few rows: the CTAs of a cluster share a row, and
// the first one joins their parts through shared memory; many: a CTA a row.  Measured (fp32): 197 rows of 152064, five alternatives, 32 us (3.7 TB/s); 256 rows 33
// (4.7 TB/s); one row 10.6, 7.2 without alternatives.
#include "vs_operators.cuh"
#include "vs_ptx.cuh"

namespace vs {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kTop = VS_MAX_TOP, kMaxCluster = 8;
constexpr int kAbove = 1024, kEqual = 256;             // candidates above the bound, and equal to it, that are kept
constexpr uint32_t kLeastNumber = 0x00800000u;         // the most negative finite logit, as ordered() has it; -inf is one less, NaN 0
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kHuge = 1e38f;
constexpr int kBins = 64;

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

// A row is read in vectors of 16 bytes from the last boundary at or ahead of its first logit, which is then number `off`; [off, end) are its logits' numbers.
// Vector i: what lies outside the row as -inf, and not read.
template <typename T>
__device__ __forceinline__ uint4 fetch(const T* row, int i, int off, int end) {
  constexpr int V = Vec<T>::n;
  if (i * V >= off && (i + 1) * V <= end) return __ldg(reinterpret_cast<const uint4*>(row) + i);
  const uint32_t nothing = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  if (i * V >= end) return make_uint4(nothing, nothing, nothing, nothing);
  uint32_t w[4];
  auto there = [&](int at) { return at >= off && at < end; };
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(T) == 4) {
      w[j] = there(i * V + j) ? __float_as_uint(row[i * V + j]) : 0xff800000u;
    } else {
      const uint16_t* r = reinterpret_cast<const uint16_t*>(row);
      const uint32_t lo = there(i * V + 2 * j) ? r[i * V + 2 * j] : 0xff80u, hi = there(i * V + 2 * j + 1) ? r[i * V + 2 * j + 1] : 0xff80u;
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
  uint32_t most[kWarps], least[kWarps];                                 // of the threads' maxima
  int bins[3][kBins];
  short holder[kThreads];              // threads whose maximum reaches the bound
  Part whole;                          // this CTA's part of the row, for the cluster's first
  int n_before, n_odd, n_above, n_equal, n_holders;
  uint32_t bound;
};

// the next larger number (NaN of +inf)
__device__ __forceinline__ float next_up(float x) { return x == INFINITY ? __int_as_float(0x7fc00000) : of_ordered(ordered(x) + 1u); }
// the larger one, NaN if either is
__device__ __forceinline__ float max_nan(float a, float b) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
  return m;
}

// kOff: rows that begin off a boundary of 16 bytes (197 rows of 152064 on them, as if they might not: 34.8 us against 32.4)
template <typename T, bool kOff>
__global__ void __launch_bounds__(kThreads, 2) token_logprobs_kernel(const __grid_constant__ ScoreArgs a) {
  __shared__ Shared sm;
  constexpr int V = Vec<T>::n, E = 16, U = E / V;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int C = a.cluster, row_i = (int)blockIdx.x / C, rank = (int)blockIdx.x - row_i * C;
  const T* row = static_cast<const T*>(a.logits) + (long long)row_i * a.row_stride;
  const int off = kOff ? (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T)) : 0, end = off + a.vocab;
  row -= off;
  const int nv = (end + V - 1) / V;
  const int v0 = (int)((long long)nv * rank / C), v1 = (int)((long long)nv * (rank + 1) / C);
  const int whole_v = min(v1, end / V), steps = (v1 - v0 + U * kThreads - 1) / (U * kThreads);
  // the vectors of one step: without a question where all threads have all of theirs
  uint4 next[U];
  auto load = [&](int v, bool whole) {
    if (whole && v - tid + U * kThreads <= whole_v) {
#pragma unroll
      for (int j = 0; j < U; ++j) next[j] = __ldg(reinterpret_cast<const uint4*>(row) + (v + j * kThreads));
    } else {
#pragma unroll
      for (int j = 0; j < U; ++j) next[j] = fetch(row, v + j * kThreads, off, v + j * kThreads < v1 ? end : 0);
    }
  };
  load(v0 + tid, off == 0 || v0 > 0);
  const int token = a.tokens != nullptr ? a.tokens[row_i] : -1;
  const bool has_token = token >= 0 && token < a.vocab;
  const int token_at = token + off;
  const float nan = __int_as_float(0x7fc00000);
  float xt = nan;                      // (no token: nothing comes before it)
  if (has_token) {
    if constexpr (sizeof(T) == 4) xt = row[token_at];
    else xt = __bfloat162float(row[token_at]);
  }
  const bool xt_nan = has_token && xt != xt;
  // what reaches this comes before the token: its logit in the vectors ahead of the token's, the next larger one from there on
  const float behind = next_up(xt);
  const int token_v = has_token ? token_at / V : 0, ahead = min(token_v, v1);

  // ---- one pass: largest, sums of the others, place of the token -----------------------------------------------
  float best_x = -INFINITY, ref = 0.f, ref2 = 0.f, slip = 0.f, sum = 0.f, sum_u = 0.f;  // ref2 = ref log2e - slip, as it is rounded
  int n_before = 0;
  auto shift_sums = [&](float by) {    // by so many powers of two
    by = fmaxf(by, -1000.f);
    const float r = ex2_approx(by);
    sum_u = r * fmaf(by, sum, sum_u);
    sum *= r;
  };
  for (int step = 0, v = v0 + tid; step < steps; ++step, v += U * kThreads) {
    const float was = best_x;
    float y[E];                                                         // what is summed: the logit, or the largest so far that it replaces
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const float reach = v + j * kThreads < ahead ? xt : behind;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float x = element<T>(next[j], e);
        y[j * V + e] = fminf(best_x, x);
        best_x = max_nan(best_x, x);
        n_before += x >= reach ? 1 : 0;
      }
    }
    if (step + 1 < steps) load(v + U * kThreads, true);
    if (best_x > -INFINITY && (was == -INFINITY || best_x - ref > 40.f)) {
      const bool finite = fabsf(best_x) < kHuge;
      const float to2 = finite ? best_x * kLog2e : 0.f, to_slip = finite ? fmaf(best_x, kLog2e, -to2) : 0.f;
      if (was != -INFINITY) shift_sums(fmaf(ref - best_x, kLog2e, to_slip - slip));
      ref = best_x; ref2 = to2; slip = to_slip;
    }
    float s = 0.f, u = 0.f;
    if (fabsf(ref) < kHuge) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float d = fmaxf(fmaf(y[i], kLog2e, -ref2), -1000.f), e = ex2_approx(d);    // (-inf: 0, and 0 in u)
        s += e;
        u = fmaf(d, e, u);
      }
    } else {                                                           // a row of the type's lowest value: it times log2e would be infinite
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float d = fmaxf(y[i] - ref, -1000.f) * kLog2e, e = ex2_approx(d);
        s += e;
        u = fmaf(d, e, u);
      }
    }
    sum += s;
    sum_u += u;
  }
  const bool odd = !(best_x < INFINITY);
  if (best_x != best_x) {                                              // NaN among them: the largest number, for the alternatives
    best_x = -INFINITY;
    for (int v = v0 + tid; v < v1; v += kThreads) {
      const uint4 w = fetch(row, v, off, end);
#pragma unroll
      for (int e = 0; e < V; ++e) best_x = fmaxf(best_x, element<T>(w, e));
    }
  }
  if (xt_nan) {                                                        // behind every number, and NaN of a lower index
    for (int v = v0 + tid; v < v1; v += kThreads)
      for (int i = max(v * V, off); i < min((v + 1) * V, end); ++i) n_before += (float)row[i] == (float)row[i] || i < token_at ? 1 : 0;
  }
  Part p = {best_x, 0.f, 0.f, 0u};
  if (best_x > -INFINITY) {
    shift_sums(fmaf(ref - best_x, kLog2e, -slip));                      // (2^-58 at the least)
    p.s = sum;
    p.u = sum_u * kLn2;
  }
  const uint32_t own_max = ordered(p.m);
  if (has_token && token_v >= v0 && token_v < v1 && tid == 0)          // equal ones ahead of the token in its own vector
    for (int i = max(token_v * V, off); i < token_at; ++i) n_before += (float)row[i] == xt ? 1 : 0;
  if (v0 == 0 && token_v > 0 && xt == -INFINITY && tid == 0) n_before -= off;            // what is not there counted as equal ones
  p.join_lanes(32);
  n_before = __reduce_add_sync(0xffffffffu, n_before);
  const bool any_odd = __any_sync(0xffffffffu, odd);
  const uint32_t warp_max = __reduce_max_sync(0xffffffffu, own_max), warp_min = __reduce_min_sync(0xffffffffu, own_max);
  if (lane == 0) { sm.part[warp] = p; sm.before[warp] = n_before; sm.odd[warp] = any_odd; sm.most[warp] = warp_max; sm.least[warp] = warp_min; }
  if (tid < kBins) sm.bins[0][tid] = 0;
  if (tid == 0) { sm.n_above = 0; sm.n_equal = 0; sm.n_holders = 0; }
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
    // a bound that at least k of the threads' maxima reach, and few more: by counting them in 64 bins between the least and the largest, then
    // again within the bin that holds the k-th, until that is near enough
    uint32_t from = max(__reduce_min_sync(0xffffffffu, sm.least[lane & (kWarps - 1)]), kLeastNumber);
    uint32_t to = max(__reduce_max_sync(0xffffffffu, sm.most[lane & (kWarps - 1)]), from);
    uint32_t bound = from;
    for (int round = 0, above = 0; ; ++round) {
      const int shift = max(0, 26 - __clz(to - from));
      if (tid < kBins) sm.bins[(round + 1) % 3][tid] = 0;
      int* bins = sm.bins[round % 3];
      if (own_max >= from && own_max <= to) atomicAdd(&bins[(own_max - from) >> shift], 1);
      __syncthreads();
      const int2 mine = reinterpret_cast<const int2*>(bins)[lane];
      int reach = mine.x + mine.y;                                      // in this lane's bins and all above them
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_down_sync(0xffffffffu, reach, o); if (lane + o < 32) reach += t; }
      const unsigned enough = __ballot_sync(0xffffffffu, above + reach >= k);
      if (enough == 0u) { bound = kLeastNumber; break; }                // fewer than k threads have a number: all that there are
      const int at = 31 - __clz(enough);
      const int here = __shfl_sync(0xffffffffu, reach, at), upper = __shfl_sync(0xffffffffu, mine.y, at), both = __shfl_sync(0xffffffffu, mine.x + mine.y, at);
      const bool in_upper = above + here - both + upper >= k;
      const int bin = 2 * at + (in_upper ? 1 : 0), inside = in_upper ? upper : both - upper;
      above += here - both + (in_upper ? 0 : upper);
      from += (uint32_t)bin << shift;
      to = min(to, from + ((1u << shift) - 1u));
      bound = from;
      if (shift == 0 || above + inside <= k + 12) break;
    }
    if (own_max >= bound) sm.holder[atomicAdd(&sm.n_holders, 1)] = (short)tid;
    __syncthreads();
    // the vectors of the threads that hold such a maximum, dealt to all threads (in little code: what runs once waits for its instructions)
    const int per = (v1 - v0 + kThreads - 1) / kThreads, n_read = sm.n_holders * per;
    for (;;) {
      const float reach = of_ordered(bound);
      auto look = [&](int v, const uint4& w) {
        float most = element<T>(w, 0);
#pragma unroll
        for (int e = 1; e < V; ++e) most = fmaxf(most, element<T>(w, e));
        if (!(most >= reach)) return;
#pragma unroll 1
        for (int at = max(v * V, off); at < min((v + 1) * V, end); ++at) {      // (few do)
          const uint32_t o = ordered((float)row[at]);
          if (o < bound) continue;
          if (o > bound) { const int to = atomicAdd(&sm.n_above, 1); if (to < kAbove) sm.above[to] = key_of(o, at); }
          else { const int to = atomicAdd(&sm.n_equal, 1); if (to < kEqual) sm.equal[to] = key_of(o, at); }
        }
      };
      if (per > 32) {                                                   // many vectors a thread: four on their way at a time
        for (int h = warp; h < sm.n_holders; h += kWarps) {
          const int first = v0 + sm.holder[h];
#pragma unroll 1
          for (int v = first + lane * kThreads; v < v1; v += 128 * kThreads) {
            uint4 w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = fetch(row, v + 32 * j * kThreads, off, v + 32 * j * kThreads < v1 ? end : 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) look(v + 32 * j * kThreads, w[j]);
          }
        }
      } else {
#pragma unroll 1
        for (int i = tid; i < n_read; i += kThreads) {
          const int h = i / per, v = v0 + sm.holder[h] + (i - h * per) * kThreads;
          look(v, fetch(row, v, off, v < v1 ? end : 0));
        }
      }
      __syncthreads();
      if (sm.n_above <= kAbove) break;
      // more than are kept: the k-th of those kept is a higher bound that k logits reach
#pragma unroll 1
      for (int c = tid; c < kAbove; c += kThreads) {
        const unsigned long long mine = sm.above[c];
        int place = 0;
#pragma unroll 1
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
            const uint4 w = fetch(row, v + lane, off, v + lane < v1 ? end : 0);
            uint32_t hits = 0u;
#pragma unroll
            for (int e = 0; e < V; ++e)
              hits |= (v + lane < v1 && (v + lane) * V + e >= off && (v + lane) * V + e < end && ordered(element<T>(w, e)) == wanted) ? 1u << e : 0u;
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
    for (int c = warp; c < n; c += kWarps) {
      const unsigned long long mine = c < n_above ? sm.above[c] : sm.equal[c - n_above];
      int place = 0;
#pragma unroll 1
      for (int i = lane; i < n; i += 32) place += (i < n_above ? sm.above[i] : sm.equal[i - n_above]) > mine ? 1 : 0;
      place = __reduce_add_sync(0xffffffffu, place);
      if (lane == 0 && place < k) sm.best[place] = mine;
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
        int lo[kMaxCluster], hi[kMaxCluster];
#pragma unroll
        for (int q = 0; q < kMaxCluster; ++q) { lo[q] = 0; hi[q] = q < C && q != c ? k : 0; }
#pragma unroll 1
        for (int step = 0; step < 6; ++step)                            // (of up to 32: side by side in all parts)
#pragma unroll
          for (int q = 0; q < kMaxCluster; ++q) {
            const int mid = (lo[q] + hi[q]) >> 1;
            const bool after = lo[q] < hi[q] && sm.best[q * kTop + min(mid, kTop - 1)] > mine;
            lo[q] = after ? mid + 1 : lo[q];
            hi[q] = after ? hi[q] : mid;
          }
        int place = j;
#pragma unroll
        for (int q = 0; q < kMaxCluster; ++q) place += lo[q];
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
    if (a.top_index != nullptr) a.top_index[(long long)row_i * k + tid] = 0x7fffffff - (int)(uint32_t)key - off;
    if (a.top_logprob != nullptr) a.top_logprob[(long long)row_i * k + tid] = logprob_of(of_ordered((uint32_t)(key >> 32)));
  }
}

template <typename T, bool kOff>
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
  return cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, kOff>, a) == cudaSuccess ? launched() : VS_ERR_CUDA;
}

}  // namespace

}  // namespace vs

extern "C" int vs_token_logprobs(const vs_scores* x, void* cuda_stream) {
  using namespace vs;
  if (x == nullptr || x->rows < 0 || x->vocab < 1 || x->dtype < 0 || x->dtype > 1 || x->top < 0) return VS_ERR_INVALID_ARG;
  if (x->vocab > (1 << 30) || x->rows > (1 << 27)) return VS_ERR_UNSUPPORTED;
  if (x->top > VS_MAX_TOP) return VS_ERR_CAPACITY;
  if (x->top > x->vocab) return VS_ERR_INVALID_ARG;
  if (x->rows == 0) return VS_OK;
  if (x->top > 0 && x->top_index == nullptr) return VS_ERR_INVALID_ARG;
  if ((x->logprob != nullptr || x->rank != nullptr) && x->tokens == nullptr) return VS_ERR_INVALID_ARG;
  const size_t el = x->dtype == 1 ? 4 : 2;
  if (x->logits == nullptr || !aligned(x->logits, el)) return VS_ERR_INVALID_ARG;
  const void* words[6] = {x->tokens, x->logprob, x->entropy, x->rank, x->top_index, x->top_logprob};
  for (const void* w : words) if (!aligned(w, 4)) return VS_ERR_INVALID_ARG;
  OnDevice on(x->device);
  if (!on.ok) return VS_ERR_CUDA;
  ScoreArgs a = {x->logits, x->tokens, x->logprob, x->entropy, x->top_logprob, x->rank, x->top_index, x->row_stride, x->rows, x->vocab, x->top, 1};
  // CTAs of a row, measured for rows of 5000 to 152064 logits (fp32, five alternatives).  A part of at least 4096 vectors keeps a CTA busy for longer
  // than joining the parts takes (one row of 32000: 7.9 us in one part, 9.0 in four; 64 rows of 5000 6.8, 11.3).  Eight parts up to eight rows (one
  // row of 152064: 17.0 us in one, 11.3 in four, 10.6 in eight; sixteen rows 17.3, 11.6, 14.0: clusters of eight wait for one another's places), four
  // while their CTAs are resident at once, two an SM (64 rows 21.7, 17.4; 100 rows 22.5, 30.0); then a CTA a row (197 rows 30.8 us in one, 39.9 in
  // two: 3.9 TB/s; 256 rows 33.3: 4.7 TB/s).
  const int vectors = (int)((x->vocab + 16 / el - 1) / (16 / el)), most = x->rows <= 8 ? 8 : (x->rows <= 74 ? 4 : 1);
  while (a.cluster < most && vectors >= 8192 * a.cluster) a.cluster *= 2;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool off = !aligned(x->logits, 16) || (x->rows > 1 && (x->row_stride * (int64_t)el) % 16 != 0);
  if (x->dtype == 1) return off ? launch<float, true>(a, st) : launch<float, false>(a, st);
  return off ? launch<bf16, true>(a, st) : launch<bf16, false>(a, st);
}
