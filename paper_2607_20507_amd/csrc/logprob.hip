// Log probabilities of given tokens under softmax(z / T), the entropy of each
// row and its n_top most likely tokens, for gfx950.
//
// With m the row's maximum, t_i = (z_i - m) / T, S = sum exp(t_i):
//   log p_i = t_i - log S,     H = log S - sum t_i exp(t_i) / S,
// both sums in one pass over the row with a running maximum (a new maximum m'
// with d = (m - m') / T turns (S, U = sum t exp t) into (e^d S, e^d (U + d S))).
// Every term of H is positive, so a peaked row loses nothing.  T = 0 is the
// point mass on the first maximum.  Two launches:
//   1. chunk   grid rows x chunks: statistics of a chunk and its n_top largest
//              logits, sorted
//   2. final   one workgroup per row: merges both
//
// The largest logits are ordered by a 64-bit key, the value (mapped to an
// integer of the same order) above the complement of the id, so that equal
// values go to the lower id and every key is different.  A workgroup keeps a
// threshold T that at least n_top elements reach and collects what passes it
// in LDS; the n_top-th largest of 256 disjoint subsets' maxima is such a
// threshold, and at most n_top subsets hold anything above it.  Masked logits
// (-inf) are never collected: where fewer than n_top remain, the final kernel
// appends the first masked ids.

#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

#include "common.h"
#include "logprob.h"

namespace spec {
namespace {

constexpr int kThreads = 256;
constexpr int kPerThread = 16;
constexpr int kStep = kThreads * kPerThread;  // elements between two looks at the collected keys
constexpr int kLimit = 512;                   // collected keys above this are thinned
constexpr int kCap = kStep + kLimit;
constexpr int kTargetBlocks = 2048;
constexpr int kMaxChunks = 64;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFloor = -200.f;  // exponents below this are 0 in fp32

struct LpStat {
  float m, s, u;  // maximum, sum 2^t, sum t 2^t (t in base 2)
  int32_t idx;    // of the first maximum
};

__device__ __forceinline__ uint64_t key_of(float v, int i) {
  const uint32_t b = __float_as_uint(v + 0.f);  // -0 counts as 0
  const uint32_t o = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
  return (static_cast<uint64_t>(o) << 32) | static_cast<uint32_t>(~i);
}
__device__ __forceinline__ float value_of(uint64_t k) {
  const uint32_t o = static_cast<uint32_t>(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}
__device__ __forceinline__ int id_of(uint64_t k) { return static_cast<int>(~static_cast<uint32_t>(k)); }

// 1 / T in base 2, finite and above 0, so that 0 and -inf times it stay what they
// are (T = 0, negative and NaN rows: any such factor)
__device__ __forceinline__ float base2_factor(float t) {
  return t > 0.f ? fmaxf(fminf(fminf(1.f / t, FLT_MAX) * kLog2e, FLT_MAX), __uint_as_float(1u)) : kLog2e;
}

__device__ __forceinline__ void stat_merge(LpStat& a, const LpStat& b, float c) {
  const float M = fmaxf(a.m, b.m);
  const float da = fmaxf((a.m - M) * c, kFloor), db = fmaxf((b.m - M) * c, kFloor);
  const float ea = exp2f(da), eb = exp2f(db);
  a.u = ea * (a.u + da * a.s) + eb * (b.u + db * b.s);
  a.s = ea * a.s + eb * b.s;
  if (b.m > a.m || (b.m == a.m && b.idx < a.idx)) a.idx = b.idx;
  a.m = M;
}

__device__ __forceinline__ LpStat wave_merge(LpStat v, float c) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    LpStat w;
    w.m = __shfl_xor(v.m, o, kWave);
    w.s = __shfl_xor(v.s, o, kWave);
    w.u = __shfl_xor(v.u, o, kWave);
    w.idx = __shfl_xor(v.idx, o, kWave);
    stat_merge(v, w, c);
  }
  return v;
}

// The collected keys of a workgroup.
struct Collect {
  alignas(16) uint64_t keys[kThreads];
  uint64_t buf[kCap];
  uint64_t t;
  int cnt;
};

// Number of the workgroup's keys above `mine` (every thread's key in s.keys).
__device__ __forceinline__ int rank_of(const Collect& s, uint64_t mine) {
  const ulonglong2* k2 = reinterpret_cast<const ulonglong2*>(s.keys);
  int r = 0;
#pragma unroll 16
  for (int i = 0; i < kThreads / 2; ++i) {
    const ulonglong2 v = k2[i];
    r += (v.x > mine) + (v.y > mine);
  }
  return r;
}

// s.t <- the n-th largest of the threads' keys (0: none), if there are n.
// Barriers on both sides.
__device__ __forceinline__ void raise_threshold(Collect& s, uint64_t mine, int n) {
  __syncthreads();
  s.keys[threadIdx.x] = mine;
  __syncthreads();
  if (mine != 0 && rank_of(s, mine) == n - 1) s.t = mine;
  __syncthreads();
}

// Thins the collected keys to at most kThreads, the n largest among them.
__device__ __forceinline__ void thin(Collect& s, int n) {
  constexpr int PER = (kCap + kThreads - 1) / kThreads;
  __syncthreads();
  int cnt = s.cnt;
  while (cnt > kThreads) {  // each turn leaves at most n ceil(cnt / 256) keys, n <= 64
    uint64_t own[PER], mx = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = i * kThreads + static_cast<int>(threadIdx.x);
      own[i] = e < cnt ? s.buf[e] : 0;
      mx = own[i] > mx ? own[i] : mx;
    }
    raise_threshold(s, mx, n);
    if (threadIdx.x == 0) s.cnt = 0;
    __syncthreads();
    const uint64_t t = s.t;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (own[i] != 0 && own[i] >= t) s.buf[atomicAdd(&s.cnt, 1)] = own[i];
    __syncthreads();
    cnt = s.cnt;
  }
}

template <bool VEC, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_chunk_kernel(int V, const float* __restrict__ logits, int64_t ld,
                                                                 const float* __restrict__ temps, int chunk,
                                                                 int n_chunks, int n_top, LpStat* __restrict__ stats,
                                                                 uint64_t* __restrict__ lists) {
  const int r = blockIdx.x / n_chunks, ch = blockIdx.x % n_chunks;
  const float* z = logits + static_cast<int64_t>(r) * ld;
  const float c = base2_factor(temps ? temps[r] : 1.f);
  const int beg = ch * chunk, end = min(V, beg + chunk);
  const int tid = threadIdx.x;
  __shared__ std::conditional_t<TOP, Collect, int> s;
  if constexpr (TOP) {
    if (tid == 0) {
      s.t = 0;
      s.cnt = 0;
    }
    __syncthreads();
  }
  // element e of the thread's 16 of a step: ids ascend with e
  auto id = [&](int base, int e) {
    return VEC ? base + (e / 4) * 4 * kThreads + 4 * tid + e % 4 : base + e * kThreads + tid;
  };
  LpStat st{-FLT_MAX, 0.f, 0.f, INT_MAX};
  float tv = -INFINITY;
  for (int base = beg; base < end; base += kStep) {
    float v[kPerThread];
    if (VEC && base + kStep <= end) {
#pragma unroll
      for (int q = 0; q < kPerThread / 4; ++q) {
        const float4 w = ld_stream(reinterpret_cast<const float4*>(z + id(base, 4 * q)));
        v[4 * q] = w.x; v[4 * q + 1] = w.y; v[4 * q + 2] = w.z; v[4 * q + 3] = w.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < kPerThread; ++e) v[e] = id(base, e) < end ? z[id(base, e)] : -INFINITY;
    }
    float vm = v[0];
#pragma unroll
    for (int e = 1; e < kPerThread; ++e) vm = fmaxf(vm, v[e]);
    int first = 0;
    if (vm > st.m || (TOP && base == beg)) {
#pragma unroll
      for (int e = kPerThread - 1; e >= 0; --e)
        if (v[e] == vm) first = e;
    }
    if (vm > st.m || (vm == st.m && st.idx == INT_MAX)) {
      const float d = fmaxf((st.m - vm) * c, kFloor), a = exp2f(d);
      st.u = a * (st.u + d * st.s);
      st.s *= a;
      st.m = vm;
      int fe = 0;
#pragma unroll
      for (int e = kPerThread - 1; e >= 0; --e)
        if (v[e] == vm) fe = e;
      st.idx = id(base, fe);
    }
#pragma unroll
    for (int e = 0; e < kPerThread; ++e) {
      const float t = (v[e] - st.m) * c;
      const float p = __builtin_amdgcn_exp2f(t);  // (a NaN stays one; a masked logit's p is 0)
      st.s += p;
      st.u = fmaf(fmaxf(t, kFloor), p, st.u);
    }
    if constexpr (TOP) {
      if (base == beg) {
        raise_threshold(s, vm > -INFINITY ? key_of(vm, id(base, first)) : 0, n_top);
        const uint64_t t = s.t;
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) {
          const uint64_t k = key_of(v[e], id(base, e));
          if (v[e] > -INFINITY && k >= t) s.buf[atomicAdd(&s.cnt, 1)] = k;
        }
        __syncthreads();
        tv = t ? value_of(t) : -INFINITY;
      } else {
        // n_top elements with lower ids are at least tv: an equal value here comes after them
        if (vm > tv) {
#pragma unroll
          for (int e = 0; e < kPerThread; ++e)
            if (v[e] > tv) s.buf[atomicAdd(&s.cnt, 1)] = key_of(v[e], id(base, e));
        }
        __syncthreads();
      }
      const bool many = s.cnt > kLimit;
      __syncthreads();  // nobody adds before everybody has looked
      if (many) {
        thin(s, n_top);
        tv = s.t ? value_of(s.t) : -INFINITY;
        __syncthreads();
      }
    }
  }
  st = wave_merge(st, c);
  __shared__ LpStat s_st[kThreads / kWave];
  if ((tid & (kWave - 1)) == 0) s_st[tid / kWave] = st;
  if constexpr (TOP) {
    thin(s, n_top);
    const int cnt = s.cnt;
    const uint64_t mine = tid < cnt ? s.buf[tid] : 0;
    __syncthreads();
    s.keys[tid] = mine;
    __syncthreads();
    uint64_t* out = lists + static_cast<size_t>(blockIdx.x) * n_top;
    if (mine != 0) {
      const int k = rank_of(s, mine);
      if (k < n_top) out[k] = mine;
    } else if (tid < n_top && tid >= cnt) {
      out[tid] = 0;
    }
  } else {
    __syncthreads();
  }
  if (tid == 0) {
    for (int w = 1; w < kThreads / kWave; ++w) stat_merge(st, s_st[w], c);
    stats[blockIdx.x] = st;
  }
}

template <bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_final_kernel(int V, const float* __restrict__ logits, int64_t ld,
                                                                 const float* __restrict__ temps,
                                                                 const int32_t* __restrict__ tokens, int n_chunks,
                                                                 int n_top, const LpStat* __restrict__ stats,
                                                                 const uint64_t* __restrict__ lists,
                                                                 float* __restrict__ logp, float* __restrict__ entropy,
                                                                 int32_t* __restrict__ top_ids,
                                                                 float* __restrict__ top_logp) {
  const int r = blockIdx.x, tid = threadIdx.x;
  const float* z = logits + static_cast<int64_t>(r) * ld;
  const float T = temps ? temps[r] : 1.f;
  const float c = base2_factor(T);
  // every wave merges the row's records (n_chunks <= 64)
  LpStat st{-FLT_MAX, 0.f, 0.f, INT_MAX};
  const int lane = tid & (kWave - 1);
  if (lane < n_chunks) st = stats[static_cast<size_t>(r) * n_chunks + lane];
  st = wave_merge(st, c);
  const bool ok = st.s > 0.f && st.m <= FLT_MAX && T >= 0.f;
  const float log_s = logf(st.s);
  auto log_p = [&](float v, int i) {
    if (!ok) return __builtin_nanf("");
    if (T == 0.f) return i == st.idx ? 0.f : -INFINITY;
    return (v - st.m) / T - log_s;
  };
  if (tid == 0) {
    if (logp) {
      const int t = tokens ? tokens[r] : -1;
      const bool in = t >= 0 && t < V;
      const float v = log_p(in ? z[t] : -INFINITY, t);
      logp[r] = in || !ok ? v : -INFINITY;
    }
    if (entropy) entropy[r] = !ok ? __builtin_nanf("") : T == 0.f ? 0.f : fmaxf(log_s - st.u * kLn2 / st.s, 0.f);
  }
  if constexpr (TOP) {
    int32_t* ids = top_ids + static_cast<size_t>(r) * n_top;
    float* lps = top_logp + static_cast<size_t>(r) * n_top;
    if (!ok) {
      if (tid < n_top) {
        ids[tid] = -1;
        lps[tid] = __builtin_nanf("");
      }
      return;
    }
    __shared__ Collect s;
    if (tid == 0) {
      s.t = 0;
      s.cnt = 0;
    }
    __syncthreads();
    const uint64_t* in = lists + static_cast<size_t>(r) * n_chunks * n_top;
    for (int e = tid; e < n_chunks * n_top; e += kThreads)
      if (in[e] != 0) s.buf[atomicAdd(&s.cnt, 1)] = in[e];
    thin(s, n_top);
    const int cnt = s.cnt;
    const uint64_t mine = tid < cnt ? s.buf[tid] : 0;
    __syncthreads();
    s.keys[tid] = mine;
    __syncthreads();
    if (mine != 0) {
      const int k = rank_of(s, mine);
      if (k < n_top) {
        ids[k] = id_of(mine);
        lps[k] = log_p(z[id_of(mine)], id_of(mine));
      }
    }
    // fewer than n_top logits are not masked: the first masked ids follow (n_top <= V)
    if (tid < kWave)
      for (int i0 = 0, found = cnt; found < n_top && i0 < V; i0 += kWave) {
        const bool masked = i0 + lane < V && z[i0 + lane] == -INFINITY;
        const uint64_t b = __ballot(masked);
        const int k = found + __popcll(b & ((1ull << lane) - 1));
        if (masked && k < n_top) {
          ids[k] = i0 + lane;
          lps[k] = -INFINITY;
        }
        found += __popcll(b);
      }
  }
}

inline size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

}  // namespace

LogprobPlan logprob_plan(int rows, int V, int n_top) {
  LogprobPlan p;
  p.rows = rows;
  p.V = V;
  p.n_top = n_top;
  int want = std::max(1, (kTargetBlocks + rows - 1) / std::max(1, rows));
  want = std::min(want, std::max(1, V / kStep));
  // at most kMaxChunks chunks, each a multiple of 1024 elements (16-byte loads)
  const int chunk = std::max((V + want - 1) / want, (V + kMaxChunks - 1) / kMaxChunks);
  p.chunk = (chunk + 1023) / 1024 * 1024;
  p.n_chunks = (V + p.chunk - 1) / p.chunk;
  return p;
}

size_t logprob_ws_bytes(const LogprobPlan& p) {
  const size_t n = static_cast<size_t>(p.rows) * p.n_chunks;
  return align256(sizeof(LpStat) * n) + align256(sizeof(uint64_t) * n * p.n_top);
}

hipError_t launch_logprobs(const LogprobPlan& p, const float* logits, int64_t ld, const float* temps,
                           const int32_t* tokens, float* logp, float* entropy, int32_t* top_ids, float* top_logp,
                           void* ws, hipStream_t st) {
  if (p.rows == 0) return hipSuccess;
  if (p.n_chunks > kMaxChunks || p.n_top > kLogprobMaxTop || static_cast<size_t>(p.rows) * p.n_chunks > kMaxGrid256)
    return hipErrorInvalidValue;
  LpStat* stats = static_cast<LpStat*>(ws);
  uint64_t* lists = reinterpret_cast<uint64_t*>(
      static_cast<char*>(ws) + align256(sizeof(LpStat) * static_cast<size_t>(p.rows) * p.n_chunks));
  const bool vec = reinterpret_cast<uintptr_t>(logits) % 16 == 0 && ld % 4 == 0;
  const bool top = p.n_top > 0;
  const auto chunk = vec ? (top ? logprob_chunk_kernel<true, true> : logprob_chunk_kernel<true, false>)
                         : (top ? logprob_chunk_kernel<false, true> : logprob_chunk_kernel<false, false>);
  launch_kernel(chunk, dim3(static_cast<uint32_t>(p.rows) * p.n_chunks), dim3(kThreads), 0, st, p.V, logits, ld,
                temps, p.chunk, p.n_chunks, p.n_top, stats, lists);
  const auto fin = top ? logprob_final_kernel<true> : logprob_final_kernel<false>;
  launch_kernel(fin, dim3(p.rows), dim3(kThreads), 0, st, p.V, logits, ld, temps, tokens, p.n_chunks, p.n_top,
                static_cast<const LpStat*>(stats), static_cast<const uint64_t*>(lists), logp, entropy, top_ids,
                top_logp);
  return hipGetLastError();
}

}  // namespace spec
