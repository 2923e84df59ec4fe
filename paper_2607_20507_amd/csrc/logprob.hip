// Log probabilities of given tokens under softmax(z / T), the entropy of each
// row and its n_top most likely tokens, for gfx950.
//
// With m the row's maximum, t_i = (z_i - m) / T, S = sum exp(t_i):
//   log p_i = t_i - log S,     H = log S - sum t_i exp(t_i) / S,
// both sums in one pass over the row with a running maximum (a new maximum m'
// with d = (m - m') / T turns (S, U = sum t exp t) into (e^d S, e^d (U + d S))).
// Every term of H is positive, so a peaked row loses nothing.  T = 0 is the
// point mass on the first maximum.
//
// HBM bound where there are many rows: 1792 x 128256 logits (919 MB) take 163 us a
// call, the chunks' kernel 156 (5.9 TB/s).  8 rows of 32000 are latency, 11.7 us: 7
// in the chunks' kernel (the votes' ballots one after another, the collection), 4 to 5
// in the final one (the ranking).  Two launches:
//   1. chunk   grid rows x chunks: statistics of a chunk and its n_top largest
//              logits, sorted
//   2. final   one workgroup per row: merges both
//
// The largest logits are ordered by a 64-bit key, the value (mapped to an
// integer of the same order) above the complement of the id, so that equal
// values go to the lower id and every key is different.  A workgroup keeps a
// value that at least n_top elements with lower ids reach and collects in LDS
// what is above it: the n_top-th largest of the threads' maxima so far, found by
// votes after steps 1, 2, 4, 8, 12, .. (20 of 128256 normal logits collect about
// 130 keys; with the first step's value alone 630, and a call of 1792 rows took
// 184 us, not 164).  Where many keys pile up all the same they are thinned to
// those above the n_top-th largest of 256 disjoint subsets' maxima, which at most
// n_top subsets are.  A chunk whose logits ascend can collect more than the buffer
// holds: it is then read once more in steps that cannot.  Masked logits (-inf) are
// never collected: where fewer than n_top remain, the final kernel appends the
// first masked ids.

#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

#include "common.h"
#include "logprob.h"

namespace spec {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kPerThread = 16;
constexpr int kStep = kThreads * kPerThread;
constexpr int kLook = 4;              // steps between two looks at the collected keys (1 and 2 at first)
constexpr int kLimit = 512;           // collected keys above this are thinned
constexpr int kCap = 2048;
constexpr int kSafeStep = kThreads * 4;  // a step of the second reading
static_assert(kSafeStep + kLimit <= kCap && kLogprobMaxTop * kPerThread <= kCap, "fits the buffer");
constexpr int kTargetBlocks = 2048;
constexpr int kMaxChunks = 64;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFloor = -200.f;  // exponents below this are 0 in fp32

struct LpStat {
  float m, s, u;  // maximum, sum 2^t, sum t 2^t (t in base 2)
  int32_t idx;    // of the first maximum
};

// Bits of v as an integer of the same order (-0 counts as 0).
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}
__device__ __forceinline__ uint64_t key_of(float v, int i) {
  return (static_cast<uint64_t>(ordered(v)) << 32) | static_cast<uint32_t>(~i);
}
__device__ __forceinline__ float value_of(uint64_t k) { return unordered(static_cast<uint32_t>(k >> 32)); }
__device__ __forceinline__ int id_of(uint64_t k) { return static_cast<int>(~static_cast<uint32_t>(k)); }

// (a - m) / 2: fp32 holds it where a - m passes the type's range, and it is as exact
// as that (but for values below 2^-126), in one instruction too.
__device__ __forceinline__ float half_diff(float a, float m) { return fmaf(a, 0.5f, -0.5f * m); }

// 2 / T in base 2 (for half_diff), finite and above 0, so that 0 and -inf times it
// stay what they are (T = 0, negative and NaN rows: any such factor)
__device__ __forceinline__ float base2_factor(float t) {
  return t > 0.f ? fmaxf(fminf(fminf(2.f / t, FLT_MAX) * kLog2e, FLT_MAX), __uint_as_float(1u)) : kLog2e;
}

__device__ __forceinline__ void stat_merge(LpStat& a, const LpStat& b, float c) {
  const float M = fmaxf(a.m, b.m);
  const float da = fmaxf(half_diff(a.m, M) * c, kFloor), db = fmaxf(half_diff(b.m, M) * c, kFloor);
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
  float reach[kWaves];
  int cnt, over;
};

__device__ __forceinline__ void collect(Collect& s, uint64_t key) {
  const int p = atomicAdd(&s.cnt, 1);
  if (p < kCap) s.buf[p] = key;
  else s.over = 1;
}

// Number of the first n (even) of s.keys above `mine`.
__device__ __forceinline__ int rank_of(const Collect& s, uint64_t mine, int n) {
  const ulonglong2* k2 = reinterpret_cast<const ulonglong2*>(s.keys);
  int r = 0;
#pragma unroll 4
  for (int i = 0; i < n / 2; ++i) {
    const ulonglong2 v = k2[i];
    r += (v.x > mine) + (v.y > mine);
  }
  return r;
}

// Thins the collected keys to at most kThreads, the n largest among them, and
// leaves in s.t a key that n of them reach.  Barriers on both sides.
__device__ __forceinline__ void thin(Collect& s, int n) {
  const int tid = threadIdx.x;
  __syncthreads();
  int cnt = min(s.cnt, kCap);
  __syncthreads();
  while (cnt > kThreads) {  // each turn leaves at most n ceil(cnt / 256) keys, n <= 64
    uint64_t mx = 0;
    for (int e = tid; e < cnt; e += kThreads) mx = s.buf[e] > mx ? s.buf[e] : mx;
    s.keys[tid] = mx;
    if (tid == 0) s.cnt = 0;
    __syncthreads();
    if (rank_of(s, mx, kThreads) == n - 1) s.t = mx;
    __syncthreads();
    const uint64_t t = s.t;
    // in place: a round's keys are read before any of them is written back, and
    // no more are written than were read
    for (int e0 = 0; e0 < cnt; e0 += kThreads) {
      const uint64_t k = e0 + tid < cnt ? s.buf[e0 + tid] : 0;
      __syncthreads();
      if (k >= t) s.buf[atomicAdd(&s.cnt, 1)] = k;
      __syncthreads();
    }
    cnt = s.cnt;
    __syncthreads();
  }
}

// The largest value to 16 leading bits that k lanes' values reach (-inf: none).
__device__ __forceinline__ float reached_by(float v, int k) {
  const uint32_t o = ordered(v);
  uint32_t t = 0;
#pragma unroll
  for (int b = 31; b >= 16; --b)
    if (__popcll(__ballot(o >= (t | (1u << b)))) >= k) t |= 1u << b;
  return t > 0x007FFFFFu ? unordered(t) : -INFINITY;
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
  const int tid = threadIdx.x, wave = tid / kWave;
  __shared__ std::conditional_t<TOP, Collect, int> s;
  if constexpr (TOP) {
    if (tid == 0) {
      s.t = 0;
      s.cnt = s.over = 0;
    }
    __syncthreads();
  }
  // element e of the thread's 16 of a step: ids ascend with e
  auto id = [&](int base, int e) {
    return VEC ? base + (e / 4) * 4 * kThreads + 4 * tid + e % 4 : base + e * kThreads + tid;
  };
  auto load = [&](int base, float (&v)[kPerThread]) {
    // (chunks are multiples of 1024 elements: whole rounds of 16-byte loads, but for a row's end)
#pragma unroll
    for (int q = 0; q < kPerThread / 4; ++q) {
      const int q0 = base + q * 4 * kThreads;
      if (VEC && q0 + 4 * kThreads <= end) {
        const float4 w = ld_stream(reinterpret_cast<const float4*>(z + id(base, 4 * q)));
        v[4 * q] = w.x; v[4 * q + 1] = w.y; v[4 * q + 2] = w.z; v[4 * q + 3] = w.w;
      } else {
#pragma unroll
        for (int e = 4 * q; e < 4 * q + 4; ++e) v[e] = id(base, e) < end ? z[id(base, e)] : -INFINITY;
      }
    }
  };
  // tv, or the value that n_top of the threads' values x reach if that is more:
  // each wave's share of them reaches its value, so all of them the least of those
  auto raise = [&](float x, float tv) {
    if constexpr (TOP) {
      const float w = reached_by(x, (n_top + kWaves - 1) / kWaves);
      __syncthreads();
      if ((tid & (kWave - 1)) == 0) s.reach[wave] = w;
      __syncthreads();
      static_assert(kWaves == 4, "one value a wave");
      tv = fmaxf(tv, fminf(fminf(s.reach[0], s.reach[1]), fminf(s.reach[2], s.reach[3])));
    }
    return tv;
  };
  LpStat st{-FLT_MAX, 0.f, 0.f, INT_MAX};
  float tv = -INFINITY;
  float v[kPerThread], next[kPerThread];
  load(beg, v);
  int i = 0;
  for (int base = beg; base < end; base += kStep, ++i) {
    if (base + kStep < end) load(base + kStep, next);
    float vm = v[0];
#pragma unroll
    for (int e = 1; e < kPerThread; ++e) vm = fmaxf(vm, v[e]);
    if (vm > st.m || (vm == st.m && st.idx == INT_MAX)) {
      const float d = fmaxf(half_diff(st.m, vm) * c, kFloor), a = exp2f(d);
      st.u = a * (st.u + d * st.s);
      st.s *= a;
      st.m = vm;
      int first = 0;
#pragma unroll
      for (int e = kPerThread - 1; e >= 0; --e)
        if (v[e] == vm) first = e;
      st.idx = id(base, first);
    }
#pragma unroll
    for (int e = 0; e < kPerThread; ++e) {
      const float t = half_diff(v[e], st.m) * c;
      const float p = __builtin_amdgcn_exp2f(t);  // (a NaN stays one; a masked logit's p is 0)
      st.s += p;
      st.u = fmaf(fmaxf(t, kFloor), p, st.u);
    }
    if constexpr (TOP) {
      // in the first step from a value that n_top elements of it reach
      if (i == 0) tv = raise(vm, tv);
      if (i == 0 ? vm >= tv : vm > tv) {  // (later an equal value comes after those that reach tv)
#pragma unroll
        for (int e = 0; e < kPerThread; ++e)
          if ((v[e] > tv || (i == 0 && v[e] == tv)) && v[e] > -INFINITY) collect(s, key_of(v[e], id(base, e)));
      }
      if ((i & (i + 1)) == 0 ? i > 0 : i % kLook == kLook - 1) {
        tv = raise(st.idx == INT_MAX ? -INFINITY : st.m, tv);
        const bool many = s.cnt > kLimit;
        __syncthreads();  // nobody adds before everybody has looked
        if (many) {
          thin(s, n_top);
          tv = fmaxf(tv, s.t ? value_of(s.t) : -INFINITY);
          __syncthreads();
        }
      }
    }
#pragma unroll
    for (int e = 0; e < kPerThread; ++e) v[e] = next[e];
  }
  if constexpr (TOP) {
    __syncthreads();
    if (s.over) {
      __syncthreads();
      if (tid == 0) {
        s.t = 0;
        s.cnt = s.over = 0;
      }
      tv = -INFINITY;
      __syncthreads();
      for (int base = beg; base < end; base += kSafeStep) {
        for (int e = 0; e < kSafeStep; e += kThreads) {
          const int j = base + e + tid;
          if (j < end && z[j] > tv) collect(s, key_of(z[j], j));
        }
        __syncthreads();
        const bool many = s.cnt > kLimit;
        __syncthreads();
        if (many) {
          thin(s, n_top);
          tv = s.t ? value_of(s.t) : -INFINITY;
          __syncthreads();
        }
      }
    }
  }
  st = wave_merge(st, c);
  __shared__ LpStat s_st[kWaves];
  if ((tid & (kWave - 1)) == 0) s_st[wave] = st;
  if constexpr (TOP) {
    thin(s, n_top);
    const int cnt = s.cnt;
    const uint64_t mine = tid < cnt ? s.buf[tid] : 0;
    s.keys[tid] = mine;
    __syncthreads();
    uint64_t* out = lists + static_cast<size_t>(blockIdx.x) * n_top;
    if (mine != 0) {
      const int k = rank_of(s, mine, (cnt + 1) & ~1);
      if (k < n_top) out[k] = mine;
    } else if (tid < n_top) {
      out[tid] = 0;  // (tid >= cnt)
    }
  } else {
    __syncthreads();
  }
  if (tid == 0) {
    for (int w = 1; w < kWaves; ++w) stat_merge(st, s_st[w], c);
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
  // every load that depends on nothing goes out first
  const uint64_t* in = lists + static_cast<size_t>(r) * n_chunks * n_top;
  constexpr int kOwn = kSafeStep / kThreads;
  uint64_t own[kOwn];
  auto load = [&](int e0) {
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int e = e0 + i * kThreads + tid;
      own[i] = e < n_chunks * n_top ? in[e] : 0;
    }
  };
  if constexpr (TOP) load(0);
  const int given = tokens ? tokens[r] : -1;
  const bool given_in = given >= 0 && given < V;
  const float z_given = given_in ? z[given] : -INFINITY;
  // every wave merges the row's records (n_chunks <= 64)
  LpStat st{-FLT_MAX, 0.f, 0.f, INT_MAX};
  const int lane = tid & (kWave - 1);
  if (lane < n_chunks) st = stats[static_cast<size_t>(r) * n_chunks + lane];
  st = wave_merge(st, c);
  // the butterfly's lanes round differently: one lane's result for all of them
  st.m = __shfl(st.m, 0, kWave);
  st.s = __shfl(st.s, 0, kWave);
  st.u = __shfl(st.u, 0, kWave);
  st.idx = __shfl(st.idx, 0, kWave);
  const bool ok = st.s > 0.f && st.m <= FLT_MAX && T >= 0.f;
  const float log_s = logf(st.s);
  auto log_p = [&](float v, int i) {
    if (!ok) return __builtin_nanf("");
    if (T == 0.f) return i == st.idx ? 0.f : -INFINITY;
    if (v == -INFINITY) return v;  // masked at T = inf too, where v / T is no number
    return 2.f * (half_diff(v, st.m) / T) - log_s;
  };
  if (tid == 0) {
    if (logp) {
      const float p = log_p(z_given, given);
      logp[r] = given_in || !ok ? p : -INFINITY;
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
    const int n_keys = n_chunks * n_top;
    uint64_t mine = own[0];
    int cnt = n_keys;
    // Up to a key per thread is ranked as it is (8 rows of 11 chunks of 5 keys 12.5
    // -> 11.7 us a call, 1792 of 2 chunks of 20 1.3 us less), more keys are thinned first.
    if (n_keys > kThreads) {
      if (tid == 0) {
        s.t = 0;
        s.cnt = s.over = 0;
      }
      __syncthreads();
      for (int e0 = 0; e0 < n_keys; e0 += kSafeStep) {
        if (e0 > 0) load(e0);
        uint64_t mx = s.t;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) mx = own[i] > mx ? own[i] : mx;
        // a value that n_top keys reach, as in the chunks (keys below it are not needed)
        const float w = reached_by(mx ? value_of(mx) : -INFINITY, (n_top + kWaves - 1) / kWaves);
        if (lane == 0) s.reach[tid / kWave] = w;
        __syncthreads();
        const uint64_t t = static_cast<uint64_t>(
            ordered(fminf(fminf(s.reach[0], s.reach[1]), fminf(s.reach[2], s.reach[3])))) << 32;
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
          if (own[i] > t) collect(s, own[i]);
        __syncthreads();
        const bool many = s.cnt > kLimit;
        __syncthreads();
        if (many) thin(s, n_top);
      }
      thin(s, n_top);
      cnt = s.cnt;
      mine = tid < cnt ? s.buf[tid] : 0;
    }
    s.keys[tid] = mine;
    const int held = __syncthreads_count(mine != 0);
    if (mine != 0) {
      const int k = rank_of(s, mine, (cnt + 1) & ~1);
      if (k < n_top) {
        ids[k] = id_of(mine);
        lps[k] = log_p(value_of(mine), id_of(mine));
      }
    }
    // fewer than n_top logits are not masked: the first masked ids follow (n_top <= V)
    if (tid < kWave)
      for (int i0 = 0, found = held; found < n_top && i0 < V; i0 += kWave) {
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
  // about kTargetBlocks workgroups, at least half a step each (with one a row, 8
  // rows of 128256 take 67 us, not 14, and 1792 rows 180, not 164)
  int want = std::max(1, (kTargetBlocks + rows - 1) / std::max(1, rows));
  want = std::min(want, std::max(1, V / (kStep / 2)));
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
