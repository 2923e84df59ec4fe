// Attention over a cache of latent vectors on gfx950: append, the products into
// and out of the latents' space, and the absorbed attention between them.

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "common.h"
#include "latent.h"
#include "latent_dev.h"

namespace spec {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

constexpr float kLatentRescaleLog2 = 8.f;

// Transposed read of 16-bit values: the 16 lanes 16 n .. give, four lanes a row, the
// addresses of 8 bytes each of a 4 x 16 block, and lane i receives its column i % 16.
__device__ __forceinline__ uint2 read_tr(uint32_t lds) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)lds));
}

__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

template <typename T>
__device__ __forceinline__ void put4(T* p, float a, float b, float c, float d) {
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2*>(p) = make_uint2(cvt_pk_bf16(a, b), cvt_pk_bf16(c, d));
  else
    *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
}
template <typename T>
__device__ __forceinline__ void put8(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(p) = make_uint4(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]),
                                              cvt_pk_bf16(v[6], v[7]));
  } else {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}
__device__ __forceinline__ void get8(const float* p, float (&v)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void get8(const bf16_t* p, float (&v)[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(u[i] << 16), v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
}

// ---------------------------------------------------------------------------
// Append: one workgroup per row and share of the heads.  A thread's unit is 8
// consecutive values (or 8 rotary pairs, whose halves are 8 consecutive values
// each).  The first share's first wave norms the latent: 8 values a lane.  Bound by
// HBM: 8192 rows of 32 heads move 330 MB in 54 to 56 us, 6 TB/s, more than a copy's 4.9: two
// bytes are read for each written.

template <typename T>
__global__ __launch_bounds__(256) void rope_latent_kernel(int H, int nope, int rope, int rank, float theta, float eps,
                                                          const float* __restrict__ q, const float* __restrict__ kv,
                                                          const T* __restrict__ norm_w, const int32_t* __restrict__ pos,
                                                          const int32_t* __restrict__ slot, uint32_t n_slots,
                                                          T* __restrict__ q_out, T* __restrict__ pages) {
  __shared__ float s_cos[32], s_sin[32];
  const int r = blockIdx.x, half = rope / 2, hq = nope + rope;
  const int h0 = static_cast<int>(static_cast<int64_t>(H) * blockIdx.y / gridDim.y);
  const int h1 = static_cast<int>(static_cast<int64_t>(H) * (blockIdx.y + 1) / gridDim.y);
  const float* qr = q + (static_cast<size_t>(r) * H + h0) * hq;
  T* o = q_out + (static_cast<size_t>(r) * H + h0) * hq;
  const uint32_t sl = static_cast<uint32_t>(slot[r]);
  const bool kept = sl < n_slots;  // (a negative slot is large)
  const float* x = kv + static_cast<size_t>(r) * (rank + rope);
  T* entry = pages + static_cast<size_t>(kept ? sl : 0) * (rank + rope);

  // the angles, in fp64, by the last threads
  const int ai = static_cast<int>(threadIdx.x) - (256 - half);
  if (ai >= 0) {
    double sn, cs;
    sincos(static_cast<double>(pos[r]) * exp(-(2.0 * ai / rope) * log(static_cast<double>(theta))), &sn, &cs);
    s_cos[ai] = static_cast<float>(cs);
    s_sin[ai] = static_cast<float>(sn);
  }
  if (blockIdx.y == 0 && threadIdx.x < kWave && kept) {
    const int e = 8 * static_cast<int>(threadIdx.x);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, w[8], ss = 0.f;
    if (e < rank) {
      get8(x + e, v);
      get8(norm_w + e, w);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = fmaf(v[j], v[j], ss);
    const float inv = 1.f / sqrtf(wave_sum(ss) / static_cast<float>(rank) + eps);
    if (e < rank) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = v[j] * inv * w[j];
      put8(entry + e, v);
    }
  }
  // the unrotated part
  const int un = nope / 8;
  for (int e = threadIdx.x; e < (h1 - h0) * un; e += 256) {
    const int at = e / un * hq + e % un * 8;
    float v[8];
    get8(qr + at, v);
    put8(o + at, v);
  }
  __syncthreads();
  // the rotated one, and the shared key as one more head
  const int ur = half / 8, own = blockIdx.y == 0 && kept ? 1 : 0;
  for (int e = threadIdx.x; e < (h1 - h0 + own) * ur; e += 256) {
    const int h = e / ur, i0 = e % ur * 8;
    const bool key = h == h1 - h0;
    const float* src = key ? x + rank : qr + h * hq + nope;
    T* dst = key ? entry + rank : o + h * hq + nope;
    float a[8], b[8], ra[8], rb[8];
    get8(src + i0, a);
    get8(src + half + i0, b);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float c = s_cos[i0 + j], sn = s_sin[i0 + j];
      ra[j] = a[j] * c - b[j] * sn;
      rb[j] = b[j] * c + a[j] * sn;
    }
    put8(dst + i0, ra);
    put8(dst + half + i0, rb);
  }
}

// Workgroup b's head and block of it, of `blocks` a head: consecutive workgroups go to
// the 8 XCDs in turn, so the blocks of a head, which read the same rows, are 8 apart and
// share an XCD's cache (384 rows of 32 heads, CT = 1: values 18 -> 13 us).
__device__ __forceinline__ int2 head_block(int b, int blocks, int H) {
  if (H % 8) return make_int2(b / blocks, b % blocks);
  const int i = b / 8;
  return make_int2(b % 8 + 8 * (i / blocks), i % blocks);
}

// The row, among all, of absorbed row i.
__device__ __forceinline__ int row_of(const LatentArgs& a, int i) { return a.row_list ? a.row_list[i] : i; }

// A call's tables, in a kernel's arguments.
struct Tables {
  uint4* to;
  uint32_t n;  // units
  uint4 unit[kLatentInline / 16];
};
struct NoTables {};
__device__ __forceinline__ void copy_tables(const NoTables&) {}
__device__ __forceinline__ void copy_tables(const Tables& t) {
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < t.n) t.to[threadIdx.x] = t.unit[threadIdx.x];
}
static_assert(kLatentInline % 16 == 0 && kLatentInline / 16 <= 256, "a unit a thread");

// ---------------------------------------------------------------------------
// Queries into the latents' space: q' [row, h, c] = sum_n q[row, h, n] w_k[h, n, c].
// A workgroup holds w_k's columns 64 cb .. of one head, a wave 16 CT of them as MFMA
// operands for its share of the rows: every fourth tile of 16 (CT = 4) or all (CT = 1,
// where there are too few tiles to share).

template <int NOPE, int CT, typename Tab>
__global__ __launch_bounds__(256) void latent_absorb_bf16_kernel(LatentArgs a, Tab tables) {
  copy_tables(tables);
  constexpr int KS = NOPE / 32;
  __shared__ uint4 sw[NOPE * 8];
  const int blocks = a.rank / 64;
  const int2 hb = head_block(blockIdx.x, blocks, a.H);
  const int h = hb.x, c0 = hb.y * 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, l16 = lane & 15;
  const bf16_t* w = static_cast<const bf16_t*>(a.w_k) + static_cast<int64_t>(h) * a.k_stride + c0;
  const bf16_t* q = static_cast<const bf16_t*>(a.q);
  bf16_t* to = static_cast<bf16_t*>(a.q_lat);
  const int hq = NOPE + a.rope, step = 16 * CT * gridDim.y;
  uint4 qf[KS], qn[KS];
  auto read = [&](int r0, uint4 (&x)[KS]) {
    const size_t from = (static_cast<size_t>(row_of(a, min(r0 + l16, a.R - 1))) * a.H + h) * hq;
#pragma unroll
    for (int s = 0; s < KS; ++s) x[s] = *reinterpret_cast<const uint4*>(q + from + 32 * s + 8 * g);
  };
  const int first = 16 * (CT * blockIdx.y + (CT == 4 ? wave : 0)), t0 = CT == 4 ? 0 : wave;  // rows, column tiles
  // row n's 16-byte chunks c at c ^ f(n): reads of four rows' 32 bytes, and writes, take every bank
  auto f = [](int n) { return (n & 3) << 1 | (n >> 2 & 1); };
#pragma unroll
  for (int i = 0; i < NOPE * 8 / 256; ++i) {
    const int u = i * 256 + threadIdx.x, n = u >> 3, c = u & 7;
    sw[n * 8 + (c ^ f(n))] = *reinterpret_cast<const uint4*>(w + static_cast<size_t>(n) * a.rank + 8 * c);
  }
  read(first, qf);
  __syncthreads();
  uint4 wf[CT][KS];
  const uint32_t base = lds_addr(sw);
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      uint2 p[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int n = 32 * s + 8 * g + 4 * t + (l16 >> 2), c = 2 * (t0 + ct) + (l16 >> 1 & 1);
        p[t] = read_tr(base + (n * 8 + (c ^ f(n))) * 16 + (l16 & 1) * 8);
      }
      wf[ct][s] = make_uint4(p[0].x, p[0].y, p[1].x, p[1].y);
    }
  for (int r0 = first; r0 < a.R; r0 += step) {
    read(r0 + step, qn);  // (past the last row: that row)
    const int r = r0 + l16;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) acc = mfma16x16x32(wf[ct][s], qf[s], acc);
      // (bf16: what the scores' products take)
      if (r < a.R)
        put4(to + (static_cast<size_t>(r) * a.H + h) * a.rank + c0 + 16 * (t0 + ct) + 4 * g, acc[0], acc[1], acc[2], acc[3]);
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = qn[s];
  }
}

template <int NOPE, typename Tab>
__global__ __launch_bounds__(256) void latent_absorb_f32_kernel(LatentArgs a, Tab tables) {
  copy_tables(tables);
  constexpr int J = NOPE / 16;
  const int blocks = a.rank / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, l16 = lane & 15;
  const int h = blockIdx.x / blocks, c0 = blockIdx.x % blocks * 64 + 16 * wave;
  const float* w = static_cast<const float*>(a.w_k) + static_cast<int64_t>(h) * a.k_stride + c0 + l16;
  // step (j, i) takes n = 16 j + 4 g + i in lane group g, so that a lane's q are float4s
  float wf[J][4];
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) wf[j][i] = w[static_cast<size_t>(16 * j + 4 * g + i) * a.rank];
  const float* q = static_cast<const float*>(a.q);
  float* to = static_cast<float*>(a.q_lat);
  const int hq = NOPE + a.rope;
  for (int r0 = 16 * blockIdx.y; r0 < a.R; r0 += 16 * gridDim.y) {
    const int r = r0 + l16, i0 = min(r, a.R - 1);
    const size_t qv = static_cast<size_t>(i0) * a.H + h, from = (static_cast<size_t>(row_of(a, i0)) * a.H + h) * hq;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    f32x4 qf[J];
#pragma unroll
    for (int j = 0; j < J; ++j) qf[j] = *reinterpret_cast<const f32x4*>(q + from + 16 * j + 4 * g);
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc = mfma_f32(wf[j][i], qf[j][i], acc);
    if (r < a.R) put4(to + qv * a.rank + c0 + 4 * g, acc[0], acc[1], acc[2], acc[3]);
  }
}

// ---------------------------------------------------------------------------
// Sums of latents to values: out[row, h, d] = sum_c o'[row, h, c] w_v[h, d, c].  A
// workgroup makes 16 CT dims of one head, its four waves a quarter of the sum each.

template <int RANK, int CT>
__global__ __launch_bounds__(256) void latent_values_bf16_kernel(LatentArgs a) {
  constexpr int KS = RANK / 128;
  __shared__ f32x4 part[2][4][CT][64];
  const int tiles = a.vdim / (16 * CT);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, l16 = lane & 15;
  const int2 hb = head_block(blockIdx.x, tiles, a.H);
  const int h = hb.x, d0 = hb.y * (16 * CT);
  const int c0 = wave * (RANK / 4) + 8 * g;
  const bf16_t* w = static_cast<const bf16_t*>(a.w_v) + static_cast<int64_t>(h) * a.v_stride +
                    static_cast<size_t>(d0 + l16) * RANK + c0;
  uint4 wf[CT][KS], of[KS], on[KS];
  const bf16_t* o = static_cast<const bf16_t*>(a.o_lat);
  bf16_t* out = static_cast<bf16_t*>(a.out);
  const int step = 16 * gridDim.y;
  auto read = [&](int r0, uint4 (&x)[KS]) {
    const size_t qv = static_cast<size_t>(min(r0 + l16, a.R - 1)) * a.H + h;
#pragma unroll
    for (int s = 0; s < KS; ++s) x[s] = *reinterpret_cast<const uint4*>(o + qv * RANK + c0 + 32 * s);
  };
  read(16 * blockIdx.y, of);
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int s = 0; s < KS; ++s) wf[ct][s] = *reinterpret_cast<const uint4*>(w + 16 * ct * RANK + 32 * s);
  int b = 0;
  for (int r0 = 16 * blockIdx.y; r0 < a.R; r0 += step, b ^= 1) {
    read(r0 + step, on);  // (past the last row: that row)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) acc = mfma16x16x32(wf[ct][s], of[s], acc);
      part[b][wave][ct][lane] = acc;
    }
    __syncthreads();  // (the other buffer's last readers passed the barrier before)
    const int r = r0 + l16;
    if (wave < CT && r < a.R) {
      const f32x4 acc = part[b][0][wave][lane] + part[b][1][wave][lane] + part[b][2][wave][lane] + part[b][3][wave][lane];
      put4(out + (static_cast<size_t>(row_of(a, r)) * a.H + h) * a.vdim + d0 + 16 * wave + 4 * g, acc[0], acc[1], acc[2], acc[3]);
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) of[s] = on[s];
  }
}

template <int RANK>
__global__ __launch_bounds__(256) void latent_values_f32_kernel(LatentArgs a) {
  constexpr int J = RANK / 64;
  __shared__ f32x4 part[4][64];
  const int tiles = a.vdim / 16;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, l16 = lane & 15;
  const int h = blockIdx.x / tiles, d0 = blockIdx.x % tiles * 16;
  const int c0 = wave * (RANK / 4) + 4 * g;
  const float* w = static_cast<const float*>(a.w_v) + static_cast<int64_t>(h) * a.v_stride +
                   static_cast<size_t>(d0 + l16) * RANK + c0;
  f32x4 wf[J];
#pragma unroll
  for (int j = 0; j < J; ++j) wf[j] = *reinterpret_cast<const f32x4*>(w + 16 * j);
  const float* o = static_cast<const float*>(a.o_lat);
  float* out = static_cast<float*>(a.out);
  for (int r0 = 16 * blockIdx.y; r0 < a.R; r0 += 16 * gridDim.y) {
    const int r = r0 + l16;
    const size_t qv = static_cast<size_t>(min(r, a.R - 1)) * a.H + h;
    f32x4 of[J];
#pragma unroll
    for (int j = 0; j < J; ++j) of[j] = *reinterpret_cast<const f32x4*>(o + qv * RANK + c0 + 16 * j);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc = mfma_f32(wf[j][i], of[j][i], acc);
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0 && r < a.R) {
      acc = part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane];
      put4(out + (static_cast<size_t>(row_of(a, r)) * a.H + h) * a.vdim + d0 + 4 * g, acc[0], acc[1], acc[2], acc[3]);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Joining a wave's or a part's state (raw maximum m, sum l, unnormalised o) with
// others': weight 2^((m - max m) scale).  A state that saw no key has m = -FLT_MAX
// and l = 0.  What is not finite stays so: a NaN anywhere, or a maximum of +inf,
// makes the row NaN; a row whose every score is -inf has l = 0 and becomes 0 / 0.

__device__ __forceinline__ float join_weight(float m, float top, float scale) {
  return __builtin_amdgcn_exp2f((m - top) * scale);
}

// The waves' states, in LDS as [WK][Q][RANK + 4] and [WK][Q][2], to the item's output.
template <typename T, int RANK, int WK, int Q, int THREADS>
__device__ __forceinline__ void join_waves(const LatentArgs& a, const LatentItem& it, const float* so, const float* sml,
                                           int tile) {
  constexpr int U = RANK / 4;
  for (int u = threadIdx.x; u < Q * U; u += THREADS) {
    const int m = u / U, c = u % U * 4;
    if (m >= it.nqv) break;
    float top = sml[2 * m];
#pragma unroll
    for (int k = 1; k < WK; ++k) top = fmaxf(top, sml[2 * (k * Q + m)]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll
    for (int k = 0; k < WK; ++k) {
      const float w = join_weight(sml[2 * (k * Q + m)], top, a.scale);
      l += w * sml[2 * (k * Q + m) + 1];
      o += w * *reinterpret_cast<const f32x4*>(so + (k * Q + m) * (RANK + 4) + c);
    }
    if (it.part < 0) {
      const float inv = 1.f / l;
      put4(static_cast<T*>(a.o_lat) + static_cast<size_t>(it.qv0 + m) * RANK + c, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    } else {
      const size_t pv = static_cast<size_t>(it.part) * tile + m;
      *reinterpret_cast<f32x4*>(a.part_o + pv * RANK + c) = o;
      if (c == 0) {
        a.part_ml[2 * pv] = top;
        a.part_ml[2 * pv + 1] = l;
      }
    }
  }
}

// One workgroup per query vector of a group and block of 1024 / PG columns: four columns
// a thread, the parts dealt to PG shares, whose sums are added in their order.  7616
// vectors of up to three parts 15 us (their sums, 40 MB, come from the caches); 32 vectors of 256 parts 6.4.
template <typename T, int RANK, int PG>
__global__ __launch_bounds__(256) void latent_combine_kernel(LatentArgs a, const LatentGroup* __restrict__ groups, int tile) {
  constexpr int CT = 256 / PG;  // threads along the columns
  static_assert(RANK % (4 * CT) == 0);
  __shared__ float s_w[kLatentMaxParts];
  __shared__ f32x4 s_o[PG][CT];
  __shared__ float s_red[4];
  const LatentGroup gr = groups[blockIdx.x / tile];
  const int m = blockIdx.x % tile;
  if (m >= gr.nqv) return;
  const int tid = threadIdx.x, ct = tid % CT, pg = tid / CT, c = blockIdx.y * (4 * CT) + 4 * ct;
  const float* ml = a.part_ml + 2 * (static_cast<size_t>(gr.part0) * tile + m);
  const float* po = a.part_o + (static_cast<size_t>(gr.part0) * tile + m) * RANK + c;
  // the first parts' sums are on their way while the weights are made
  constexpr int B = 8;
  f32x4 v[B];
#pragma unroll
  for (int b = 0; b < B; ++b)
    v[b] = *reinterpret_cast<const f32x4*>(po + static_cast<size_t>(min(pg + b * PG, gr.nparts - 1)) * tile * RANK);
  float top = -FLT_MAX;
  for (int p = tid; p < gr.nparts; p += 256) top = fmaxf(top, ml[static_cast<size_t>(2) * tile * p]);
  top = wave_max(top);
  if ((tid & 63) == 0) s_red[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
  __syncthreads();
  float l = 0.f;
  for (int p = tid; p < gr.nparts; p += 256) {
    const float w = join_weight(ml[static_cast<size_t>(2) * tile * p], top, a.scale);
    s_w[p] = w;
    l += w * ml[static_cast<size_t>(2) * tile * p + 1];
  }
  l = wave_sum(l);
  if ((tid & 63) == 0) s_red[tid >> 6] = l;
  __syncthreads();
  l = s_red[0] + s_red[1] + s_red[2] + s_red[3];
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = pg; p0 < gr.nparts; p0 += B * PG) {
#pragma unroll
    for (int b = 0; b < B; ++b)
      if (p0 + b * PG < gr.nparts) o += s_w[p0 + b * PG] * v[b];
    if (p0 + B * PG < gr.nparts) {
#pragma unroll
      for (int b = 0; b < B; ++b)
        v[b] = *reinterpret_cast<const f32x4*>(po + static_cast<size_t>(min(p0 + (B + b) * PG, gr.nparts - 1)) * tile * RANK);
    }
  }
  s_o[pg][ct] = o;
  __syncthreads();
  if (pg) return;
#pragma unroll
  for (int i = 1; i < PG; ++i) o += s_o[i][ct];
  const float inv = 1.f / l;
  put4(static_cast<T*>(a.o_lat) + static_cast<size_t>(gr.qv0 + m) * RANK + c, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
}

// ---------------------------------------------------------------------------
// Absorbed attention, bf16.  A workgroup holds 16 WQ query vectors of one
// sequence; its four waves are WQ shares of them times WK shares of the keys.  32
// keys at a time go to LDS (direct loads of their two pages), where the waves of a
// share read them twice: as rows for S^T = C Q'^T (A = 16 keys x 32 dims), and
// transposed for O'^T = C^T P^T (A = 16 dims x 32 keys).  The transposed reads take
// the keys in the order in which a lane's score accumulators hold them, so the
// probabilities go from one product to the other in registers.
// Chunks of 16 bytes of token t's latent sit at c ^ f(t): the 8 lanes of a row read
// (8 tokens, one chunk: 128 bytes) and the 32 of a transposed one (8 tokens, two
// chunks: 256 bytes) take every bank once.
// The running maximum (of raw scores) is raised only when a score exceeds it by more
// than 2^8; differences are taken before the scale, so scores of any size keep theirs.
// The queries in the latents' space, the probabilities and the sums that go on to w_v are
// rounded to bf16, as the cache and the weights are: the matrix instructions take
// nothing wider, and a second bf16 part of the sums alone would double what the values'
// kernel reads to take a row's error from 0.0031 to 0.0026.
// What bounds it: tiles of 64 (64 sequences, 384 rows of 32 heads over 512 .. 4096 keys,
// 73 us) that a chunk's scores, softmax and sums take turns: of the cycles in which a CU
// holds waves LDS is in use 38% (the second product's reads feed one 16-row product each),
// MFMA 36%, vector instructions 24%; tiles of 32 (one row over 131001 keys, 33 us) HBM, 151 MB
// at 4.6 TB/s; short contexts the chain of a chunk's loads, two products and softmax, about 2 us,
// and that few CUs have one: 6 rows of 32 heads over 2053 keys (17 us) are 51 workgroups of four
// chunks in turn, MFMA busy 13% and waves waiting 36% of their time.  A tile of 16 has one buffer a
// key share, whose next loads leave when its chunk is done: 8 sequences of 256 .. 512 keys (rank
// 256, 12 us) wait half of the time.
// Two workgroups a CU (WK = 1) leave 256 registers a wave: rank 512 spills 12 (32 rotated dims)
// or 15, of which the second kind reads one again in the keys' loop.
// A key that some row does not see may hold a value that is not finite (a slot past the
// sequence anything at all), whose product with the row's probability 0 would be NaN.
// So chunks with such keys are cleaned in LDS between the two products: values that
// are not finite become 0, and the rows that do see their key get a NaN score.

template <int RANK, int ROPE, int WQ, int WK>
__global__ __launch_bounds__(256, WK == 1 ? 2 : 1) void attn_latent_bf16_kernel(LatentArgs a, const LatentItem* __restrict__ items) {
  constexpr int CL = RANK / 8, CR = ROPE / 8;    // 16-byte chunks of a token's latent and key
  constexpr int DL = RANK / 32, DR = ROPE / 32;  // k-steps of the scores
  constexpr int DT = RANK / 16;                  // 16-dim output tiles
  constexpr int NB = WK == 4 ? 1 : 2;            // chunk buffers of a key share
  constexpr int PD = WK == 1 ? 4 : 8;            // operands read ahead (two workgroups a CU leave fewer registers)
  constexpr int BU = 32 * (CL + CR);             // 16-byte units of a chunk
  constexpr int Q = 16 * WQ;
  constexpr int TP = 64 / CL, RT = 64 / CR;      // tokens a load covers: latents, keys
  constexpr int NLL = 32 / TP, NL = NLL + 32 / RT;  // loads of a chunk: its latents', all
  constexpr int kEntry = (CL + CR) * 16;
  constexpr int kJoin = WK > 1 ? WK * Q * (RANK + 4) * 4 / 16 : 0;
  constexpr int kUnits = WK * NB * BU > kJoin ? WK * NB * BU : kJoin;
  static_assert(WQ * WK == 4 && NLL % WQ == 0);
  __shared__ __attribute__((aligned(256))) uint4 buf[kUnits];
  __shared__ float s_ml[WK > 1 ? 2 * WK * Q : 1];
  __shared__ uint32_t s_flag[4];
  const LatentItem it = items[blockIdx.x];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wq = wave % WQ, wk = wave / WQ;
  const int g = lane >> 4, l16 = lane & 15;
  const char* pool = static_cast<const char*>(a.pages);
  const int32_t* list = a.page_list + it.page0;
  const int np = (it.t1 + 15) >> 4;
  const int c0 = it.t0 >> 5, nch = (it.t1 - it.t0 + 31) >> 5;
  const int nit = (nch + WK - 1) / WK;
  auto f = [](int t) { return (t & 7) << 1 | (t >> 2 & 1); };
  auto fr = [&](int t) { return CR == 8 ? (t & 3) << 1 | (t >> 2 & 1) : t >> 1 & 3; };

  // page ids, 64 (of 32 chunks) in a wave's lanes, the next 64 asked for ahead; past the
  // item's last page it stands for the others
  int cp = c0;  // the chunk of lanes 0 and 1
  int32_t ids = list[min(2 * c0 + lane, np - 1)], ids_next = list[min(2 * c0 + 64 + lane, np - 1)];
  // lane offsets of the loads
  const uint32_t ld_lat = (lane % CL ^ (TP == 2 ? (lane >> 5) * 2 : 0)) * 16;
  const uint32_t ld_key = lane / CR * kEntry + (CL + (lane % CR ^ fr(lane / CR))) * 16;
  auto buffer = [&](int b) { return lds_addr(&buf[(wk * NB + b) * BU]); };  // (a multiple of 256)
  // the wave's loads of chunk c into buffer b
  auto issue = [&](int c, int b) {
    if (c >= cp + 32) {
      cp += 32;
      ids = ids_next;
      ids_next = list[min(2 * cp + 64 + lane, np - 1)];
    }
    size_t page[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      page[i] = static_cast<size_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(ids, 2 * (c - cp) + i))) * (16 * kEntry);
#pragma unroll
    for (int j = 0; j < (NL + WQ - 1) / WQ; ++j) {
      const int i = WQ * j + wq;
      if (NL % WQ != 0 && i >= NL) break;
      const bool key = WQ * j >= NLL;
      const int first = key ? (i - NLL) * RT : i * TP;
      const char* base = pool + (first >> 4 ? page[1] : page[0]) + (first & 15) * kEntry;
      // (f of a load's second token, first + 1, is f(first) ^ 2)
      uint32_t at;
      if (key) at = ld_key;
      else if (TP == 1) at = xor_here(ld_lat, f(first) * 16);
      else at = xor_here(ld_lat, f(first) * 16) + (lane >> 5) * kEntry;
      load_lds16(base, at, buffer(b) + i * 1024);
    }
  };

  // the lane's query vector
  const int m = 16 * wq + l16;
  const bool ok = m < it.nqv;
  auto pos_of = [&](int i) { return it.pos0 + (it.qv0 + i) / a.H - it.row0; };
  const int klim = ok ? min(pos_of(m), it.t1 - 1) : -1;  // the last key it sees (-1: none, padding)
  const int pos_lo = pos_of(0);
  uint4 qf[DL + DR];
  {
    const size_t qv = static_cast<size_t>(it.qv0 + (ok ? m : 0));
    const bf16_t* ql = static_cast<const bf16_t*>(a.q_lat) + qv * RANK + 8 * g;
    const bf16_t* qr = static_cast<const bf16_t*>(a.q) + (qv + static_cast<size_t>(it.qoff) * a.H) * (a.nope + ROPE) + a.nope + 8 * g;
#pragma unroll
    for (int s = 0; s < DL + DR; ++s)
      qf[s] = ok ? *reinterpret_cast<const uint4*>(s < DL ? ql + 32 * s : qr + 32 * (s - DL)) : make_uint4(0, 0, 0, 0);
  }
  float mneg = FLT_MAX, mlim = -INFINITY, lrun[2] = {0.f, 0.f};
  f32x4 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    asm volatile("" : "+a"(acc[dt]));
  }

  // lane constants of the reads
  // (of a k-step's or output tile's number, the bits that f changes are an exclusive or of the address)
  const uint32_t k_off = l16 * (CL * 16) + ((g ^ f(l16)) * 16);
  const int tv = 4 * g + (l16 >> 2);
  const uint32_t v_off = tv * (CL * 16) + (((l16 >> 1 & 1) ^ f(tv)) * 16) + (l16 & 1) * 8;
  const uint32_t r_off = l16 * (CR * 16) + (g ^ fr(l16)) * 16;
  typedef __attribute__((address_space(3))) const u32x4* lds_units;
  auto unit_at = [](uint32_t lds) { return __builtin_bit_cast(uint4, *(lds_units)(uintptr_t)lds); };

  // Both products read their operands PD ahead: read earlier, as the compiler would,
  // they take registers that there are not.
  uint4 ring[PD];
  f32x4 sc[2];
  // one chunk, c, in buffer b; masked: some row of the workgroup does not see some key of the step's chunks
  auto chunk = [&](int c, int b, bool masked) {
    {
      uint32_t ka[4] = {buffer(b) + k_off}, rb = buffer(b) + 32 * CL * 16 + r_off;
#pragma unroll
      for (int i = 1; i < 4; ++i) ka[i] = xor_here(ka[0], i * 64);
      auto read_k = [&](int u) {  // k-step u / 2 of key tile u % 2
        const int s = u >> 1, hh = u & 1;
        if (s < DL) return unit_at(ka[s & 3] + (s >> 2) * 256 + hh * (16 * CL * 16));
        return unit_at((s > DL ? xor_here(rb, 64) : rb) + hh * (16 * CR * 16));
      };
      f32x4 x[2];
#pragma unroll
      for (int u = 0; u < PD; ++u) ring[u] = read_k(u);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < 2 * (DL + DR); ++u) {
        if (u < 2) x[u] = mfma_first_v(ring[u % PD], qf[u >> 1]);
        else mfma_in_place_v(ring[u % PD], qf[u >> 1], x[u & 1]);
        if (u + PD < 2 * (DL + DR)) ring[u % PD] = read_k(u + PD);
        __builtin_amdgcn_sched_barrier(0);
      }
      sums_ready();
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        asm volatile("" : "+v"(x[hh]));  // (in its place until here)
        sc[hh] = x[hh];
      }
    }
    if (masked) {
      asm volatile("");
      uint4* lat = &buf[(wk * NB + b) * BU];
      if (WQ > 1) {
        SPEC_WAIT_VM_LDS(63);
        block_sync();  // every wave of the share has its scores
      }
      uint32_t flags = 0;  // of the chunk's keys: a latent that is not finite
#pragma unroll 1
      for (int i = wq; i < NLL; i += WQ) {
        const uint4 v = lat[64 * i + lane];
        const uint64_t bad = __ballot((nonfinite_bits(v.x) | nonfinite_bits(v.y) | nonfinite_bits(v.z) | nonfinite_bits(v.w)) != 0);
        if (bad == 0) continue;
        lat[64 * i + lane] = drop_nonfinite(v);
        if (TP == 1) flags |= 1u << i;
        else flags |= (static_cast<uint32_t>(bad) ? 1u : 0u) << (2 * i) | (bad >> 32 ? 2u : 0u) << (2 * i);
      }
      if (WQ > 1) {
        if (lane == 0) s_flag[wave] = flags;
        SPEC_WAIT_VM_LDS(63);
        block_sync();
#pragma unroll
        for (int i = 0; i < WQ; ++i) flags |= s_flag[wk * WQ + i];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = 16 * (j / 4) + 4 * g + j % 4;
        if (32 * c + k > klim) sc[j / 4][j % 4] = -INFINITY;
        else if (flags >> k & 1) sc[j / 4][j % 4] = __builtin_nanf("");
      }
    }
    // the second product's first operands are on their way during the softmax
    uint32_t va[8] = {buffer(b) + v_off};
#pragma unroll
    for (int i = 1; i < 8; ++i) va[i] = xor_here(va[0], i * 32);
    auto read_v = [&](int dt) {
      const uint32_t at = va[dt & 7] + (dt >> 3) * 256;
      const uint2 x = read_tr(at), y = read_tr(at + 16 * RANK * 2);
      return make_uint4(x.x, x.y, y.x, y.y);
    };
#pragma unroll
    for (int u = 0; u < PD; ++u) ring[u] = read_v(u);
    float top = sc[0][0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, sc[j / 4][j % 4]);
    if (__any(top > mlim)) {
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      float alpha = 1.f;
      if (top > mlim) {
        alpha = __builtin_amdgcn_exp2f((-mneg - top) * a.scale);
        mneg = -top;
        mlim = top + kLatentRescaleLog2 / a.scale;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) lrun[i] *= alpha;
      sums_ready();
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) scale_in_place(acc[dt], alpha);
    }
    float p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f((sc[j / 4][j % 4] + mneg) * a.scale);
#pragma unroll
    for (int j = 0; j < 8; ++j) lrun[j % 2] += p[j];
    // bf16, as the values that they weight: the rounding stays below the output's
    const uint4 pf = make_uint4(cvt_pk_bf16(p[0], p[1]), cvt_pk_bf16(p[2], p[3]), cvt_pk_bf16(p[4], p[5]), cvt_pk_bf16(p[6], p[7]));
    operands_ready();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      mfma_in_place(ring[dt % PD], pf, acc[dt]);
      if (dt + PD < DT) ring[dt % PD] = read_v(dt + PD);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // (a share's chunk past the last is loaded from the last page, and masked)
  if (NB == 2) issue(c0 + wk, 0);
  for (int j = 0; j < nit; ++j) {
    const int c = c0 + j * WK + wk, b = NB == 2 ? j & 1 : 0;
    if (NB == 2) {
      SPEC_WAIT_VM_LDS(0);
      block_sync();  // chunk j has landed, and every wave is done with the one before
      if (j + 1 < nit) issue(c + WK, (j + 1) & 1);
    } else {  // a buffer of the wave's own
      SPEC_WAIT_VM_LDS(0);
      wave_fence();
      issue(c, 0);
      SPEC_WAIT_VM_LDS(0);
      wave_fence();
    }
    const int last = 32 * (c0 + (j + 1) * WK) - 1;  // (the same for every share: a masked chunk has barriers)
    chunk(c, b, last > pos_lo || last >= it.t1);
  }

  sums_ready(acc);
  float l = lrun[0] + lrun[1];
  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
  if constexpr (WK == 1) {
    if (!ok) return;
    if (it.part < 0) {
      const float inv = 1.f / l;
      bf16_t* o = static_cast<bf16_t*>(a.o_lat) + static_cast<size_t>(it.qv0 + m) * RANK + 4 * g;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const f32x4 v = acc[dt] * inv;
        put4(o + 16 * dt, v[0], v[1], v[2], v[3]);
      }
    } else {
      const size_t pv = static_cast<size_t>(it.part) * Q + m;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(a.part_o + pv * RANK + 16 * dt + 4 * g) = acc[dt];
      if (g == 0) {
        a.part_ml[2 * pv] = -mneg;
        a.part_ml[2 * pv + 1] = l;
      }
    }
  } else {
    __syncthreads();  // every wave is done with its keys
    float* so = reinterpret_cast<float*>(buf);
    const int at = wk * Q + m;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(so + at * (RANK + 4) + 16 * dt + 4 * g) = acc[dt];
    if (g == 0) {
      s_ml[2 * at] = -mneg;
      s_ml[2 * at + 1] = l;
    }
    __syncthreads();
    join_waves<bf16_t, RANK, WK, Q, 256>(a, it, so, s_ml, Q);
  }
}

// ---------------------------------------------------------------------------
// Absorbed attention, fp32: 16 query vectors a workgroup, whose waves take its pages in
// turn: eight, four where registers allow no more.  What bounds it is waiting for the cache: a
// page's 34 loads (rank 256) are asked for one ahead of their use, a chain of some 17 answers, and
// the next page's id behind them.  5 rows of 4 heads over 133 keys take 17 us in two workgroups
// whose waves have one page or two: they wait 62% of their time, and their pages' MFMAs, 136 of 32
// cycles each, are 13% of it (asking for a page's values before its softmax 17.4).  One row of 4 heads
// over 30000 keys is 34 us a call where the bytes take 7, 1024 rows of 16 heads behind 3000 keys 742
// where the flops take 146.
// fp32 MFMA throughout (16 x 16 x 4), operands straight from the cache: k-step (j, i)
// of the scores takes dim 16 j + 4 g + i in lane group g, and output tile (j, t) holds
// dims 64 j + 4 row + t, so that every load is 16 bytes a lane and a lane's scores are
// the probabilities it supplies.

template <int RANK, int ROPE>
__global__ __launch_bounds__(64 * latent_f32_waves(RANK), 1) void attn_latent_f32_kernel(LatentArgs a, const LatentItem* __restrict__ items) {
  constexpr int D = RANK + ROPE, J = D / 16, JV = RANK / 64;
  constexpr int WK = latent_f32_waves(RANK), Q = 16;
  __shared__ float so[WK * Q * (RANK + 4)];
  __shared__ float s_ml[2 * WK * Q];
  const LatentItem it = items[blockIdx.x];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  const float* pool = static_cast<const float*>(a.pages);
  const int32_t* list = a.page_list + it.page0;
  const bool ok = l16 < it.nqv;
  const size_t qv = static_cast<size_t>(it.qv0 + (ok ? l16 : 0));
  auto pos_of = [&](int m) { return it.pos0 + (it.qv0 + m) / a.H - it.row0; };
  const int klim = ok ? min(pos_of(l16), it.t1 - 1) : -1;
  const int pos_lo = pos_of(0), pos_hi = min(pos_of(it.nqv - 1), it.t1 - 1);
  f32x4 qf[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const float* src = 16 * j < RANK ? static_cast<const float*>(a.q_lat) + qv * RANK + 16 * j
                                     : static_cast<const float*>(a.q) + (qv + static_cast<size_t>(it.qoff) * a.H) * (a.nope + ROPE) + a.nope + 16 * j - RANK;
    qf[j] = ok ? *reinterpret_cast<const f32x4*>(src + 4 * g) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  float mneg = FLT_MAX, mlim = -INFINITY, lrun = 0.f;
  f32x4 acc[4 * JV];
#pragma unroll
  for (int i = 0; i < 4 * JV; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int t0 = it.t0 + 16 * wave; t0 <= pos_hi; t0 += 16 * WK) {
    const float* page = pool + static_cast<size_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(list[t0 >> 4]))) * (16 * D);
    f32x4 sc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const f32x4 k = *reinterpret_cast<const f32x4*>(page + l16 * D + 16 * j + 4 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[i & 1] = mfma_f32(k[i], qf[j][i], sc[i & 1]);
    }
    f32x4 s = sc[0] + sc[1];
    const float* vrow = page + 4 * g * D + 4 * l16;  // keys 4 g + i
    bool bad = false;
    if (t0 + 15 > pos_lo || t0 + 15 >= it.t1) {
      bool odd = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) odd |= !finite(s[i]);
      bad = __any(odd);
      uint32_t flags = 0;
      if (bad) {
#pragma unroll 1
        for (int i = 0; i < 4; ++i)
#pragma unroll 1
          for (int j = 0; j < JV; ++j) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(vrow + i * D + 64 * j);
            if (!(finite(v[0]) && finite(v[1]) && finite(v[2]) && finite(v[3]))) flags |= 1u << i;
          }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) flags |= __shfl_xor(flags, o, kWave);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (t0 + 4 * g + i > klim) s[i] = -INFINITY;
        else if (flags >> i & 1) s[i] = __builtin_nanf("");
      }
    }
    float m = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    if (__any(m > mlim)) {
      m = fmaxf(m, __shfl_xor(m, 16, kWave));
      m = fmaxf(m, __shfl_xor(m, 32, kWave));
      if (m > mlim) {
        const float alpha = __builtin_amdgcn_exp2f((-mneg - m) * a.scale);
        mneg = -m;
        mlim = m + kLatentRescaleLog2 / a.scale;
        lrun *= alpha;
#pragma unroll
        for (int i = 0; i < 4 * JV; ++i) acc[i] *= alpha;
      }
    }
    f32x4 p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[i] = __builtin_amdgcn_exp2f((s[i] + mneg) * a.scale);
      lrun += p[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < JV; ++j) {
        f32x4 v = *reinterpret_cast<const f32x4*>(vrow + i * D + 64 * j);
        if (bad) {
#pragma unroll
          for (int t = 0; t < 4; ++t) v[t] = finite(v[t]) ? v[t] : 0.f;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[4 * j + t] = mfma_f32(v[t], p[i], acc[4 * j + t]);
      }
  }
  lrun += __shfl_xor(lrun, 16, kWave);
  lrun += __shfl_xor(lrun, 32, kWave);
  const int at = wave * Q + l16;
#pragma unroll
  for (int j = 0; j < JV; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *reinterpret_cast<f32x4*>(so + at * (RANK + 4) + 64 * j + 16 * g + 4 * r) =
          f32x4{acc[4 * j][r], acc[4 * j + 1][r], acc[4 * j + 2][r], acc[4 * j + 3][r]};
  if (g == 0) {
    s_ml[2 * at] = -mneg;
    s_ml[2 * at + 1] = lrun;
  }
  __syncthreads();
  join_waves<float, RANK, WK, Q, 64 * WK>(a, it, so, s_ml, Q);
}

template <int RANK, int ROPE>
hipError_t launch_attention(const LatentArgs& a, const LatentItem* items, int n, int tile, hipStream_t st) {
  if (a.dtype == 0) {
    if (tile != 16) return hipErrorInvalidValue;
    launch_kernel(attn_latent_f32_kernel<RANK, ROPE>, dim3(n), dim3(64 * latent_f32_waves(RANK)), 0, st, a, items);
  } else if (tile == 16) {
    launch_kernel(attn_latent_bf16_kernel<RANK, ROPE, 1, 4>, dim3(n), dim3(256), 0, st, a, items);
  } else if (tile == 32) {
    launch_kernel(attn_latent_bf16_kernel<RANK, ROPE, 2, 2>, dim3(n), dim3(256), 0, st, a, items);
  } else if (tile == 64) {
    launch_kernel(attn_latent_bf16_kernel<RANK, ROPE, 4, 1>, dim3(n), dim3(256), 0, st, a, items);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

// Whether the two bf16 products take 64 columns a wave (CT = 4), which reads the rows a
// quarter as often, rather than 16, which shares few rows out better.  32 heads of rank
// 512, CT = 1 / 4, us: absorb of 32 rows 4.1 / 3.6, 64 rows 5.0 / 3.9, 384 rows 16 / 9.3; values
// 3.9 / 4.1, 6.0 / 4.5, 16 / 9.2.
bool wide_columns(const LatentArgs& a) { return a.dtype == 1 && a.R >= 48; }

// Row blocks of the two products, of at most about `groups` workgroups.  Each brings
// its weights again: 384 rows of 32 heads, values (CT = 4) in 256 / 512 / 1024 / 1536
// workgroups 9.2 / 9.8 / 12.7 / 16.6 us, absorb in 256 / 512 / 1024 12 / 9.3 / 10.9.
unsigned row_blocks(unsigned row_tiles, unsigned columns, unsigned groups) {
  return std::max(1u, std::min(row_tiles, groups / std::max(1u, columns)));
}

}  // namespace

hipError_t launch_rope_latent(int dtype, int R, int H, int nope, int rope, int rank, float theta, float eps,
                              const float* q, const float* kv, const void* norm_w, const int32_t* pos,
                              const int32_t* slot, int num_pages, void* q_out, void* pages, hipStream_t st) {
  if (R <= 0) return hipSuccess;
  if (static_cast<size_t>(R) > kMaxGrid256) return hipErrorInvalidValue;
  // a row's heads are shared out while that fills the chip
  int shares = std::max(1, std::min(H / 4, 512 / R));
  const dim3 grid(R, shares);
  const uint32_t n_slots = 16u * static_cast<uint32_t>(num_pages);
  if (dtype == 0)
    launch_kernel(rope_latent_kernel<float>, grid, dim3(256), 0, st, H, nope, rope, rank, theta, eps, q, kv,
                  static_cast<const float*>(norm_w), pos, slot, n_slots, static_cast<float*>(q_out), static_cast<float*>(pages));
  else
    launch_kernel(rope_latent_kernel<bf16_t>, grid, dim3(256), 0, st, H, nope, rope, rank, theta, eps, q, kv,
                  static_cast<const bf16_t*>(norm_w), pos, slot, n_slots, static_cast<bf16_t*>(q_out), static_cast<bf16_t*>(pages));
  return hipGetLastError();
}

hipError_t launch_latent_absorb(const LatentArgs& a, hipStream_t st, void* to, const void* tables, size_t n) {
  if (a.R <= 0 || n > kLatentInline || n % 16 || reinterpret_cast<uintptr_t>(to) % 16) return hipErrorInvalidValue;
  const unsigned columns = static_cast<unsigned>(a.H) * (a.rank / 64);
  const bool wide = wide_columns(a);
  const unsigned rows = wide ? 64 : 16;  // of a workgroup at a time
  const dim3 grid(columns, row_blocks((a.R + rows - 1) / rows, columns, wide ? 512 : 1024));
  auto go = [&](auto tab) {
    using Tab = decltype(tab);
    if (a.nope == 64 && a.dtype == 0) launch_kernel(latent_absorb_f32_kernel<64, Tab>, grid, dim3(256), 0, st, a, tab);
    else if (a.nope == 128 && a.dtype == 0) launch_kernel(latent_absorb_f32_kernel<128, Tab>, grid, dim3(256), 0, st, a, tab);
    else if (a.nope == 64 && wide) launch_kernel(latent_absorb_bf16_kernel<64, 4, Tab>, grid, dim3(256), 0, st, a, tab);
    else if (a.nope == 64) launch_kernel(latent_absorb_bf16_kernel<64, 1, Tab>, grid, dim3(256), 0, st, a, tab);
    else if (a.nope == 128 && wide) launch_kernel(latent_absorb_bf16_kernel<128, 4, Tab>, grid, dim3(256), 0, st, a, tab);
    else if (a.nope == 128) launch_kernel(latent_absorb_bf16_kernel<128, 1, Tab>, grid, dim3(256), 0, st, a, tab);
    else return hipErrorInvalidValue;
    return hipGetLastError();
  };
  if (n == 0) return go(NoTables{});
  Tables t;
  t.to = static_cast<uint4*>(to);
  t.n = static_cast<uint32_t>(n / 16);
  std::memcpy(t.unit, tables, n);
  return go(t);
}

hipError_t launch_latent_values(const LatentArgs& a, hipStream_t st) {
  if (a.R <= 0) return hipSuccess;
  const bool wide = wide_columns(a);
  const unsigned columns = static_cast<unsigned>(a.H) * (a.vdim / (wide ? 64 : 16));
  const dim3 grid(columns, row_blocks((static_cast<unsigned>(a.R) + 15) / 16, columns, wide ? 256 : 1024));
  if (a.rank == 256 && a.dtype == 0) launch_kernel(latent_values_f32_kernel<256>, grid, dim3(256), 0, st, a);
  else if (a.rank == 512 && a.dtype == 0) launch_kernel(latent_values_f32_kernel<512>, grid, dim3(256), 0, st, a);
  else if (a.rank == 256 && wide) launch_kernel(latent_values_bf16_kernel<256, 4>, grid, dim3(256), 0, st, a);
  else if (a.rank == 256) launch_kernel(latent_values_bf16_kernel<256, 1>, grid, dim3(256), 0, st, a);
  else if (a.rank == 512 && wide) launch_kernel(latent_values_bf16_kernel<512, 4>, grid, dim3(256), 0, st, a);
  else if (a.rank == 512) launch_kernel(latent_values_bf16_kernel<512, 1>, grid, dim3(256), 0, st, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_latent_attention(const LatentArgs& a, const LatentItem* items, int n_items, int tile, hipStream_t st) {
  if (n_items <= 0) return hipSuccess;
  if (n_items > latent_max_items(a.dtype == 0 ? latent_f32_waves(a.rank) : 0)) return hipErrorInvalidValue;
  if (a.rank == 512 && a.rope == 64) return launch_attention<512, 64>(a, items, n_items, tile, st);
  if (a.rank == 512 && a.rope == 32) return launch_attention<512, 32>(a, items, n_items, tile, st);
  if (a.rank == 256 && a.rope == 64) return launch_attention<256, 64>(a, items, n_items, tile, st);
  if (a.rank == 256 && a.rope == 32) return launch_attention<256, 32>(a, items, n_items, tile, st);
  return hipErrorInvalidValue;
}

hipError_t launch_latent_combine(const LatentArgs& a, const LatentGroup* groups, int n_groups, int tile, int max_parts,
                                 hipStream_t st) {
  if (n_groups <= 0) return hipSuccess;
  if (static_cast<size_t>(n_groups) * tile > kMaxGrid256 || max_parts > kLatentMaxParts) return hipErrorInvalidValue;
  auto go = [&](auto t, auto rank) {
    using T = decltype(t);
    constexpr int RANK = decltype(rank)::value;
    // many parts: more workgroups, each of fewer columns
    constexpr int few = 1024 / RANK, many = 16;
    const unsigned n = static_cast<unsigned>(n_groups) * tile;
    if (max_parts <= 8 * few)
      launch_kernel(latent_combine_kernel<T, RANK, few>, dim3(n), dim3(256), 0, st, a, groups, tile);
    else
      launch_kernel(latent_combine_kernel<T, RANK, many>, dim3(n, RANK * many / 1024), dim3(256), 0, st, a, groups, tile);
    return hipGetLastError();
  };
  if (a.dtype == 0) return a.rank == 512 ? go(float{}, std::integral_constant<int, 512>{}) : go(float{}, std::integral_constant<int, 256>{});
  return a.rank == 512 ? go(bf16_t{}, std::integral_constant<int, 512>{}) : go(bf16_t{}, std::integral_constant<int, 256>{});
}

}  // namespace spec
