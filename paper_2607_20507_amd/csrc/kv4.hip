// The 4-bit KV cache (kv4_layout.h): append, read back, attention.

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "host_util.h"
#include "kv4.h"
#include "kv4_layout.h"

namespace spec {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// ---------------------------------------------------------------------------
// values <-> codes

__device__ __forceinline__ float scale_of_byte(uint32_t b) { return __uint_as_float(b << 23); }

// Codes of two values (a in the low nibble) with the scale s = 2^E.  The
// instruction rounds to the nearest level, ties to the even code.
template <int SEL>
__device__ __forceinline__ uint32_t put_codes(uint32_t w, float a, float b, float s) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, s, SEL);
}

// The two values of byte SEL of w as bf16 (low nibble in the low half).  Only
// the exponent field of s counts, so callers pass a scale byte shifted there
// with whatever bits surround it.
template <int SEL>
__device__ __forceinline__ uint32_t get_codes(uint32_t w, uint32_t s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, __uint_as_float(s), SEL));
}
// Scale byte B of a word, moved to the exponent field of a float.
template <int B>
__device__ __forceinline__ uint32_t scale_bits(uint32_t w) {
  return B == 0 ? w << 23 : B == 1 ? w << 15 : B == 2 ? w << 7 : w >> 1;
}

// One 4-byte unit: 8 values of one token as bf16.
__device__ __forceinline__ uint4 get8(uint32_t w, uint32_t s) {
  return make_uint4(get_codes<0>(w, s), get_codes<1>(w, s), get_codes<2>(w, s), get_codes<3>(w, s));
}

// 8 tokens of one V byte column (w0: tokens 0..3, w1: 4..7; s0, s1 their scale
// bytes): the low nibbles' dim and the high nibbles' dim, 8 tokens each.
__device__ __forceinline__ void get8_tokens(uint32_t w0, uint32_t w1, uint32_t s0, uint32_t s1, uint4& lo, uint4& hi) {
  const uint32_t t0 = get_codes<0>(w0, scale_bits<0>(s0)), t1 = get_codes<1>(w0, scale_bits<1>(s0));
  const uint32_t t2 = get_codes<2>(w0, scale_bits<2>(s0)), t3 = get_codes<3>(w0, scale_bits<3>(s0));
  const uint32_t t4 = get_codes<0>(w1, scale_bits<0>(s1)), t5 = get_codes<1>(w1, scale_bits<1>(s1));
  const uint32_t t6 = get_codes<2>(w1, scale_bits<2>(s1)), t7 = get_codes<3>(w1, scale_bits<3>(s1));
  auto low = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); };
  auto high = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); };
  lo = make_uint4(low(t0, t1), low(t2, t3), low(t4, t5), low(t6, t7));
  hi = make_uint4(high(t0, t1), high(t2, t3), high(t4, t5), high(t6, t7));
}

// Whether one of 4 scale bytes is at least 252: no other block holds a value that
// is not finite.
__device__ __forceinline__ bool scale_near_top(uint32_t w) {
  const uint32_t x = ~w & 0xFCFCFCFCu;  // a byte of 0 for each such scale
  return ((x - 0x01010101u) & ~x & 0x80808080u) != 0;
}

// 0xFF in the bytes of w that equal b.
__device__ __forceinline__ uint32_t bytes_equal(uint32_t w, uint32_t b) {
  const uint32_t x = w ^ (b * 0x01010101u);
  return ((~(((x & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | x) & 0x80808080u) >> 7) * 255u;
}

// Zeroes the values that are not finite among 4 bytes of codes with their scales:
// all under the scale 255, magnitudes of 2^128 and more under 253 (4 and 6) and
// 254 (2 and more).
__device__ __forceinline__ void drop_nonfinite(uint32_t& codes, uint32_t& scales) {
  const uint32_t nan = bytes_equal(scales, 255u);
  const uint32_t two = codes >> 2 & 0x11111111u, four = two & codes >> 1;
  codes &= ~(nan | bytes_equal(scales, 253u) & (four * 15u) | bytes_equal(scales, 254u) & (two * 15u));
  scales &= ~nan;
}

template <typename T>
__device__ __forceinline__ void put8(T* dst, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                                pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  } else {
    reinterpret_cast<float4*>(dst)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(dst)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}
// 8 bf16 values to T, exact
template <typename T>
__device__ __forceinline__ void put8_bf16(T* dst, const uint4& u) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(dst) = u;
  } else {
    reinterpret_cast<uint4*>(dst)[0] = make_uint4(u.x << 16, u.x & 0xFFFF0000u, u.y << 16, u.y & 0xFFFF0000u);
    reinterpret_cast<uint4*>(dst)[1] = make_uint4(u.z << 16, u.z & 0xFFFF0000u, u.w << 16, u.w & 0xFFFF0000u);
  }
}

// Bits of the larger magnitude of a and b (as integers: an infinity or a NaN
// is above every finite magnitude, and the largest survives).
__device__ __forceinline__ uint32_t mag_max(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// ---------------------------------------------------------------------------
// RoPE + append.  One workgroup per row.  Thread (head, t) rotates pairs
// 8 t .. 8 t + 7 of a q or k head: dims 8 t .. and hd / 2 + 8 t .., which are
// one 4-byte unit each of two blocks of the key, whose other units are held by
// the 3 neighbouring lanes.  Angles, sines and the keys' rotation are in fp64,
// so that a key's code depends on its exact value and not on the order of the
// roundings before it; q is rotated in fp32.
//
// HBM bound: 8192 rows of 32 / 8 heads of 128 (202 MB of fp32 in, 76 MB out) take
// 51 us, 5.4 TB/s.  Workgroups go to the 8 XCDs in turn, and a page's cache lines
// hold parts of all of its tokens, so rows in their order leave every XCD's cache
// with pieces of lines: 114 MB written.  Here kXcdRows consecutive rows share an
// XCD (16, 32 or 64: 74.1 -> 68.6 us with the read-back of 8192 rows after it);
// the rows behind the last whole round keep their order.
constexpr int kXcdRows = 32;
template <typename T>
__global__ __launch_bounds__(256) void rope_kv4_kernel(int Hq, int Hkv, int hd, float theta,
                                                       const float* __restrict__ qkv, const int32_t* __restrict__ pos,
                                                       const int32_t* __restrict__ slot, int num_pages,
                                                       T* __restrict__ q, uint8_t* __restrict__ kpool,
                                                       uint8_t* __restrict__ vpool) {
  int r = blockIdx.x;
  if (r < static_cast<int>(gridDim.x & ~(8u * kXcdRows - 1)))
    r = (r & ~(8 * kXcdRows - 1)) + r % 8 * kXcdRows + r / 8 % kXcdRows;
  const int half = hd / 2, groups = half / 8;
  const float* x = qkv + static_cast<size_t>(r) * (Hq + 2 * Hkv) * hd;
  __shared__ double s_cos[64], s_sin[64];
  if (static_cast<int>(threadIdx.x) < half) {
    double sn, cs;
    sincos(static_cast<double>(pos[r]) * exp(-(2.0 * threadIdx.x / hd) * log(static_cast<double>(theta))), &sn, &cs);
    s_cos[threadIdx.x] = cs;
    s_sin[threadIdx.x] = sn;
  }
  __syncthreads();
  const int sl = slot[r];
  const bool keep = sl >= 0 && sl < 16 * num_pages;
  const int page = keep ? sl >> 4 : 0, off = sl & 15;
  const int bb = kv4_block_bytes(hd);
  // (head, t) pairs in steps of the workgroup: the 4 lanes of a block run the
  // same iterations (groups % 4 == 0)
  for (int e = threadIdx.x; e < (Hq + Hkv) * groups; e += blockDim.x) {
    const int h = e / groups, t = e % groups, i0 = 8 * t;
    const float4* pa = reinterpret_cast<const float4*>(x + h * hd + i0);
    const float4* pb = reinterpret_cast<const float4*>(x + h * hd + i0 + half);
    const float4 a0 = pa[0], a1 = pa[1], b0 = pb[0], b1 = pb[1];
    const float av[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
    const float bv[8] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
    float ra[8], rb[8];
    if (h < Hq) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float c = static_cast<float>(s_cos[i0 + j]), sn = static_cast<float>(s_sin[i0 + j]);
        ra[j] = av[j] * c - bv[j] * sn;
        rb[j] = bv[j] * c + av[j] * sn;
      }
      T* o = q + (static_cast<size_t>(r) * Hq + h) * hd;
      put8(o + i0, ra);
      put8(o + i0 + half, rb);
      continue;
    }
    uint32_t ma = 0, mb = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const double c = s_cos[i0 + j], sn = s_sin[i0 + j];
      const double a = av[j], b = bv[j];
      ra[j] = static_cast<float>(a * c - b * sn);
      rb[j] = static_cast<float>(b * c + a * sn);
      ma = mag_max(ma, mag(ra[j]));
      mb = mag_max(mb, mag(rb[j]));
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      ma = mag_max(ma, __shfl_xor(ma, o, kWave));
      mb = mag_max(mb, __shfl_xor(mb, o, kWave));
    }
    if (!keep) continue;
    uint8_t* blk = kpool + (static_cast<size_t>(page) * Hkv + (h - Hq)) * bb;
    auto put = [&](const float (&v)[8], uint32_t m, int d0) {
      const int s = d0 / 32, g = d0 / 8 % 4;
      const uint32_t sb = kv4_scale_of(m);
      const float sc = scale_of_byte(sb);
      uint32_t w = put_codes<0>(0u, v[0], v[1], sc);
      w = put_codes<1>(w, v[2], v[3], sc);
      w = put_codes<2>(w, v[4], v[5], sc);
      w = put_codes<3>(w, v[6], v[7], sc);
      *reinterpret_cast<uint32_t*>(blk + kv4_k_unit(off, s, g, hd)) = w;
      if (g == 0) blk[kv4_k_scale(off, s, hd)] = static_cast<uint8_t>(sb);
    };
    put(ra, ma, i0);
    put(rb, mb, i0 + half);
  }
  if (!keep) return;
  // values: thread (head, block, i) holds dims 32 b + i and 32 b + 16 + i
  for (int e = threadIdx.x; e < Hkv * half; e += blockDim.x) {
    const int h = e / half, b = e % half / 16, i = e % 16;
    const float* v = x + (Hq + Hkv + h) * hd + 32 * b + i;
    const float lo = v[0], hi = v[16];
    uint32_t m = mag_max(mag(lo), mag(hi));
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) m = mag_max(m, __shfl_xor(m, o, kWave));
    const uint32_t sb = kv4_scale_of(m);
    uint8_t* blk = vpool + (static_cast<size_t>(page) * Hkv + h) * bb;
    blk[kv4_v_byte(off, b, i)] = static_cast<uint8_t>(put_codes<0>(0u, lo, hi, scale_of_byte(sb)));
    if (i == 0) blk[kv4_v_scale(off, b, hd)] = static_cast<uint8_t>(sb);
  }
}

// ---------------------------------------------------------------------------
// Read back: one workgroup per (16 rows, kv head), so that a page that was
// appended in order is read once and rows are written in 16-byte units.  Bound by
// what it writes: 4096 rows of 8 heads of 128 (4.5 MB in, 16.8 out) take 7.7 us a
// call, a launch of 3 among them; 8192 rows 12 us, 3.5 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void kv4_read_kernel(int R, int Hkv, int hd, const int32_t* __restrict__ slot,
                                                       int num_pages, const uint8_t* __restrict__ kpool,
                                                       const uint8_t* __restrict__ vpool, T* __restrict__ k,
                                                       T* __restrict__ v) {
  const int r0 = blockIdx.x / Hkv * 16, h = blockIdx.x % Hkv;
  const int bb = kv4_block_bytes(hd);
  const int units = hd / 8;
  for (int e = threadIdx.x; e < 16 * units; e += blockDim.x) {
    const int r = r0 + e / units, u = e % units;
    if (r >= R) break;
    const int sl = slot[r];
    if (sl < 0 || sl >= 16 * num_pages) continue;
    const uint8_t* blk = kpool + (static_cast<size_t>(sl >> 4) * Hkv + h) * bb;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(blk + kv4_k_unit(sl & 15, u / 4, u % 4, hd));
    const uint32_t s = blk[kv4_k_scale(sl & 15, u / 4, hd)];
    put8_bf16(k + (static_cast<size_t>(r) * Hkv + h) * hd + 8 * u, get8(w, s << 23));
  }
  // values: thread (row, block, half) takes 8 byte columns, dims 32 b + 8 o .. and 32 b + 16 + 8 o ..
  for (int e = threadIdx.x; e < 16 * (hd / 16); e += blockDim.x) {
    const int r = r0 + e / (hd / 16), b = e % (hd / 16) / 2, o = e % 2;
    if (r >= R) break;
    const int sl = slot[r];
    if (sl < 0 || sl >= 16 * num_pages) continue;
    const uint8_t* blk = vpool + (static_cast<size_t>(sl >> 4) * Hkv + h) * bb;
    const uint32_t s = static_cast<uint32_t>(blk[kv4_v_scale(sl & 15, b, hd)]) << 23;
    uint32_t t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = get_codes<0>(blk[kv4_v_byte(sl & 15, b, 8 * o + i)], s);
    auto low = [&](int i) { return __builtin_amdgcn_perm(t[i + 1], t[i], 0x05040100u); };
    auto high = [&](int i) { return __builtin_amdgcn_perm(t[i + 1], t[i], 0x07060302u); };
    T* dst = v + (static_cast<size_t>(r) * Hkv + h) * hd + 32 * b + 8 * o;
    put8_bf16(dst, make_uint4(low(0), low(2), low(4), low(6)));
    put8_bf16(dst + 16, make_uint4(high(0), high(2), high(4), high(6)));
  }
}

// ---------------------------------------------------------------------------
// Expansion to bf16 pages, which the prompt form's attention reads: one workgroup
// per (page, kv head).  A prompt's attention reads every key once for each 256 / G
// of its rows, so they are converted once and written out (HBM bound: 8192 keys
// of 8 heads of 128, 8.9 MB in and 33.5 out, 8.5 us, 4.9 TB/s): 2% of the time of 8192
// rows, and much of it for few rows behind many keys (the planner's comment).
template <int HD>
__global__ __launch_bounds__(256) void kv4_expand_kernel(const int32_t* __restrict__ src, int Hkv,
                                                         const uint8_t* __restrict__ kpool,
                                                         const uint8_t* __restrict__ vpool, bf16_t* __restrict__ kdst,
                                                         bf16_t* __restrict__ vdst) {
  constexpr int DS = HD / 32, BB = kv4_block_bytes(HD);
  const int p = blockIdx.x / Hkv, h = blockIdx.x % Hkv;
  const size_t from = (static_cast<size_t>(src[p]) * Hkv + h) * BB;
  const size_t to = (static_cast<size_t>(p) * Hkv + h) * 16 * HD;
  // K: destination unit ((s 2 + hh) 4 + g) 8 + j is source unit s of lane unit (hh, g, j)
  for (int u = threadIdx.x; u < 2 * HD; u += blockDim.x) {
    const int j = u % 8, g = u / 8 % 4, hh = u / 32 % 2, s = u / 64;
    const uint8_t* blk = kpool + from;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(
        blk + (HD == 128 ? ((hh * 4 + g) * 8 + j) * 16 : ((g * 8 + j) * 2 + hh) * 8) + 4 * s);
    const uint32_t sb = blk[kv4_code_bytes(HD) + (j * 2 + hh) * DS + s];
    reinterpret_cast<uint4*>(kdst + to)[u] = get8(w, sb << 23);
  }
  // V: 8 tokens of a byte column are two destination units
  for (int e = threadIdx.x; e < HD; e += blockDim.x) {
    const int i = e % 16, th = e / 16 % 2, b = e / 32;
    const uint8_t* blk = vpool + from;
    const uint2 w = *reinterpret_cast<const uint2*>(blk + kv4_v_byte(8 * th, b, i));
    const uint2 s = *reinterpret_cast<const uint2*>(blk + kv4_v_scale(8 * th, b, HD));
    uint4 lo, hi;
    get8_tokens(w.x, w.y, s.x, s.y, lo, hi);
    uint4* o = reinterpret_cast<uint4*>(vdst + to);
    o[(2 * b * 2 + th) * 16 + i] = lo;
    o[((2 * b + 1) * 2 + th) * 16 + i] = hi;
  }
}

// ---------------------------------------------------------------------------
// Attention over the 4-bit cache: items, lanes and softmax as the bf16 verify
// attention (attention.hip): S^T = K Q^T and O^T = V^T P^T on the matrix cores,
// 32 keys at a time, a query vector's statistics in the lanes of its column.
// The operands come from the 4-bit pages: a lane's K operand is 4 bytes of one
// key and one scale, its V^T operand 8 bytes (8 tokens, two dims) with 8
// scales, converted in registers to bf16, which holds every value exactly.
// T = float: q and the probabilities are split into three bf16 parts (24 bits
// of fraction), whose products with the cache's values are exact in fp32.
//
// Bound by HBM where a tile has up to 16 query vectors: 131000 keys of 8 heads of
// 128 (142 MB) take 26 us, 5.4 TB/s.  With 32 by instruction issue and the
// longest items' chains: at 64 sequences of 4 .. 8 rows and 512 .. 4096 keys (127
// MB, 30 us) a CU holds waves in 56 of 86 thousand cycles, and of those vector
// instructions take 67%, matrix ones 26%; a 32-key chunk has about 235 of the
// former, 64 of them conversions, 32 that bring tokens beside each other, 32 that
// shift scales and 32 exponents and their arguments.  Small calls are latency: one
// sequence of 2000 keys 12.9 us.

template <typename T>
struct Parts;
template <>
struct Parts<bf16_t> { static constexpr int n = 1; };
template <>
struct Parts<float> { static constexpr int n = 3; };

// Two fp32 -> N pairs of bf16 whose sums are the values (N = 1: rounded once, which
// for probabilities is what the matrix instructions take: three parts would triple
// the products of instruction-bound tiles for an error against 64 bits of 0.0017
// instead of 0.0022 to 0.0024, the output's own rounding in both).
template <int N>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    w[i] = cvt_pk_bf16(a, b);
    if (i + 1 < N) {
      a -= __uint_as_float(w[i] << 16);
      b -= __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}

// Exponents are one FMA, p = 2^(raw scale - M), with M the rounded base-2 logit of
// the maximum, and a wave's sums are relative to 2^M: a new maximum rescales them
// by 2^(M - M'), not by the raw difference.  The largest exponent is off from 0 by
// up to M 2^-24.  A 4-bit cache, whose blocks have any scale, may have larger M than
// this: a wave that meets one starts over in a form that takes the difference of
// the raw scores first (one instruction more per score) and whose sums are relative
// to the raw maximum.  (Both forms in one loop: 16 rows of 64 sequences of 1000 keys
// 54 us, 50 so.)  Waves and parts are joined by the differences of their raw
// maxima, which fp32 holds where it does not hold those of the logits M.
constexpr float kFarLog2 = 16777216.f;
// A maximum is raised only by a score more than 2^8 times as probable: fewer
// rescalings, and probabilities stay below 2^8.
constexpr float kRescaleLog2 = 8.f;

// The call's tables: in device memory, or in the kernel's arguments, which saves
// the launch that would bring them there.
struct TabMem {
  const AttnItem* items;
  const int32_t* pt;
};
struct TabArgs {
  uint32_t n, o_it, o_pt;  // 4-byte words: all, the first item, the page table
  int32_t w[kUploadInline / 4];
};
__device__ __forceinline__ int32_t global_page(const TabMem& t, size_t i) { return t.pt[i]; }
__device__ __forceinline__ int32_t global_page(const TabArgs&, size_t) { return 0; }  // (always in LDS)
static_assert(sizeof(AttnItem) == 32, "eight words an item");

__device__ __forceinline__ void store4(bf16_t* o, const f32x4& v) {
  *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}
__device__ __forceinline__ void store4(float* o, const f32x4& v) {
  *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
}

template <int HD>
__device__ __forceinline__ float score_scale() { return kLog2e / sqrtf(static_cast<float>(HD)); }

// Exponent of the factor that brings sums relative to 2^M (M = m scale, rounded) to
// 2^(m scale).
__device__ __forceinline__ float to_raw(float m, float scale, float M) { return -fmaf(m, scale, -M); }

// The waves' states are merged through LDS, each wave taking some of the output
// tiles, and the output or the partial is written.  m: raw score of a query vector's
// maximum in the wave (-inf: no key), to which (far) or to whose rounded logit the
// wave's sums are relative; l: the wave's sum (in every element).
template <typename T, int HD, int NT, int W>
__device__ __forceinline__ void finish(const AttnArgs& a, const AttnItem& it, int gkv, int M, int lane, int wave, bool far,
                                       const float (&m)[NT], const f32x4 (&l)[NT], const f32x4 (&acc)[HD / 16][NT]) {
  constexpr int DT = HD / 16;
  const int g = lane >> 4, l16 = lane & 15;
  const int G = a.Hq / a.Hkv;
  const float scale = score_scale<HD>();
  // one query tile after the other: the buffer of all would leave room for fewer
  // workgroups on a CU
  __shared__ f32x4 s_acc[W][DT][kWave];
  __shared__ f32x4 s_st[W][16];  // logit of the maximum, sum, maximum, whether far
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if (16 * nt >= M) break;
    if (nt > 0) __syncthreads();
    if (g == 0) s_st[wave][l16] = f32x4{m[nt] * scale, l[nt][0], m[nt], far ? 1.f : 0.f};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) s_acc[wave][dt][lane] = acc[dt][nt];
    __syncthreads();
    const int v = 16 * nt + l16;
    f32x4 st[W];
    float mm = -INFINITY, any = 0.f, e[W], lt = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      st[w] = s_st[w][l16];
      mm = fmaxf(mm, st[w][0]);
      any += st[w][3];
    }
    float part = 1.f, top = -INFINITY;  // what a partial's sums are multiplied by, and its raw maximum
    if (it.part >= 0 || any > 0.f) {
#pragma unroll
      for (int w = 0; w < W; ++w) top = fmaxf(top, st[w][2]);
    }
    if (any > 0.f) {
#pragma unroll
      for (int w = 0; w < W; ++w)
        e[w] = st[w][2] == -INFINITY
                   ? 0.f
                   : exp2f(fmaf(st[w][2] - top, scale, st[w][3] > 0.f ? 0.f : to_raw(st[w][2], scale, st[w][0])));
    } else {
#pragma unroll
      for (int w = 0; w < W; ++w) e[w] = st[w][0] == -INFINITY ? 0.f : exp2f(st[w][0] - mm);
      if (it.part >= 0 && top > -INFINITY) part = exp2f(to_raw(top, scale, mm));
    }
#pragma unroll
    for (int w = 0; w < W; ++w) lt += e[w] * st[w][1];
    if (v < M)
    for (int dt = wave; dt < DT; dt += W) {
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W; ++w) o += e[w] * s_acc[w][dt][lane];
      if (it.part < 0) {
        store4(static_cast<T*>(a.out) + (static_cast<size_t>(it.row0 + v / G) * a.Hq + gkv * G + v % G) * HD + 16 * dt + 4 * g,
               o * (1.f / lt));
      } else {
        const size_t pm = (static_cast<size_t>(it.part) * a.Hkv + gkv) * 64 + v;
        store4(a.part_o + pm * HD + 16 * dt + 4 * g, o * part);
        if (dt == 0 && g == 0) reinterpret_cast<float2*>(a.part_ml)[pm] = make_float2(top, lt * part);
      }
    }
  }
}

template <typename T, int HD, int NT, int W, typename Tab>
__global__ __launch_bounds__(64 * W, NT * Parts<T>::n <= 3 ? 2 : 1) void attn_kv4_kernel(AttnArgs a, const Tab tab) {
  constexpr int DS = HD / 32, DT = HD / 16, BB = kv4_block_bytes(HD), CB = kv4_code_bytes(HD);
  constexpr int NP = Parts<T>::n;
  const int gkv = blockIdx.x % a.Hkv;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int g = lane >> 4, l16 = lane & 15;
  constexpr bool kInArgs = std::is_same_v<Tab, TabArgs>;
  // page ids of the item, in LDS unless it has more than fit
  __shared__ int32_t s_tab[kInArgs ? kUploadInline / 4 : kKv4StagedPages];
  AttnItem it;
  const int32_t* s_pt = s_tab;
  size_t pt = 0;  // the sequence's page ids in tab.pt
  int p0 = 0;     // first page of s_pt
  bool staged = true;
  if constexpr (kInArgs) {
    // arguments lie in host memory: one round trip for all of the tables instead
    // of one for the item and one for its pages
    for (uint32_t i = threadIdx.x; i < tab.n; i += kWave * W) s_tab[i] = tab.w[i];
    __syncthreads();
    const int32_t* p = s_tab + tab.o_it + blockIdx.x / a.Hkv * 8;
    auto word = [&](int i) { return __builtin_amdgcn_readfirstlane(p[i]); };
    it = AttnItem{word(0), word(1), word(2), word(3), word(4), word(5), word(6), word(7)};
    s_pt = s_tab + tab.o_pt + it.seq * a.max_pages;
  } else {
    it = tab.items[blockIdx.x / a.Hkv];
    pt = static_cast<size_t>(it.seq) * a.max_pages;
    p0 = it.t0 >> 4;
    const int np = it.t1 > it.t0 ? ((it.t1 - 1) >> 4) - p0 + 1 : 0;
    staged = np <= kKv4StagedPages;
    if (staged)
      for (int i = threadIdx.x; i < np; i += kWave * W) s_tab[i] = tab.pt[pt + p0 + i];
    __syncthreads();
  }
  const int G = a.Hq / a.Hkv;
  const int M = it.nrows * G;
  const uint8_t* kp = static_cast<const uint8_t*>(a.kpool);
  const uint8_t* vp = static_cast<const uint8_t*>(a.vpool);

  uint4 qf[NT][DS][NP];
  int vpos[NT];
  bool vval[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int m = 16 * nt + l16;
    vval[nt] = m < M;
    const int mm = vval[nt] ? m : 0;
    vpos[nt] = it.pos0 + mm / G;
    const T* base = static_cast<const T*>(a.q) + (static_cast<size_t>(it.row0 + mm / G) * a.Hq + gkv * G + mm % G) * HD + g * 8;
#pragma unroll
    for (int s = 0; s < DS; ++s) {
      if constexpr (NP == 1) {
        qf[nt][s][0] = vval[nt] ? reinterpret_cast<const uint4*>(base)[4 * s] : make_uint4(0, 0, 0, 0);
      } else {
        uint32_t w[4][NP];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 v = reinterpret_cast<const float2*>(base + 32 * s)[j];
          split_pair<NP>(vval[nt] ? v.x : 0.f, vval[nt] ? v.y : 0.f, w[j]);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) qf[nt][s][i] = make_uint4(w[0][i], w[1][i], w[2][i], w[3][i]);
      }
    }
  }
  const float scale = score_scale<HD>();
  const int pos_lo = it.pos0;  // every row of the item sees the keys up to here
  int klim[NT];                // the last key a query vector sees (-1: none, a padding vector)
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) klim[nt] = vval[nt] ? min(vpos[nt], it.t1 - 1) : -1;
  // the running maximum of the raw scores, the score above which it is raised,
  // minus its base-2 logit
  // (sums of the probabilities as the products see them, rounded, by a product
  // with ones: 16 additions a chunk less, and the rounding cancels in the quotient)
  float mrun[NT], mlim[NT], mneg[NT];
  f32x4 lrun[NT];
  const uint4 ones = make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);
  bool dropped;
  f32x4 acc[DT][NT];
  const int cfirst = it.t0 + 32 * wave;  // the wave's first chunk; it takes every W-th
  auto any_page = [&](int t) -> size_t {
    if (kInArgs || staged) return s_pt[(t >> 4) - p0];
    return global_page(tab, pt + (t >> 4));
  };

  // codes and scales of one 32-key chunk's operands (keys past t1 clamped to
  // a valid page; their scores are masked and their V entries zeroed)
  struct Raw {
    uint32_t kc[2 * DS], ks[DS / 2];  // [key tile][step] (hd 64 too: a lane's 16 bytes hold both tiles)
    uint32_t vc[2 * DS], vs[2 * DS];  // [block][token half]
  };
  auto load_v = [&](Raw& w, int c0, auto page) {
    const uint8_t* blk = vp + (page(min(c0 + 8 * g, it.t1 - 1)) * a.Hkv + gkv) * BB;
    const int th = g & 1;
#pragma unroll
    for (int i = 0; i < HD / 64; ++i) {
      const uint4 u = ld_stream(reinterpret_cast<const uint4*>(blk) + (i * 2 + th) * 16 + l16);
      w.vc[4 * i] = u.x; w.vc[4 * i + 1] = u.y; w.vc[4 * i + 2] = u.z; w.vc[4 * i + 3] = u.w;
      const uint4 s = *(reinterpret_cast<const uint4*>(blk + CB) + th * (DS / 2) + i);
      w.vs[4 * i] = s.x; w.vs[4 * i + 1] = s.y; w.vs[4 * i + 2] = s.z; w.vs[4 * i + 3] = s.w;
    }
    asm volatile("" ::: "memory");
  };

  // The wave's sums over its chunks, in the form for large logits (FAR) or not; whether
  // the form does not hold a logit.
  auto walk = [&](auto page, auto far_form) -> bool {
    constexpr bool FAR = decltype(far_form)::value;
    bool far = false;
    dropped = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      mrun[nt] = mlim[nt] = -INFINITY;
      mneg[nt] = 0.f;
      lrun[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    auto load_k = [&](Raw& w, int c0) {
      const uint8_t* blk = kp + (page(min(c0 + 16 * (l16 >> 3), it.t1 - 1)) * a.Hkv + gkv) * BB;
      const int j = l16 & 7;
#pragma unroll
      for (int i = 0; i < HD / 64; ++i) {
        const uint4 u = ld_stream(reinterpret_cast<const uint4*>(blk) + (HD == 128 ? (i * 4 + g) * 8 + j : g * 8 + j));
        w.kc[4 * i] = u.x; w.kc[4 * i + 1] = u.y; w.kc[4 * i + 2] = u.z; w.kc[4 * i + 3] = u.w;
      }
      const uint32_t* sp = reinterpret_cast<const uint32_t*>(blk + CB) + j * (DS / 2);
#pragma unroll
      for (int i = 0; i < DS / 2; ++i) w.ks[i] = sp[i];
      // (loads stay where they are issued: the compiler had moved the scales' to
      // their use, a memory latency in every chunk)
      asm volatile("" ::: "memory");
    };
    // the chunk of keys c0 .. held in w, which then takes the wave's chunk of keys cn ..
    auto chunk = [&](Raw& w, int c0, int cn) {
      const bool full = c0 + 32 <= it.t1 && c0 + 31 <= pos_lo;  // no masks
      f32x4 sc[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) sc[nt][0] = sc[nt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      auto step = [&](auto s_) {
        constexpr int s = decltype(s_)::value;
        if constexpr (s < DS) {
          const uint4 k0 = get8(w.kc[s], scale_bits<s % 4>(w.ks[s / 4]));
          const uint4 k1 = get8(w.kc[DS + s], scale_bits<(DS + s) % 4>(w.ks[(DS + s) / 4]));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < NP; ++i) {
              sc[nt][0] = mfma16x16x32(k0, qf[nt][s][i], sc[nt][0]);
              sc[nt][1] = mfma16x16x32(k1, qf[nt][s][i], sc[nt][1]);
            }
        }
      };
      step(std::integral_constant<int, 0>{});
      step(std::integral_constant<int, 1>{});
      step(std::integral_constant<int, 2>{});
      step(std::integral_constant<int, 3>{});
      load_k(w, cn);
      float raw[NT][8], mx[NT];
      bool grow = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int j = 0; j < 8; ++j) raw[nt][j] = (j < 4) ? sc[nt][0][j] : sc[nt][1][j - 4];
      }
      if (!full) {
        asm volatile("");  // keeps the masks a branch
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 8; ++j) raw[nt][j] = c0 + 8 * g + j <= klim[nt] ? raw[nt][j] : -INFINITY;
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mx[nt] = raw[nt][0];
#pragma unroll
        for (int j = 1; j < 8; ++j) mx[nt] = fmaxf(mx[nt], raw[nt][j]);
        grow |= mx[nt] > mlim[nt];
      }
      if (__any(grow)) {  // a new maximum: the same in every lane of a query vector
        bool large = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float m = mx[nt];
          m = fmaxf(m, __shfl_xor(m, 16, kWave));
          m = fmaxf(m, __shfl_xor(m, 32, kWave));
          m = m > mlim[nt] ? m : mrun[nt];
          const float neg = m == -INFINITY ? 0.f : -m * scale;
          const float alpha =
              mrun[nt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(FAR ? (mrun[nt] - m) * scale : neg - mneg[nt]);
          mrun[nt] = m;
          mlim[nt] = m + kRescaleLog2 / scale;
          mneg[nt] = neg;
          large |= fabsf(neg) > kFarLog2;
          lrun[nt] *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) acc[dt][nt] *= alpha;
        }
        if constexpr (!FAR) far |= __any(large) != 0;
      }
      uint4 pf[NT][NP];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          p[j] = __builtin_amdgcn_exp2f(FAR ? (raw[nt][j] - (mrun[nt] == -INFINITY ? 0.f : mrun[nt])) * scale
                                            : fmaf(raw[nt][j], scale, mneg[nt]));
        uint32_t h[4][NP];
#pragma unroll
        for (int j = 0; j < 4; ++j) split_pair<NP>(p[2 * j], p[2 * j + 1], h[j]);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          pf[nt][i] = make_uint4(h[0][i], h[1][i], h[2][i], h[3][i]);
          lrun[nt] = mfma16x16x32(ones, pf[nt][i], lrun[nt]);
        }
      }
      if (c0 + 32 > it.t1) {  // keys past the end hold anything, and 0 x NaN is not 0
        asm volatile("");
        const int nvalid = min(max(it.t1 - (c0 + 8 * g), 0), 8);
        const uint64_t keep = nvalid == 8 ? ~0ull : (1ull << (8 * nvalid)) - 1;
#pragma unroll
        for (int i = 0; i < 2 * DS; ++i) {
          w.vc[i] &= static_cast<uint32_t>(i % 2 ? keep >> 32 : keep);
          w.vs[i] &= static_cast<uint32_t>(i % 2 ? keep >> 32 : keep);
        }
      }
      if (!full || NP > 1) {
        // a value that is not finite may lie in a key that some row does not see, and
        // the parts of a probability may be 0 or negative
        bool top = false;
#pragma unroll
        for (int i = 0; i < 2 * DS; ++i) top |= scale_near_top(w.vs[i]);
        if (__any(top)) {
          dropped = true;
#pragma unroll
          for (int i = 0; i < 2 * DS; ++i) drop_nonfinite(w.vc[i], w.vs[i]);
        }
      }
#pragma unroll
      for (int b = 0; b < DS; ++b) {
        uint4 v[2];
        get8_tokens(w.vc[2 * b], w.vc[2 * b + 1], w.vs[2 * b], w.vs[2 * b + 1], v[0], v[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int n = 0; n < NP; ++n) acc[2 * b + i][nt] = mfma16x16x32(v[i], pf[nt][n], acc[2 * b + i][nt]);
      }
      load_v(w, cn, page);
    };
    // The wave's chunks: the next one's operands are loaded as soon as this one's
    // are converted.  (Two chunks in flight took more registers and no less time:
    // 64 sequences 42.7 .. 47.1 us against 43.7 .. 47.1, 131000 keys 37.3 and 36.4.)
    Raw raw;
    if (cfirst < it.t1) {
      load_k(raw, cfirst);
      load_v(raw, cfirst, page);
    }
    for (int c0 = cfirst; c0 < it.t1 && !far; c0 += 32 * W) chunk(raw, c0, min(c0 + 32 * W, it.t1 - 1));
    return far;
  };
  bool far;
  if constexpr (kInArgs) {
    far = walk([&](int t) -> size_t { return s_pt[(t >> 4) - p0]; }, std::false_type{});
  } else {
    if (staged) far = walk([&](int t) -> size_t { return s_pt[(t >> 4) - p0]; }, std::false_type{});
    else far = walk([&](int t) -> size_t { return global_page(tab, pt + (t >> 4)); }, std::false_type{});
  }
  if (far) walk(any_page, std::true_type{});
  // what the dropped values do to the rows that see them (rare, so after the walk,
  // where it takes no registers from it)
  if (dropped)
    for (int c0 = cfirst; c0 < it.t1; c0 += 32 * W) {
      if (NP == 1 && c0 + 32 <= it.t1 && c0 + 31 <= pos_lo) continue;  // nothing was dropped there
      Raw raw;
      load_v(raw, c0, any_page);
#pragma unroll
      for (int b = 0; b < DS; ++b) {
        uint4 v[2];
        get8_tokens(raw.vc[2 * b], raw.vc[2 * b + 1], raw.vs[2 * b], raw.vs[2 * b + 1], v[0], v[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint4 marks = nonfinite_marks(v[i]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            acc[2 * b + i][nt] += nonfinite_sum(mfma16x16x32(marks, seen_keys(klim[nt] - (c0 + 8 * g)), f32x4{0.f, 0.f, 0.f, 0.f}));
        }
      }
    }
  finish<T, HD, NT, W>(a, it, gkv, M, lane, wave, far, mrun, lrun, acc);
}

// Merges the parts of split items: with M the largest maximum of raw scores, out =
// sum 2^((m - M) scale) o over sum 2^((m - M) scale) l.  A query vector's parts are shared by P threads for each 4
// dims, 8 / P vectors a workgroup of 256 (head dim 64: twice as many): a thread's
// loads of up to 8 parts are in flight together.  A launch and two round trips to
// memory: 4 us with 2 parts a vector (64 sequences) and with 64 (131000 keys).
template <typename T, int HD, int P>
__global__ __launch_bounds__(256) void combine_kv4_kernel(AttnArgs a, const AttnGroup* __restrict__ groups) {
  constexpr int TQ = HD / 4, QV = 256 / TQ / P, B = 8;
  const AttnGroup gr = groups[blockIdx.x];
  const int gkv = blockIdx.y, G = a.Hq / a.Hkv;
  const int d0 = 4 * (static_cast<int>(threadIdx.x) % TQ), sl = static_cast<int>(threadIdx.x) / TQ;
  const int pg = sl % P, v = blockIdx.z * QV + sl / P;
  const bool in = v < gr.nrows * G;
  const size_t base = (static_cast<size_t>(gr.part0) * a.Hkv + gkv) * 64 + (in ? v : 0);
  const size_t stride = static_cast<size_t>(a.Hkv) * 64;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
  const float scale = score_scale<HD>();
  float M = -INFINITY, den = 0.f;
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = pg; p0 < gr.nparts; p0 += B * P) {
    float2 c[B];
    f32x4 o[B];
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const size_t pm = base + min(p0 + i * P, gr.nparts - 1) * stride;
      c[i] = ml[pm];
      o[i] = *reinterpret_cast<const f32x4*>(a.part_o + pm * HD + d0);
      if (p0 + i * P >= gr.nparts) {
        c[i] = make_float2(-INFINITY, 0.f);
        o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
    float mx = M;
#pragma unroll
    for (int i = 0; i < B; ++i) mx = fmaxf(mx, c[i].x);
    if (mx == -INFINITY) {  // sums of 0, or NaN where every score of a part was one (it raises no maximum)
#pragma unroll
      for (int i = 0; i < B; ++i) den += c[i].y;
      continue;
    }
    const float e0 = M == -INFINITY ? 0.f : exp2f((M - mx) * scale);
    num *= e0;
    den *= e0;
    M = mx;
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const float e = c[i].x == -INFINITY ? 0.f : exp2f((c[i].x - mx) * scale);
      num += e * o[i];
      den += e * c[i].y;
    }
  }
  if constexpr (P > 1) {
    __shared__ f32x4 s_num[256];
    __shared__ float s_m[256], s_den[256];
    s_num[threadIdx.x] = num;
    s_m[threadIdx.x] = M;
    s_den[threadIdx.x] = den;
    __syncthreads();
    if (pg > 0) return;
#pragma unroll
    for (int i = 1; i < P; ++i) M = fmaxf(M, s_m[threadIdx.x + i * TQ]);
    num = f32x4{0.f, 0.f, 0.f, 0.f};
    den = 0.f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int t = threadIdx.x + i * TQ;
      const float e = s_m[t] == -INFINITY ? 0.f : exp2f((s_m[t] - M) * scale);
      num += e * s_num[t];
      den += e * s_den[t];
    }
  }
  if (in)
    store4(static_cast<T*>(a.out) + (static_cast<size_t>(gr.row0 + v / G) * a.Hq + gkv * G + v % G) * HD + d0, num * (1.f / den));
}

template <typename T, int HD>
void launch_combine(const AttnArgs& a, const AttnGroup* groups, int n_groups, int max_parts, int nt, hipStream_t st) {
  const int per = 1024 / HD;  // vectors of a workgroup with P = 1
  auto go = [&](auto p_) {
    constexpr int P = decltype(p_)::value;
    launch_kernel(combine_kv4_kernel<T, HD, P>, dim3(n_groups, a.Hkv, (16 * nt * P + per - 1) / per), dim3(256), 0, st, a,
                  groups);
  };
  // 64 parts (131000 keys): P = 1 9.6 us, 8 3.9; 2 parts of 64 sequences 4.1 and 5.1; 8
  // sequences of 4000 keys, 8 parts each, 25.0 and 27.8 us a call
  if (max_parts <= 8) go(std::integral_constant<int, 1>{});
  else go(std::integral_constant<int, 8>{});
}

template <typename T, int HD, typename Tab>
hipError_t launch_items(const AttnArgs& a, const Tab& tab, int n_items, int nt, int w, hipStream_t st) {
  const dim3 grid(n_items * a.Hkv);
  auto go = [&](auto nt_, auto w_) {
    constexpr int NT = decltype(nt_)::value, W = decltype(w_)::value;
    launch_kernel(attn_kv4_kernel<T, HD, NT, W, Tab>, grid, dim3(64 * W), 0, st, a, tab);
    return hipGetLastError();
  };
  using std::integral_constant;
  if (nt == 1 && w == 4) return go(integral_constant<int, 1>{}, integral_constant<int, 4>{});
  if (nt == 2 && w == 4) return go(integral_constant<int, 2>{}, integral_constant<int, 4>{});
  if constexpr (Parts<T>::n == 1) {
    if (nt == 4 && w == 4) return go(integral_constant<int, 4>{}, integral_constant<int, 4>{});
    if (nt == 1 && w == 8) return go(integral_constant<int, 1>{}, integral_constant<int, 8>{});
    if (nt == 2 && w == 8) return go(integral_constant<int, 2>{}, integral_constant<int, 8>{});
  }
  return hipErrorInvalidValue;
}

template <typename T, int HD>
hipError_t launch_attn(const AttnArgs& a, const Kv4Tables& t, int n_items, int n_groups, int max_parts, int nt, int w,
                       hipStream_t st) {
  if (t.inline_bytes) {
    TabArgs tab;
    if (t.inline_bytes > kUploadInline || n_groups > 0) return hipErrorInvalidValue;
    tab.n = static_cast<uint32_t>(t.inline_bytes / 4);
    tab.o_it = static_cast<uint32_t>(t.o_it / 4);
    tab.o_pt = static_cast<uint32_t>(t.o_pt / 4);
    std::memcpy(tab.w, t.tables, t.inline_bytes);
    return launch_items<T, HD>(a, tab, n_items, nt, w, st);
  }
  const TabMem tab{reinterpret_cast<const AttnItem*>(t.tables + t.o_it), reinterpret_cast<const int32_t*>(t.tables + t.o_pt)};
  const hipError_t e = launch_items<T, HD>(a, tab, n_items, nt, w, st);
  if (e != hipSuccess || n_groups <= 0) return e;
  launch_combine<T, HD>(a, reinterpret_cast<const AttnGroup*>(t.tables + t.o_gr), n_groups, max_parts, nt, st);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_kv4(int dtype, int R, int Hq, int Hkv, int hd, float theta, const float* qkv,
                           const int32_t* pos, const int32_t* slot, int num_pages, void* q, void* kpool, void* vpool,
                           hipStream_t st) {
  if (hd != 64 && hd != 128) return hipErrorInvalidValue;
  if (R <= 0) return hipSuccess;
  if (static_cast<size_t>(R) > kMaxGrid256) return hipErrorInvalidValue;
  auto go = [&](auto* qp) {
    using T = std::remove_pointer_t<decltype(qp)>;
    launch_kernel(rope_kv4_kernel<T>, dim3(R), dim3(256), 0, st, Hq, Hkv, hd, theta, qkv, pos, slot, num_pages, qp,
                  static_cast<uint8_t*>(kpool), static_cast<uint8_t*>(vpool));
  };
  if (dtype == 0) go(static_cast<float*>(q));
  else go(static_cast<bf16_t*>(q));
  return hipGetLastError();
}

hipError_t launch_kv4_read(int dtype, int R, int Hkv, int hd, const int32_t* slot, int num_pages, const void* kpool,
                           const void* vpool, void* k, void* v, hipStream_t st) {
  if (hd != 64 && hd != 128) return hipErrorInvalidValue;
  if (R <= 0) return hipSuccess;
  const size_t blocks = (static_cast<size_t>(R) + 15) / 16 * Hkv;
  if (blocks > kMaxGrid256) return hipErrorInvalidValue;
  const dim3 grid(static_cast<uint32_t>(blocks));
  auto go = [&](auto* kd, auto* vd) {
    using T = std::remove_pointer_t<decltype(kd)>;
    launch_kernel(kv4_read_kernel<T>, grid, dim3(256), 0, st, R, Hkv, hd, slot, num_pages,
                  static_cast<const uint8_t*>(kpool), static_cast<const uint8_t*>(vpool), kd, vd);
  };
  if (dtype == 0) go(static_cast<float*>(k), static_cast<float*>(v));
  else go(static_cast<bf16_t*>(k), static_cast<bf16_t*>(v));
  return hipGetLastError();
}

hipError_t launch_kv4_expand(int n, const int32_t* src, int Hkv, int hd, const void* kpool, const void* vpool,
                             void* kdst, void* vdst, hipStream_t st) {
  if (hd != 64 && hd != 128) return hipErrorInvalidValue;
  if (n <= 0) return hipSuccess;
  if (static_cast<size_t>(n) * Hkv > kMaxGrid256) return hipErrorInvalidValue;
  const auto kernel = hd == 128 ? kv4_expand_kernel<128> : kv4_expand_kernel<64>;
  launch_kernel(kernel, dim3(n * Hkv), dim3(256), 0, st, src, Hkv, static_cast<const uint8_t*>(kpool),
                static_cast<const uint8_t*>(vpool), static_cast<bf16_t*>(kdst), static_cast<bf16_t*>(vdst));
  return hipGetLastError();
}

hipError_t launch_attention_kv4(const AttnArgs& a, const Kv4Tables& t, int n_items, int n_groups, int max_parts,
                                int nt, int w, hipStream_t st) {
  if (n_items <= 0) return hipSuccess;
  if (static_cast<size_t>(n_items) * a.Hkv * w > 4 * kMaxGrid256 || (a.hd != 64 && a.hd != 128)) return hipErrorInvalidValue;
  if (a.dtype == 0)
    return a.hd == 128 ? launch_attn<float, 128>(a, t, n_items, n_groups, max_parts, nt, w, st)
                       : launch_attn<float, 64>(a, t, n_items, n_groups, max_parts, nt, w, st);
  return a.hd == 128 ? launch_attn<bf16_t, 128>(a, t, n_items, n_groups, max_parts, nt, w, st)
                     : launch_attn<bf16_t, 64>(a, t, n_items, n_groups, max_parts, nt, w, st);
}

}  // namespace spec
