// The expanded form of the attention over a latent cache, for long runs of rows:
// every head's keys and values are made from the latents once, then attended to.

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "common.h"
#include "kv_layout.h"
#include "latent.h"

namespace spec {
namespace {

// ---------------------------------------------------------------------------
// Expansion: keys and values of the listed pages, k[t, h, n] = sum_c c[t, c] w_k[h, n, c]
// and v likewise, in the operand order of kv_layout.h, a block of 16 tokens per (page,
// head); the shared keys in the same order, a block per page.
// A workgroup makes 128 tokens x 128 features (two units of 64, each of one head's keys
// or values), four waves 64 x 64 each, 32 of the sum at a time through LDS (direct
// loads, NS - 1 stages ahead).  Of every 32 rows of a product, tile 0 takes rows 8 i +
// 0..3 and tile 1 rows 8 i + 4..7, so that a lane's two tiles hold 8 consecutive dims of
// a token (keys: the weight's rows are the product's rows) or 8 consecutive tokens of a
// dim (values: the tokens are), one 16-byte unit, and a wave's stores whole runs of 512
// bytes or more.  Chunk c of row r sits at c ^ key(r): the 8 rows that 8 lanes read,
// in either order, take every bank once.
// 7000 tokens of 32 heads (59 GFLOP, 115 MB written) take 78 us, 41 at the rate of a large
// library product: 12 of the 16 stages 45, the stores 7, launches and each workgroup's first
// loads the rest.  LDS is busy for more than half of the cycles (reads 28%, their conflicts 9%,
// the direct loads' writes about 18%), the matrix pipe for 38%.  256 x 256 tiles of 8 waves 85,
// stages of 64 in two buffers 80, the next stage's operands read under this one's
// products 82, workgroups that begin at different parts of the sum 81.

__global__ __launch_bounds__(256, 3) void latent_expand_kernel(LatentArgs a, const int32_t* __restrict__ list, int n_pages,
                                                               int col_blocks, bf16_t* __restrict__ kx,
                                                               bf16_t* __restrict__ vx, bf16_t* __restrict__ rx) {
  constexpr int KB = 32, NS = 3;  // of the sum a stage, stages
  __shared__ uint4 st[NS][128 * 4], sw[NS][128 * 4];
  const int cb = blockIdx.x % col_blocks, tb = blockIdx.x / col_blocks;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  const int uk = a.nope / 64, units = uk + a.vdim / 64;  // of a head: keys', all
  const int entry = a.rank + a.rope;
  const bf16_t* pool = static_cast<const bf16_t*>(a.pages);
  auto key = [](int r) { return (r >> 1 & 1) | ((r >> 2 ^ r >> 3) & 1) << 1; };

  // a wave's loads of a stage: 16 rows (a page) of tokens, and of the weight, twice
  const char *from_t[2], *from_w[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = 2 * wave + j;
    const size_t page = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(list[min(8 * tb + i, n_pages - 1)]));
    from_t[j] = reinterpret_cast<const char*>(pool + page * 16 * entry);
    const int u = min(2 * cb + (i >> 2), a.H * units - 1), h = u / units, hu = u % units;
    const bf16_t* w = hu < uk ? static_cast<const bf16_t*>(a.w_k) + h * a.k_stride + static_cast<size_t>(64) * hu * a.rank
                              : static_cast<const bf16_t*>(a.w_v) + h * a.v_stride + static_cast<size_t>(64) * (hu - uk) * a.rank;
    from_w[j] = reinterpret_cast<const char*>(w + static_cast<size_t>(16 * (i & 3)) * a.rank);
  }
  const int lr = lane >> 2, lc = (lane & 3) ^ key(lr);
  const uint32_t at_t = (lr * entry + 8 * lc) * 2, at_w = (lr * a.rank + 8 * lc) * 2;
  auto issue = [&](int k, int b) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = 2 * wave + j;
      load_lds16(from_t[j] + 2 * KB * k, at_t, lds_addr(&st[b][64 * i]));
      load_lds16(from_w[j] + 2 * KB * k, at_w, lds_addr(&sw[b][64 * i]));
    }
  };

  // the wave's 64 tokens and its unit
  const int wt = wave >> 1, wu = wave & 1;
  const int u = 2 * cb + wu, h = u / units, hu = u % units;
  const bool values = hu >= uk;
  // rows of the product: the weight's for keys, the tokens for values
  int off[2];  // of a lane's row in tile 0 and 1 of a 32-row pair
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int r = 8 * (l16 >> 2) + (l16 & 3) + 4 * t;
    off[t] = r * 4 + (g ^ key(r));
  }
  const int col_off = l16 * 4 + (g ^ key(l16));
  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int nk = a.rank / KB;
#pragma unroll
  for (int k = 0; k < NS - 1; ++k) issue(k, k);  // (at least 8 stages)
  for (int k = 0; k < nk; ++k) {
    // stage k has landed, every wave is done with stage k - 1, whose buffer takes stage k + NS - 1
    if (k + 1 < nk) {
      SPEC_WAIT_VM_LDS(4 * (NS - 2));
    } else {
      SPEC_WAIT_VM_LDS(0);
    }
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    if (k + NS - 1 < nk) issue(k + NS - 1, (k + NS - 1) % NS);
    const uint4* tok = &st[k % NS][wt * 256];
    const uint4* wgt = &sw[k % NS][wu * 256];
    const uint4* rows = values ? tok : wgt;
    const uint4* cols = values ? wgt : tok;
    uint4 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = rows[(i >> 1) * 128 + off[i & 1]];
      y[i] = cols[i * 64 + col_off];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = mfma16x16x32(x[i], y[j], acc[i][j]);
  }
  if (u < a.H * units) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 lo = acc[2 * i][j], hi = acc[2 * i + 1][j];
        const uint4 v = make_uint4(cvt_pk_bf16(lo[0], lo[1]), cvt_pk_bf16(lo[2], lo[3]), cvt_pk_bf16(hi[0], hi[1]),
                                   cvt_pk_bf16(hi[2], hi[3]));
        const int row = 32 * i + 8 * g;                                                 // .. + 7
        const int col = 16 * j + l16;
        const int t = 64 * wt + (values ? row : col);
        const int page = 8 * tb + (t >> 4);
        if (page >= n_pages) continue;
        if (values) {
          const int d = 64 * (hu - uk) + col;
          *reinterpret_cast<uint4*>(vx + (static_cast<size_t>(page) * a.H + h) * 16 * a.vdim + kv_v_off(t & 15, d)) = v;
        } else {
          const int d = 64 * hu + row;
          *reinterpret_cast<uint4*>(kx + (static_cast<size_t>(page) * a.H + h) * 16 * a.nope + kv_k_off(t & 15, d)) = v;
        }
      }
  }
  if (cb == 0) {
    const int cr = a.rope / 8;
    for (int e = threadIdx.x; e < 128 * cr; e += 256) {
      const int t = e / cr, c = e % cr, page = 8 * tb + (t >> 4);
      if (page >= n_pages) break;
      const bf16_t* src = pool + static_cast<size_t>(static_cast<uint32_t>(list[page])) * 16 * entry + (t & 15) * entry + a.rank;
      *reinterpret_cast<uint4*>(rx + static_cast<size_t>(page) * 16 * a.rope + kv_k_off(t & 15, 8 * c)) =
          *reinterpret_cast<const uint4*>(src + 8 * c);
    }
  }
}

// ---------------------------------------------------------------------------
// Attention to the expanded pages: one workgroup of 8 waves (two per SIMD) per (block
// of 128 NT consecutive rows, head, range of keys: all, or a part where blocks and
// heads leave CUs idle).  The structure is the K / V cache's prompt kernel's
// (attention.hip): 64 keys at a time in LDS, three buffers; each wave both products for
// its own 16 NT rows; a 32-key chunk is a matrix phase and a vector phase, and waves 4..7
// run one phase behind waves 0..3, with which they share the SIMDs.  A key's score has
// the head's own dims and the shared ones, whose block every head reads.
// p = 2^(score scale - max scale), one FMA a score; the rounding of max scale is one factor
// for all of a row, and divides out.  Where a row's logits reach 2^16 that factor could
// matter (and from 2^30 on overflow): there a chunk's scores become their differences to
// the maximum first.  Values that are not finite are
// dropped from chunks in which some row does not see their key, and added after the
// walk for the rows that do.
// 8192 rows of 32 heads (687 GFLOP of attention) take 690 to 750 us, 0.92 to 1.0 PFLOP/s, 1000 rows
// behind 6000 others 147: MFMA (busy 48% of the cycles) and the softmax's vector instructions
// (43%) of a SIMD's two waves add up more than they overlap.  Four waves of 64 rows, a
// wave's own two chunks interleaved instead, 788 us.

constexpr float kPromptRescaleLog2 = 8.f;
constexpr float kPromptLargeLogit = 65536.f;

__device__ __forceinline__ uint32_t keep_pair(uint32_t w, int valid) {
  return valid >= 2 ? w : valid == 1 ? w & 0xFFFFu : 0u;
}

template <int NOPE, int ROPE, int VD, int NT>
__global__ __launch_bounds__(512, 1) void attn_latent_prompt_kernel(LatentArgs a, const LatentItem* __restrict__ items,
                                                                    const bf16_t* __restrict__ kx,
                                                                    const bf16_t* __restrict__ vx,
                                                                    const bf16_t* __restrict__ rx,
                                                                    float* __restrict__ part_o,
                                                                    float* __restrict__ part_ml) {
  constexpr int DN = NOPE / 32, DS = DN + ROPE / 32;  // k-steps of the scores: own dims, all
  constexpr int DT = VD / 16;
  constexpr int NW = 8, NB = 3;
  constexpr int KU = 2 * NOPE, RU = 2 * ROPE, VU = 2 * VD;  // 16-byte units of a page's block
  constexpr int LK = KU / 64, LV = VU / 64, LR = RU / 64;   // loads of one
  // a wave's loads of a stage: of the four pages' keys, values and (LR = 1: waves 0..3) shared keys
  constexpr int WK = 4 * LK / NW, WV = 4 * LV / NW, LPW = WK + WV;
  static_assert(4 * LK % NW == 0 && 4 * LV % NW == 0 && 4 * LR <= NW);
  __shared__ uint4 sk[NB][4 * KU], sv[NB][4 * VU], sr[NB][4 * RU];
  // the rows' rotated dims, each wave's as it multiplies them (in registers they are 16 too many)
  __shared__ uint4 sq[NW][NT][DS - DN][64];
  const int h = blockIdx.x % a.H;
  const LatentItem it = items[blockIdx.x / a.H];  // (qv0: its first row, nqv: rows)
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  const int t0 = it.t0, t1 = it.t1, ns = (t1 - t0 + 63) >> 6;

  // the next stage into buffer b.  Pages past the sequence's last are other pages, or what
  // the workspace has behind them (their keys are masked, and their values not used)
  const int page0 = it.page0 + (t0 >> 4);
  const char* next_k = reinterpret_cast<const char*>(kx) + (static_cast<size_t>(page0) * a.H + h) * (32 * NOPE);
  const char* next_v = reinterpret_cast<const char*>(vx) + (static_cast<size_t>(page0) * a.H + h) * (32 * VD);
  const char* next_r = reinterpret_cast<const char*>(rx) + static_cast<size_t>(page0) * (32 * ROPE);
  const size_t page_k = static_cast<size_t>(a.H) * (32 * NOPE), page_v = static_cast<size_t>(a.H) * (32 * VD);
  size_t of_k[WK], of_v[WV];
#pragma unroll
  for (int n = 0; n < WK; ++n) of_k[n] = (NW * n + wave) / LK * page_k + (NW * n + wave) % LK * 1024;
#pragma unroll
  for (int n = 0; n < WV; ++n) of_v[n] = (NW * n + wave) / LV * page_v + (NW * n + wave) % LV * 1024;
  auto issue = [&](int b) {
#pragma unroll
    for (int n = 0; n < WK; ++n) load_lds16(next_k + of_k[n], lane * 16, lds_addr(&sk[b][(NW * n + wave) * 64]));
#pragma unroll
    for (int n = 0; n < WV; ++n) load_lds16(next_v + of_v[n], lane * 16, lds_addr(&sv[b][(NW * n + wave) * 64]));
    if (4 * LR == NW || wave < 4 * LR) load_lds16(next_r + wave * 1024, lane * 16, lds_addr(&sr[b][wave * 64]));
    next_k += 4 * page_k;
    next_v += 4 * page_v;
    next_r += 4 * 32 * ROPE;
  };

  uint4 qf[NT][DN];
  int klim[NT];  // the last key each row sees (-1: none, padding)
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int m = 16 * (NT * wave + nt) + l16;
    const bool ok = m < it.nqv;
    klim[nt] = ok ? min(it.pos0 + m, t1 - 1) : -1;
    const bf16_t* base = static_cast<const bf16_t*>(a.q) + (static_cast<size_t>(it.qv0 + (ok ? m : 0)) * a.H + h) * (NOPE + ROPE) + 8 * g;
#pragma unroll
    for (int s = 0; s < DS; ++s) {
      const uint4 x = ok ? *reinterpret_cast<const uint4*>(base + 32 * s) : make_uint4(0, 0, 0, 0);
      if (s < DN) qf[nt][s] = x;
      else sq[wave][nt][s - DN][lane] = x;
    }
  }
  const int pos_lo = it.pos0 + 16 * NT * wave;
  const int pos_hi = min(it.pos0 + min(16 * NT * (wave + 1), it.nqv), t1) - 1;
  const float scale = a.scale;
  // minus the running maximum, minus its logit (-inf: no key yet, every p is 0; 0 where logits
  // are large), the score above which it is raised (-inf: no key yet), two partial sums of p
  float mneg[NT], add[NT], mlim[NT], lrun[NT][2];
  bool large = false;  // some logit of the wave is
  f32x4 acc[DT][NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    mlim[nt] = add[nt] = -INFINITY;
    mneg[nt] = 0.f;
    lrun[nt][0] = lrun[nt][1] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // the head's own dims of the next chunk's keys, read a phase ahead
  uint4 kf[2][DN], vf[DT];
  auto read_k = [&](int b, int hf) {
    const uint4* kb = &sk[b][(2 * hf + (l16 >> 3)) * KU];
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
#pragma unroll
      for (int s = 0; s < DN; ++s) kf[hh][s] = kb[((s * 2 + hh) * 4 + g) * 8 + (l16 & 7)];
  };
  auto read_v = [&](int b, int hf, int q) {
    const uint4* vb = &sv[b][(2 * hf + (g >> 1)) * VU];
#pragma unroll
    for (int dt = q * DT / 4; dt < (q + 1) * DT / 4; ++dt) vf[dt] = vb[(dt * 2 + (g & 1)) * 16 + l16];
  };
  f32x4 sc[NT][2];
  uint4 pf[NT];
  // the shared keys and the rows' rotated dims, read under the own dims' products
  uint4 kr[2][DS - DN], qr[NT][DS - DN];
  auto read_r = [&](int b, int hf) {
    const uint4* rb = &sr[b][(2 * hf + (l16 >> 3)) * RU];
#pragma unroll
    for (int s = 0; s < DS - DN; ++s)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) kr[hh][s] = rb[((s * 2 + hh) * 4 + g) * 8 + (l16 & 7)];
#pragma unroll
    for (int s = 0; s < DS - DN; ++s)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) qr[nt][s] = sq[wave][nt][s][lane];
  };
  auto scores = [&] {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) sc[nt][0] = sc[nt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < DS; ++s)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
          sc[nt][hh] = mfma16x16x32(s < DN ? kf[hh][s] : kr[hh][s - DN], s < DN ? qf[nt][s] : qr[nt][s - DN], sc[nt][hh]);
  };
  bool dropped = false;
  auto output = [&](int c0) {
    if (c0 + 32 > t1) {
      asm volatile("");
      const int nvalid = min(max(t1 - (c0 + 8 * g), 0), 8);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        vf[dt].x = keep_pair(vf[dt].x, nvalid);
        vf[dt].y = keep_pair(vf[dt].y, nvalid - 2);
        vf[dt].z = keep_pair(vf[dt].z, nvalid - 4);
        vf[dt].w = keep_pair(vf[dt].w, nvalid - 6);
      }
    }
    if (c0 + 31 > pos_lo) {
      asm volatile("");
      uint32_t bad = 0;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        bad |= nonfinite_bits(vf[dt].x) | nonfinite_bits(vf[dt].y) | nonfinite_bits(vf[dt].z) | nonfinite_bits(vf[dt].w);
      if (__any(bad != 0)) {
        dropped = true;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vf[dt] = drop_nonfinite(vf[dt]);
      }
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) acc[dt][nt] = mfma16x16x32(vf[dt], pf[nt], acc[dt][nt]);
  };
  auto softmax = [&](int c0, int b, int hf) {
    read_v(b, hf, 0);
    read_v(b, hf, 1);
    if (c0 + 31 > pos_lo || c0 + 31 >= t1) {
      asm volatile("");
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c0 + 8 * g + j > klim[nt]) sc[nt][j / 4][j % 4] = -INFINITY;
    }
    float mx[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      mx[nt] = sc[nt][0][0];
#pragma unroll
      for (int j = 1; j < 8; ++j) mx[nt] = fmaxf(mx[nt], sc[nt][j / 4][j % 4]);
    }
    bool up = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) up |= mx[nt] > mlim[nt];
    if (__any(up)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float m = mx[nt];
        m = fmaxf(m, __shfl_xor(m, 16, kWave));
        m = fmaxf(m, __shfl_xor(m, 32, kWave));
        if (m > mlim[nt]) {
          const float logit = m * scale;
          const bool big = !(fabsf(logit) < kPromptLargeLogit);
          const float to = big ? 0.f : -logit;
          const float alpha = mlim[nt] == -INFINITY ? 0.f
                              : __builtin_amdgcn_exp2f(big || add[nt] == 0.f ? (-mneg[nt] - m) * scale : to - add[nt]);
          mneg[nt] = -m;
          add[nt] = to;
          mlim[nt] = m + kPromptRescaleLog2 / scale;
#pragma unroll
          for (int i = 0; i < 2; ++i) lrun[nt][i] *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) acc[dt][nt] *= alpha;
        }
      }
      large = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) large |= __any(!(fabsf(mneg[nt] * scale) < kPromptLargeLogit));
    }
    if (large) {
      asm volatile("");
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        if (!(fabsf(mneg[nt] * scale) < kPromptLargeLogit)) sc[nt][0] += mneg[nt], sc[nt][1] += mneg[nt];
    }
    read_v(b, hf, 2);
    read_v(b, hf, 3);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(fmaf(sc[nt][j / 4][j % 4], scale, add[nt]));
#pragma unroll
      for (int j = 0; j < 8; ++j) lrun[nt][j % 2] += p[j];
      pf[nt] = make_uint4(cvt_pk_bf16(p[0], p[1]), cvt_pk_bf16(p[2], p[3]), cvt_pk_bf16(p[4], p[5]), cvt_pk_bf16(p[6], p[7]));
    }
  };
  auto phase_end = [&] {
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
  };

  issue(0);
  if (ns > 1) {
    issue(1);
    SPEC_WAIT_VM_LDS(LPW);
  } else {
    SPEC_WAIT_VM_LDS(0);
  }
  phase_end();  // stage 0 has landed
  read_k(0, 0);
  if (wave >= 4) phase_end();  // waves 4..7 run one phase behind
  for (int j = 0; j < ns; ++j) {
    const int b = j % NB, bn = (j + 1) % NB;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int c0 = t0 + 64 * j + 32 * hf;
      // matrix phase (chunks above every row of this wave are left out); the sums come
      // first, so that their operands are gone when the scores' need registers
      if (c0 > t0 && c0 - 32 <= pos_hi) output(c0 - 32);
      __builtin_amdgcn_sched_barrier(0);
      if (c0 <= pos_hi) {
        read_r(b, hf);
        scores();
      }
      if (hf == 0) read_k(b, 1);
      else if (j + 1 < ns) read_k(bn, 0);
      // stage j + 1 has landed before any wave reads it, a phase on
      if (hf == 0) __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
      phase_end();
      // vector phase.  Every wave is past its reads of stage j - 1, so its buffer takes stage j + 2
      if (hf == 0 && j + 2 < ns) issue((j + 2) % NB);
      __builtin_amdgcn_s_setprio(1);
      if (c0 <= pos_hi) softmax(c0, b, hf);
      __builtin_amdgcn_s_setprio(0);
      SPEC_WAIT_VM_LDS(63);  // (LDS reads only)
      phase_end();
    }
  }
  if (t0 + 64 * ns - 32 <= pos_hi) output(t0 + 64 * ns - 32);
  if (wave < 4) phase_end();
  if (dropped)
    for (int c0 = max(max(pos_lo - 31, 0) / 32 * 32, t0); c0 <= pos_hi; c0 += 32) {
      if (c0 + 31 <= pos_lo) continue;
      const uint4* vb = reinterpret_cast<const uint4*>(
          vx + ((static_cast<size_t>(it.page0) + min((c0 + 8 * g) >> 4, (t1 - 1) >> 4)) * a.H + h) * (16 * VD));
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const uint4 marks = nonfinite_marks(vb[(dt * 2 + (g & 1)) * 16 + l16]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          acc[dt][nt] += nonfinite_sum(mfma16x16x32(marks, seen_keys(klim[nt] - (c0 + 8 * g)), f32x4{0.f, 0.f, 0.f, 0.f}));
      }
    }

#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float l = lrun[nt][0] + lrun[nt][1];
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    const int m = 16 * (NT * wave + nt) + l16;
    if (m >= it.nqv) continue;
    if (it.part < 0) {
      const float inv = 1.f / l;
      bf16_t* o = static_cast<bf16_t*>(a.out) + (static_cast<size_t>(it.qv0 + m) * a.H + h) * VD + 4 * g;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const f32x4 v = acc[dt][nt] * inv;
        *reinterpret_cast<uint2*>(o + 16 * dt) = make_uint2(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]));
      }
    } else {
      // a part's reference is its maximum itself, without the rounding of its logit
      const bool none = mlim[nt] == -INFINITY;
      const float fix = none || add[nt] == 0.f ? 1.f : __builtin_amdgcn_exp2f(-fmaf(-mneg[nt], scale, add[nt]));
      const size_t pv = (static_cast<size_t>(it.part) * (16 * NT * NW) + m) * a.H + h;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(part_o + pv * VD + 16 * dt + 4 * g) = acc[dt][nt] * fix;
      if (g == 0) *reinterpret_cast<float2*>(part_ml + 2 * pv) = make_float2(none ? -FLT_MAX : -mneg[nt], l * fix);
    }
  }
}

// The parts of a block's rows to its output: a thread has four dims of one row and head.
template <int VD>
__global__ __launch_bounds__(256) void latent_prompt_combine_kernel(LatentArgs a, const LatentGroup* __restrict__ groups, int rows,
                                                                    const float* __restrict__ part_o,
                                                                    const float* __restrict__ part_ml) {
  constexpr int U = VD / 4, HB = 256 / U;  // threads of a head, heads of a workgroup
  const LatentGroup gr = groups[blockIdx.x / rows];
  const int r = blockIdx.x % rows, h = blockIdx.y * HB + threadIdx.x / U, d = 4 * (threadIdx.x % U);
  if (r >= gr.nqv || h >= a.H) return;
  const size_t first = (static_cast<size_t>(gr.part0) * rows + r) * a.H + h, step = static_cast<size_t>(rows) * a.H;
  constexpr int B = 8;
  float top = -FLT_MAX;
  for (int p0 = 0; p0 < gr.nparts; p0 += B) {
    float m[B];
#pragma unroll
    for (int b = 0; b < B; ++b) m[b] = part_ml[2 * (first + min(p0 + b, gr.nparts - 1) * step)];
#pragma unroll
    for (int b = 0; b < B; ++b) top = fmaxf(top, m[b]);
  }
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  for (int p0 = 0; p0 < gr.nparts; p0 += B) {
    f32x4 v[B];
    float2 ml[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const size_t at = first + min(p0 + b, gr.nparts - 1) * step;
      v[b] = *reinterpret_cast<const f32x4*>(part_o + at * VD + d);
      ml[b] = *reinterpret_cast<const float2*>(part_ml + 2 * at);
    }
#pragma unroll
    for (int b = 0; b < B; ++b)
      if (p0 + b < gr.nparts) {
        const float w = __builtin_amdgcn_exp2f((ml[b].x - top) * a.scale);
        l += w * ml[b].y;
        o += w * v[b];
      }
  }
  o *= 1.f / l;
  *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.out) + (static_cast<size_t>(gr.qv0 + r) * a.H + h) * VD + d) =
      make_uint2(cvt_pk_bf16(o[0], o[1]), cvt_pk_bf16(o[2], o[3]));
}

template <int NOPE, int ROPE, int VD>
hipError_t launch_prompt(const LatentArgs& a, const LatentItem* items, unsigned n, int rows, const LatentExpanded& x, hipStream_t st) {
  const bf16_t *k = static_cast<const bf16_t*>(x.k), *v = static_cast<const bf16_t*>(x.v), *key = static_cast<const bf16_t*>(x.key);
  if (rows == 256) launch_kernel(attn_latent_prompt_kernel<NOPE, ROPE, VD, 2>, dim3(n), dim3(512), 0, st, a, items, k, v, key, x.part_o, x.part_ml);
  else launch_kernel(attn_latent_prompt_kernel<NOPE, ROPE, VD, 1>, dim3(n), dim3(512), 0, st, a, items, k, v, key, x.part_o, x.part_ml);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_latent_expand(const LatentArgs& a, const int32_t* list, int n_pages, const LatentExpanded& x, hipStream_t st) {
  const int units = a.H * (a.nope + a.vdim) / 64;
  const size_t cols = (static_cast<size_t>(units) + 1) / 2, rows = (static_cast<size_t>(n_pages) + 7) / 8;
  if (cols * rows > kMaxGrid256) return hipErrorInvalidValue;
  launch_kernel(latent_expand_kernel, dim3(static_cast<unsigned>(cols * rows)), dim3(256), 0, st, a, list, n_pages,
                static_cast<int>(cols), static_cast<bf16_t*>(x.k), static_cast<bf16_t*>(x.v), static_cast<bf16_t*>(x.key));
  return hipGetLastError();
}

hipError_t launch_latent_prompt(const LatentArgs& a, const LatentItem* items, int n_items, int rows, const LatentExpanded& x,
                                hipStream_t st) {
  if (rows != 128 && rows != 256) return hipErrorInvalidValue;
  const size_t n = static_cast<size_t>(n_items) * a.H;
  if (n == 0) return hipSuccess;
  if (n > kMaxGrid256 / 2) return hipErrorInvalidValue;
  const int sizes = (a.nope == 128 ? 4 : 0) + (a.rope == 64 ? 2 : 0) + (a.vdim == 128 ? 1 : 0);
  const unsigned g = static_cast<unsigned>(n);
  switch (sizes) {
    case 0: return launch_prompt<64, 32, 64>(a, items, g, rows, x, st);
    case 1: return launch_prompt<64, 32, 128>(a, items, g, rows, x, st);
    case 2: return launch_prompt<64, 64, 64>(a, items, g, rows, x, st);
    case 3: return launch_prompt<64, 64, 128>(a, items, g, rows, x, st);
    case 4: return launch_prompt<128, 32, 64>(a, items, g, rows, x, st);
    case 5: return launch_prompt<128, 32, 128>(a, items, g, rows, x, st);
    case 6: return launch_prompt<128, 64, 64>(a, items, g, rows, x, st);
    default: return launch_prompt<128, 64, 128>(a, items, g, rows, x, st);
  }
}

hipError_t launch_latent_prompt_combine(const LatentArgs& a, const LatentGroup* groups, int n_groups, int rows,
                                        const LatentExpanded& x, hipStream_t st) {
  if (n_groups <= 0) return hipSuccess;
  const int hb = 1024 / a.vdim;
  const size_t n = static_cast<size_t>(n_groups) * rows;
  const dim3 grid(static_cast<unsigned>(n), (a.H + hb - 1) / hb);
  if (n * grid.y > kMaxGrid256) return hipErrorInvalidValue;
  if (a.vdim == 128) launch_kernel(latent_prompt_combine_kernel<128>, grid, dim3(256), 0, st, a, groups, rows, x.part_o, x.part_ml);
  else launch_kernel(latent_prompt_combine_kernel<64>, grid, dim3(256), 0, st, a, groups, rows, x.part_o, x.part_ml);
  return hipGetLastError();
}

}  // namespace spec
