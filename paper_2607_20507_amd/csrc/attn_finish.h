// The end of a work item of the split-key attention kernels: the waves' softmax
// states are merged and the output or the partial is written.
#pragma once

#include <hip/hip_runtime.h>

#include "attention.h"
#include "common.h"

namespace spec {

__device__ __forceinline__ void attn_store4(bf16_t* o, const f32x4& v) {
  *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}
__device__ __forceinline__ void attn_store4(float* o, const f32x4& v) {
  *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
}

// keep the first `valid` (0, 1, 2) bf16 halves of a 32-bit word
__device__ __forceinline__ uint32_t mask_pair(uint32_t w, int valid) {
  return valid >= 2 ? w : (valid == 1 ? (w & 0xFFFFu) : 0u);
}

// Lane (g = lane / 16, l16 = lane % 16) holds, for query vector 16 nt + l16, dims
// 16 dt + 4 g .. + 3 of the unnormalised output, the running maximum (base-2
// logits, equal in the 4 lanes of a vector) and its share of the sum.
template <typename T, int HD, int NT, int W>
__device__ __forceinline__ void attn_finish(const AttnArgs& a, const AttnItem& it, int gkv, int M, int lane, int wave,
                                            float (&mrun)[NT], const float (&lrun)[NT],
                                            f32x4 (&acc)[HD / 16][NT]) {
  constexpr int DT = HD / 16;
  const int g = lane >> 4, l16 = lane & 15;
  const int G = a.Hq / a.Hkv;
  float ltot[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float lt = lrun[nt];
    lt += __shfl_xor(lt, 16, kWave);
    lt += __shfl_xor(lt, 32, kWave);
    ltot[nt] = lt;
  }
  if (W > 1) {
    // waves 1..W-1 hand their state to wave 0 (same lane layout in every wave)
    __shared__ float s_acc[W > 1 ? W - 1 : 1][NT][DT][4][kWave];
    __shared__ float s_ml[W > 1 ? W - 1 : 1][NT][2][kWave];
    if (wave > 0) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        s_ml[wave - 1][nt][0][lane] = mrun[nt];
        s_ml[wave - 1][nt][1][lane] = ltot[nt];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 4; ++r) s_acc[wave - 1][nt][dt][r][lane] = acc[dt][nt][r];
      }
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float mm = mrun[nt];
      for (int w = 0; w < W - 1; ++w) mm = fmaxf(mm, s_ml[w][nt][0][lane]);
      if (mm == -INFINITY) continue;  // no key of the item for this query vector
      const float e0 = (mrun[nt] == -INFINITY) ? 0.f : exp2f(mrun[nt] - mm);
      float lt = ltot[nt] * e0;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt][nt] *= e0;
      for (int w = 0; w < W - 1; ++w) {
        const float mw = s_ml[w][nt][0][lane];
        const float ew = (mw == -INFINITY) ? 0.f : exp2f(mw - mm);
        lt += ew * s_ml[w][nt][1][lane];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[dt][nt][r] += ew * s_acc[w][nt][dt][r][lane];
      }
      mrun[nt] = mm;
      ltot[nt] = lt;
    }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float lt = ltot[nt];
    const int m = 16 * nt + l16;
    if (m >= M) continue;
    if (it.part < 0) {
      const float inv = (lt > 0.f) ? 1.f / lt : 0.f;
      T* o = static_cast<T*>(a.out) + (static_cast<size_t>(it.row0 + m / G) * a.Hq + gkv * G + m % G) * HD;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) attn_store4(o + 16 * dt + 4 * g, acc[dt][nt] * inv);
    } else {
      const size_t pm = static_cast<size_t>(it.part * a.Hkv + gkv) * 64 + m;
      float* po = a.part_o + pm * HD;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        *reinterpret_cast<float4*>(po + 16 * dt + 4 * g) =
            make_float4(acc[dt][nt][0], acc[dt][nt][1], acc[dt][nt][2], acc[dt][nt][3]);
      if (g == 0) {
        a.part_ml[pm * 2] = mrun[nt];
        a.part_ml[pm * 2 + 1] = lt;
      }
    }
  }
}

}  // namespace spec
