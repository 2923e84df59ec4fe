// The 4-bit KV cache: rotary embedding + append, read back, expansion to bf16
// pages, and paged causal attention over it (host-side launch interface).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attention.h"

namespace spec {

// launch_rope_kv with the K and V rows quantised into 4-bit pages
// (kv4_layout.h; head dim 64 or 128).  A row whose slot is outside
// 0 .. 16 num_pages - 1 has only its q written.
hipError_t launch_rope_kv4(int dtype, int R, int Hq, int Hkv, int hd, float theta, const float* qkv,
                           const int32_t* pos, const int32_t* slot, int num_pages, void* q, void* kpool, void* vpool,
                           hipStream_t st);

// k, v [R, Hkv, hd] (dtype) <- the rows held in the slots; rows with a slot
// outside the pool are left as they were.
hipError_t launch_kv4_read(int dtype, int R, int Hkv, int hd, const int32_t* slot, int num_pages, const void* kpool,
                           const void* vpool, void* k, void* v, hipStream_t st);

// bf16 pages dst 0 .. n - 1 (kv_layout.h) <- the 4-bit pages src[0 .. n - 1], K and V.
hipError_t launch_kv4_expand(int n, const int32_t* src, int Hkv, int hd, const void* kpool, const void* vpool,
                             void* kdst, void* vdst, hipStream_t st);

// As launch_attention_bf16 (items, groups and partials), kpool / vpool 4-bit
// pages; q and out are fp32 or bf16 (a.dtype).  The page table, items and groups
// are at byte offsets o_pt, o_it and o_gr of `tables`: device memory, or, with
// `inline_bytes` > 0 (at most kUploadInline), host memory that travels in the
// kernel's arguments (no groups then, and items of at most kKv4StagedPages
// pages).
constexpr int kKv4StagedPages = 512;
struct Kv4Tables {
  const char* tables = nullptr;
  size_t inline_bytes = 0, o_pt = 0, o_it = 0, o_gr = 0;
};
hipError_t launch_attention_kv4(const AttnArgs& a, const Kv4Tables& t, int n_items, int n_groups, int max_parts,
                                int nt, int w, hipStream_t st);

}  // namespace spec
