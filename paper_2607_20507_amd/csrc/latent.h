// Attention of models that keep one latent vector and one rotated key a token:
// its paged cache's append and the attention over it (host-side launch interface).
//
// A token's cache entry is [latent c (rank) | shared key (rope)], row-major in
// pages of 16 tokens.  Head h has the key [w_k[h] c | shared key] and the value
// w_v[h] c.  The absorbed form never makes them: it takes a query's unrotated
// part to the latents' space first (q' = w_k[h]^T q), attends to the latents
// themselves, and takes the sum back (out = w_v[h] o').  Every head then reads the
// same keys and values, so that a tile's query vectors are any rows and heads of
// one sequence: query vector row * H + head.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <vector>

namespace spec {

// Query vectors [qv0, qv0 + nqv) of one sequence, whose first row (of the rows that
// take the form) is row0 at position pos0 and whose page ids start at entry page0
// of the page list, against its keys [t0, t1), t0 a multiple of 32.  Its rows are qoff
// rows further on among all rows of the call.
// part >= 0: an unnormalised partial; part < 0: the normalised output.
struct LatentItem {
  int32_t qv0, nqv, row0, pos0, page0, t0, t1, part, qoff;
};

// The parts of one tile's query vectors.
struct LatentGroup {
  int32_t qv0, nqv, part0, nparts;
};

// A sequence's rows [row0, row0 + nrows), of those that take the form, at positions
// pos0.. .
struct LatentSegment {
  int32_t row0, nrows, pos0, page0, qoff;
};

struct LatentPlan {
  int tile = 16;  // query vectors an item holds at most: 16, 32 or 64 (fp32: 16)
  std::vector<LatentItem> items;
  std::vector<LatentGroup> groups;
  int n_parts = 0;
};

// Tiles and key splits of the absorbed form (at most kLatentMaxParts parts in all).
constexpr int kLatentMaxParts = 512;
// fp32_waves: 0 for bf16, else the waves that share an fp32 item's pages.
LatentPlan plan_latent(const std::vector<LatentSegment>& segs, int H, int fp32_waves);
constexpr int latent_f32_waves(int rank) { return rank == 256 ? 8 : 4; }

// Tiles of those segments (there are at most that many items, or a few hundred), and the
// most items that a launch takes: one workgroup each of 256 threads, or of an fp32 item's
// waves, and a launch counts its threads in 32 bits.
int64_t latent_tiles(const std::vector<LatentSegment>& segs, int H, int fp32_waves);
constexpr int64_t latent_max_items(int fp32_waves) { return ((int64_t{1} << 32) - 1) / (fp32_waves > 4 ? 64 * fp32_waves : 256); }

// Items of the expanded form (below): blocks of `rows` (256 or 128) rows, those with
// most keys first.
struct LatentPromptPlan {
  int rows = 256;
  std::vector<LatentItem> items;
  std::vector<LatentGroup> groups;  // (qv0, nqv: a row and rows)
  int n_parts = 0;
};
LatentPromptPlan plan_latent_prompt(const std::vector<LatentSegment>& segs, int H);

// Whether a sequence of nrows rows behind pos0 others takes the expanded form; weights:
// elements of w_k and w_v.
bool latent_expands(int nrows, int pos0, int64_t weights);

struct LatentArgs {
  int dtype;  // 0 fp32, 1 bf16 (q, pages, weights, out, q_lat, o_lat)
  int H, nope, rope, rank, vdim;
  int R = 0;                          // rows that take the absorbed form
  const int32_t* row_list = nullptr;  // which of all rows they are (null: the first R)
  float scale;             // of the scores, times log2 e
  const void* q;           // [rows, H, nope + rope]
  const void* pages;       // [P][16][rank + rope]
  const void* w_k;         // [H][nope][rank], k_stride elements between heads
  const void* w_v;         // [H][vdim][rank], v_stride elements between heads
  int64_t k_stride, v_stride;
  const int32_t* page_list;
  void* out;               // [rows, H, vdim]
  void* q_lat;             // [R, H, rank]: the absorbed rows' queries in the latents' space
  void* o_lat;             // [R, H, rank]: their weighted sums of latents
  float* part_o;           // [parts][tile][rank]
  float* part_ml;          // [parts][tile][2]: raw maximum and sum
};

// q_out [R, H, nope + rope] <- q with its rotary part rotated; the slots' entries
// <- the normed latents and rotated keys.  Rows whose slot is outside 0 ..
// 16 num_pages - 1 have only their q written.
hipError_t launch_rope_latent(int dtype, int R, int H, int nope, int rope, int rank, float theta, float eps,
                              const float* q, const float* kv, const void* norm_w, const int32_t* pos,
                              const int32_t* slot, int num_pages, void* q_out, void* pages, hipStream_t st);

// The queries' product.  With n > 0 (at most kLatentInline bytes, a multiple of 16) its
// first workgroup also copies the call's tables to `to` (16-byte aligned), in the
// kernel's arguments: one launch less before the attention that reads them.
constexpr size_t kLatentInline = 3584;
hipError_t launch_latent_absorb(const LatentArgs& a, hipStream_t st, void* to = nullptr, const void* tables = nullptr, size_t n = 0);
hipError_t launch_latent_attention(const LatentArgs& a, const LatentItem* items, int n_items, int tile, hipStream_t st);
// (max_parts: the most parts of a group)
hipError_t launch_latent_combine(const LatentArgs& a, const LatentGroup* groups, int n_groups, int tile, int max_parts,
                                 hipStream_t st);
hipError_t launch_latent_values(const LatentArgs& a, hipStream_t st);

// The expanded form (bf16): every head's keys [n_pages][H][16 x nope] and values
// [n_pages][H][16 x vdim] of the listed pages, and the shared keys [n_pages][16 x
// rope], in kv_layout.h's order; then items of at most `rows` rows (qv0, nqv: a row and
// rows; page0: the sequence's first expanded page; t0 a multiple of 64), each of which is
// one workgroup a head; then the parts' join.
struct LatentExpanded {
  void *k = nullptr, *v = nullptr, *key = nullptr;
  float* part_o = nullptr;   // [parts][rows][H][vdim]
  float* part_ml = nullptr;  // [parts][rows][H][2]
};
hipError_t launch_latent_expand(const LatentArgs& a, const int32_t* list, int n_pages, const LatentExpanded& x, hipStream_t st);
hipError_t launch_latent_prompt(const LatentArgs& a, const LatentItem* items, int n_items, int rows, const LatentExpanded& x,
                                hipStream_t st);

hipError_t launch_latent_prompt_combine(const LatentArgs& a, const LatentGroup* groups, int n_groups, int rows,
                                        const LatentExpanded& x, hipStream_t st);

}  // namespace spec
