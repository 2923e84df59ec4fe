// Context-free entry points: the decision pass on caller logits, the draft
// sampler, the generator, and single-kernel entry points (include/spec_ops.h).

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <exception>
#include <mutex>
#include <string>
#include <vector>

#include "../../include/spec.h"
#include "../../include/spec_ops.h"
#include "attention.h"
#include "elem.h"
#include "gemm.h"
#include "host_util.h"
#include "kv4.h"
#include "kv4_layout.h"
#include "latent.h"
#include "logprob.h"
#include "vocab.h"

using namespace spec;

namespace {

constexpr int kOpMaxParts = 4096;
constexpr int kMaxSlotPages = INT32_MAX / kPage;  // a slot (page * 16 + offset) is an int32
constexpr int32_t kMaxExtent = 1 << 30;           // of a row or sequence: with a tile added it is still an int32
constexpr int32_t kMaxHeads = 65535;              // a grid dimension; an int32 also times the head dim

std::mutex g_mu;
Stager& stager() {
  static Stager s;
  return s;
}

spec_status hip_status(hipError_t e) {
  if (e == hipSuccess) return SPEC_OK;
  if (e == hipErrorInvalidValue) return SPEC_E_UNSUPPORTED;
  return SPEC_E_HIP;
}

// Refusal of a context-free call, explained by spec_last_error(NULL).
spec_status refuse(spec_status s, const char* msg) {
  set_global_error(msg);
  return s;
}

// Status of a call's last launch, with a message if it failed.
spec_status launched(hipError_t e, const char* call) {
  const spec_status s = hip_status(e);
  if (s == SPEC_E_UNSUPPORTED) set_global_error((std::string(call) + ": more workgroups than a launch holds").c_str());
  else if (s != SPEC_OK) set_global_error((std::string(call) + ": " + hipGetErrorString(e)).c_str());
  return s;
}

bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

// Tables of a call to its workspace.  A stream that is being captured takes
// only tables that travel in a kernel's arguments, so that a replay finds them.
spec_status upload_tables(void* ws, const MetaBlock& mb, const char* what, hipStream_t st) {
  const size_t n = mb.size();
  if (n > kUploadInline) {
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(st, &cap) != hipSuccess) return refuse(SPEC_E_HIP, what);
    if (cap != hipStreamCaptureStatusNone) return refuse(SPEC_E_UNSUPPORTED, what);
  }
  std::lock_guard<std::mutex> lk(g_mu);
  return stager().upload(ws, mb.data(), n, st) == hipSuccess ? SPEC_OK : refuse(SPEC_E_HIP, "uploading a call's tables failed");
}

}  // namespace

namespace spec {
EventTimer& global_timer() {
  static EventTimer t;
  return t;
}
}  // namespace spec

extern "C" {

size_t spec_sample_workspace_bytes(int32_t B, int32_t total_rows, int32_t V) {
  if (B <= 0 || total_rows <= 0 || V <= 0) return 0;
  return align_up(sizeof(VRow) * total_rows) + align_up(sizeof(VSeq) * B) +
         vocab_ws_bytes(vocab_plan(B, total_rows, V));
}

spec_status spec_sample_verify(int32_t B, const int32_t* k, const float* temperature,
                               const int64_t* seq_ids, const int32_t* base_pos,
                               const float* p_logits, const float* q_logits,
                               const int32_t* draft_tokens, int32_t V, uint64_t seed,
                               int32_t* n_accepted, int32_t* out_tokens, void* workspace,
                               size_t workspace_bytes, void* stream) {
  if (B < 0 || V <= 0) return SPEC_E_INVALID;
  if (B == 0) return SPEC_OK;
  if (!k || !temperature || !seq_ids || !base_pos || !p_logits || !n_accepted || !out_tokens || !workspace)
    return SPEC_E_INVALID;
  int kmax = 0, np = 0, nq = 0;
  for (int b = 0; b < B; ++b) {
    if (k[b] < 0 || k[b] > 15 || !(temperature[b] >= 0.f)) return SPEC_E_INVALID;
    kmax = std::max(kmax, k[b]);
    np += k[b] + 1;
    nq += k[b];
  }
  if (nq > 0 && (!q_logits || !draft_tokens)) return SPEC_E_INVALID;
  const int rows_n = np + nq;
  if (workspace_bytes < spec_sample_workspace_bytes(B, rows_n, V)) return SPEC_E_INVALID;
  std::vector<VRow> rows(rows_n);
  std::vector<VSeq> seqs(B);
  int pr = 0, qr = 0;
  for (int b = 0; b < B; ++b) {
    const float t = temperature[b];
    const float it = t > 0.f ? 1.f / t : 0.f;
    VSeq s{};
    s.k = k[b];
    s.p_row = pr;
    s.q_row = np + qr;
    s.tok_row = qr;
    s.base_pos = base_pos[b];
    s.t = t;
    s.seq_lo = static_cast<uint32_t>(static_cast<uint64_t>(seq_ids[b]));
    s.seq_hi = static_cast<uint32_t>(static_cast<uint64_t>(seq_ids[b]) >> 32);
    seqs[b] = s;
    for (int j = 0; j <= k[b]; ++j)
      rows[pr + j] = VRow{p_logits + static_cast<size_t>(pr + j) * V, it, t > 0.f ? 0 : 1};
    for (int j = 0; j < k[b]; ++j)
      rows[np + qr + j] = VRow{q_logits + static_cast<size_t>(qr + j) * V, it, t > 0.f ? 0 : 1};
    pr += k[b] + 1;
    qr += k[b];
  }
  char* ws = static_cast<char*>(workspace);
  const size_t orow = 0, oseq = align_up(sizeof(VRow) * rows_n);
  const size_t ovoc = oseq + align_up(sizeof(VSeq) * B);
  MetaBlock mb;
  mb.add(rows);
  mb.add(seqs);
  hipStream_t st = static_cast<hipStream_t>(stream);
  std::lock_guard<std::mutex> lk(g_mu);
  // the metadata block lays rows then seqs out exactly at orow / oseq
  hipError_t e = stager().upload(ws, mb.data(), oseq + sizeof(VSeq) * B, st);
  if (e != hipSuccess) return SPEC_E_HIP;
  // the vector path reads 16-byte units from each row
  const bool aligned = (reinterpret_cast<uintptr_t>(p_logits) & 15) == 0 &&
                       (nq == 0 || (reinterpret_cast<uintptr_t>(q_logits) & 15) == 0);
  e = launch_vocab_pass(vocab_plan(B, rows_n, V, B * (2 * kmax + 1)), reinterpret_cast<const VRow*>(ws + orow),
                        reinterpret_cast<const VSeq*>(ws + oseq), draft_tokens, seed, kmax, n_accepted,
                        out_tokens, ws + ovoc, st, &global_timer(), nullptr, aligned);
  return hip_status(e);
}

spec_status spec_sample_draft(int32_t n, const float* logits, int32_t V, const float* temperature,
                              const int64_t* seq_ids, const int32_t* pos, uint64_t seed,
                              int32_t* tokens, void* workspace, size_t workspace_bytes, void* stream) {
  if (n < 0 || V <= 0) return SPEC_E_INVALID;
  if (n == 0) return SPEC_OK;
  if (!logits || !temperature || !seq_ids || !pos || !tokens || !workspace) return SPEC_E_INVALID;
  const DraftPlan p = draft_plan(n, V);
  const size_t odr = 0, ows = align_up(sizeof(DRow) * n);
  if (workspace_bytes < ows + draft_ws_bytes(p)) return SPEC_E_INVALID;
  std::vector<DRow> rows(n);
  for (int i = 0; i < n; ++i) {
    if (!(temperature[i] >= 0.f)) return SPEC_E_INVALID;
    DRow d{};
    d.ptr = logits + static_cast<size_t>(i) * V;
    d.t = temperature[i];
    d.pos = pos[i];
    d.seq_lo = static_cast<uint32_t>(static_cast<uint64_t>(seq_ids[i]));
    d.seq_hi = static_cast<uint32_t>(static_cast<uint64_t>(seq_ids[i]) >> 32);
    d.out = i;
    d.guide = -1;
    rows[i] = d;
  }
  char* ws = static_cast<char*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (n <= kDraftInline) return hip_status(launch_draft_sample_inline(p, rows.data(), seed, tokens, ws + ows, st));
  std::lock_guard<std::mutex> lk(g_mu);
  hipError_t e = stager().upload(ws + odr, rows.data(), sizeof(DRow) * n, st);
  if (e != hipSuccess) return SPEC_E_HIP;
  return hip_status(launch_draft_sample(p, reinterpret_cast<const DRow*>(ws + odr), seed, tokens, ws + ows, st));
}

spec_status spec_philox_uniform(uint64_t seed, int64_t seq_id, int32_t pos, int32_t purpose, int32_t n,
                                float* out, void* stream) {
  if (n < 0 || (n > 0 && !out)) return SPEC_E_INVALID;
  return hip_status(launch_philox_uniform(seed, static_cast<uint64_t>(seq_id), pos, purpose, n, out,
                                          static_cast<hipStream_t>(stream)));
}

size_t spec_op_gemm_workspace_bytes(int32_t R, int32_t Nw) {
  return (R <= 0 || Nw <= 0) ? 0 : gemm_splitk_bytes(R, Nw);
}

spec_status spec_pack_weight(void* w, int32_t rows, int32_t K, int32_t rot_rows, int32_t head_dim,
                             void* stream) {
  if (!w || rows < 0 || K <= 0 || rot_rows < 0 || rot_rows > rows) return SPEC_E_INVALID;
  if (K % 128 != 0) return SPEC_E_UNSUPPORTED;
  if (rot_rows > 0 && (head_dim <= 0 || head_dim % 16 != 0 || head_dim > 256 || rot_rows % head_dim != 0))
    return SPEC_E_UNSUPPORTED;
  return hip_status(launch_pack_weight(w, rows, K, rot_rows, head_dim, static_cast<hipStream_t>(stream)));
}

spec_status spec_pack_model(spec_model_desc* m, void* stream) {
  if (!m || !m->layers || !m->lm_head) return SPEC_E_INVALID;
  if (m->weight_layout != SPEC_LAYOUT_ROWMAJOR) return SPEC_E_STATE;
  if (m->dtype == SPEC_F32) return SPEC_OK;
  if (m->dtype != SPEC_BF16 || m->n_layers <= 0 || m->d_model <= 0 || m->ffn_dim <= 0 || m->n_heads <= 0 ||
      m->n_kv_heads <= 0 || m->head_dim <= 0 || m->vocab <= 0)
    return SPEC_E_INVALID;
  const int d = m->d_model, f = m->ffn_dim, hd = m->head_dim, qd = m->n_heads * hd;
  if (d % 128 || f % 128 || qd % 128 || hd % 16) return SPEC_E_UNSUPPORTED;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int qkv_rows = (m->n_heads + 2 * m->n_kv_heads) * hd, rot = (m->n_heads + m->n_kv_heads) * hd;
  const size_t esz = 2;
  std::vector<const void*> done;  // matrices shared between layers are converted once
  auto once = [&](const void* p) {
    if (std::find(done.begin(), done.end(), p) != done.end()) return false;
    done.push_back(p);
    return true;
  };
  auto pack = [&](const void* p, int rows, int K, int rr) -> hipError_t {
    if (!p || !once(p)) return hipSuccess;
    return launch_pack_weight(const_cast<void*>(p), rows, K, rr, hd, st);
  };
  for (int l = 0; l < m->n_layers; ++l) {
    const spec_layer_weights& L = m->layers[l];
    hipError_t e = pack(L.wqkv, qkv_rows, d, rot);
    if (e == hipSuccess) e = pack(L.wo, d, qd, 0);
    if (e == hipSuccess && L.w_gate_up && once(L.w_gate_up)) {
      e = launch_pack_weight(const_cast<void*>(L.w_gate_up), f, d, 0, hd, st);
      if (e == hipSuccess)
        e = launch_pack_weight(static_cast<char*>(const_cast<void*>(L.w_gate_up)) + static_cast<size_t>(f) * d * esz,
                               f, d, 0, hd, st);
    }
    if (e == hipSuccess) e = pack(L.w_down, d, f, 0);
    if (e != hipSuccess) return hip_status(e);
  }
  const hipError_t e = pack(m->lm_head, m->vocab, d, 0);
  if (e != hipSuccess) return hip_status(e);
  m->weight_layout = SPEC_LAYOUT_TILED;
  return SPEC_OK;
}

spec_status spec_op_gemm(int32_t dtype, int32_t R, int32_t N, int32_t K, const void* X, const void* W,
                         void* Y, int32_t epilogue, void* workspace, size_t workspace_bytes, void* stream) {
  if ((dtype != SPEC_F32 && dtype != SPEC_BF16) || R < 0 || N < 0 || K <= 0 || !X || !W || !Y)
    return SPEC_E_INVALID;
  if (epilogue < SPEC_EPI_STORE_F32 || epilogue > SPEC_EPI_SWIGLU) return SPEC_E_INVALID;
  if (dtype == SPEC_BF16 && K % 128 != 0) return SPEC_E_UNSUPPORTED;
  return hip_status(launch_gemm(dtype == SPEC_F32 ? 0 : 1, R, N, K, X, W, Y, epilogue,
                                static_cast<hipStream_t>(stream), nullptr, static_cast<float*>(workspace),
                                workspace ? workspace_bytes : 0));
}

spec_status spec_op_rmsnorm(int32_t dtype, int32_t R, int32_t d, const float* h, const void* w, float eps,
                            void* y, void* stream) {
  if ((dtype != SPEC_F32 && dtype != SPEC_BF16) || R < 0 || d <= 0 || !h || !w || !y) return SPEC_E_INVALID;
  return hip_status(launch_rmsnorm(dtype == SPEC_F32 ? 0 : 1, R, d, h, nullptr, w, eps, y,
                                   static_cast<hipStream_t>(stream)));
}

spec_status spec_op_rope_kv(int32_t dtype, int32_t R, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                            float theta, const float* qkv, const int32_t* pos, const int32_t* slot,
                            void* q_out, void* k_pages, void* v_pages, void* stream) {
  if ((dtype != SPEC_F32 && dtype != SPEC_BF16) || R < 0 || n_heads <= 0 || n_kv_heads <= 0 ||
      head_dim <= 0 || head_dim % 2 || head_dim > 256)
    return SPEC_E_INVALID;
  if (R == 0) return SPEC_OK;
  if (!qkv || !pos || !slot || !q_out || !k_pages || !v_pages) return SPEC_E_INVALID;
  return hip_status(launch_rope_kv(dtype == SPEC_F32 ? 0 : 1, R, n_heads, n_kv_heads, head_dim, theta, qkv,
                                   pos, slot, q_out, k_pages, v_pages, static_cast<hipStream_t>(stream)));
}

size_t spec_op_attention_workspace_bytes(int32_t n_seqs, int32_t total_rows, int32_t max_pages,
                                         int32_t n_kv_heads, int32_t head_dim) {
  if (n_seqs <= 0 || total_rows <= 0) return 0;
  const size_t meta = align_up(sizeof(int32_t) * (static_cast<size_t>(n_seqs) * max_pages + 2 * total_rows)) +
                      align_up(sizeof(AttnItem) * (static_cast<size_t>(total_rows) + kOpMaxParts)) +
                      align_up(sizeof(AttnGroup) * total_rows);
  return meta + align_up(sizeof(float) * static_cast<size_t>(kOpMaxParts) * n_kv_heads * 64 * head_dim) +
         align_up(sizeof(float) * static_cast<size_t>(kOpMaxParts) * n_kv_heads * 64 * 2);
}

spec_status spec_op_attention(int32_t dtype, int32_t n_seqs, const int32_t* rows, const int32_t* pos0,
                              const int32_t* page_table, int32_t max_pages, int32_t n_heads,
                              int32_t n_kv_heads, int32_t head_dim, const void* q, const void* k_pages,
                              const void* v_pages, void* out, void* workspace, size_t workspace_bytes,
                              void* stream) {
  if ((dtype != SPEC_F32 && dtype != SPEC_BF16) || n_seqs < 0 || max_pages <= 0 || n_heads <= 0 ||
      n_kv_heads <= 0 || n_heads % n_kv_heads)
    return SPEC_E_INVALID;
  if (head_dim != 64 && head_dim != 128) return SPEC_E_UNSUPPORTED;
  if (n_seqs == 0) return SPEC_OK;
  if (!rows || !pos0 || !page_table || !q || !k_pages || !v_pages || !out || !workspace) return SPEC_E_INVALID;
  int R = 0;
  std::vector<AttnSegment> segs;
  std::vector<int32_t> rseq, rpos;
  for (int i = 0; i < n_seqs; ++i) {
    if (rows[i] <= 0 || pos0[i] < 0 || ((pos0[i] + rows[i] + 15) / 16) > max_pages) return SPEC_E_INVALID;
    segs.push_back(AttnSegment{i, R, rows[i], pos0[i]});
    for (int r = 0; r < rows[i]; ++r) {
      rseq.push_back(i);
      rpos.push_back(pos0[i] + r);
    }
    R += rows[i];
  }
  if (workspace_bytes < spec_op_attention_workspace_bytes(n_seqs, R, max_pages, n_kv_heads, head_dim))
    return SPEC_E_INVALID;
  AttnPlan plan = plan_attention(segs, n_heads / n_kv_heads, n_kv_heads, kOpMaxParts);
  MetaBlock mb;
  const size_t opt = mb.add(page_table, static_cast<size_t>(n_seqs) * max_pages);
  const size_t ors = mb.add(rseq), orp = mb.add(rpos);
  const size_t oit = mb.add(plan.items), ogr = mb.add(plan.groups);
  char* ws = static_cast<char*>(workspace);
  const size_t meta_bytes = align_up(sizeof(int32_t) * (static_cast<size_t>(n_seqs) * max_pages + 2 * R)) +
                            align_up(sizeof(AttnItem) * (static_cast<size_t>(R) + kOpMaxParts)) +
                            align_up(sizeof(AttnGroup) * R);
  if (mb.size() > meta_bytes + 4 * 256) return SPEC_E_UNSUPPORTED;
  char* part = ws + align_up(meta_bytes + 4 * 256);
  hipStream_t st = static_cast<hipStream_t>(stream);
  {
    std::lock_guard<std::mutex> lk(g_mu);
    if (stager().upload(ws, mb.data(), mb.size(), st) != hipSuccess) return SPEC_E_HIP;
  }
  AttnArgs a;
  a.dtype = dtype == SPEC_F32 ? 0 : 1;
  a.Hq = n_heads;
  a.Hkv = n_kv_heads;
  a.hd = head_dim;
  a.q = q;
  a.kpool = k_pages;
  a.vpool = v_pages;
  a.page_table = reinterpret_cast<const int32_t*>(ws + opt);
  a.max_pages = max_pages;
  a.out = out;
  a.part_o = reinterpret_cast<float*>(part);
  a.part_ml = reinterpret_cast<float*>(part + align_up(sizeof(float) * static_cast<size_t>(kOpMaxParts) *
                                                       n_kv_heads * 64 * head_dim));
  if (a.dtype == 1 && plan.prefill)
    return hip_status(launch_attention_prefill_bf16(a, reinterpret_cast<const AttnItem*>(ws + oit),
                                                    static_cast<int>(plan.items.size()), plan.few_keys, st));
  if (a.dtype == 1)
    return hip_status(launch_attention_bf16(a, reinterpret_cast<const AttnItem*>(ws + oit),
                                            static_cast<int>(plan.items.size()),
                                            reinterpret_cast<const AttnGroup*>(ws + ogr),
                                            static_cast<int>(plan.groups.size()), plan.nt, plan.w, st));
  return hip_status(launch_attention_f32(a, R, reinterpret_cast<const int32_t*>(ws + ors),
                                         reinterpret_cast<const int32_t*>(ws + orp), st));
}

// ---------------------------------------------------------------------------
// token log probabilities

size_t spec_token_logprobs_workspace_bytes(int32_t rows, int32_t V, int32_t n_top) {
  if (rows <= 0 || V <= 0 || V > kMaxExtent || n_top < 0 || n_top > kLogprobMaxTop) return 0;
  return logprob_ws_bytes(logprob_plan(rows, V, n_top));
}

spec_status spec_token_logprobs(int32_t rows, int32_t V, const float* logits, int64_t row_stride,
                                const float* temperature, const int32_t* tokens, int32_t n_top, float* logprobs,
                                float* entropy, int32_t* top_ids, float* top_logprobs, void* workspace,
                                size_t workspace_bytes, void* stream) {
  if (rows < 0 || V <= 0 || row_stride < V) return refuse(SPEC_E_INVALID, "spec_token_logprobs: need rows >= 0, V > 0, row_stride >= V");
  if (V > kMaxExtent) return refuse(SPEC_E_UNSUPPORTED, "spec_token_logprobs: V must be at most 2^30");
  if (n_top < 0 || n_top > kLogprobMaxTop || n_top > V)
    return refuse(SPEC_E_INVALID, "spec_token_logprobs: need 0 <= n_top <= min(64, V)");
  if (rows == 0) return SPEC_OK;
  if (!logits || !workspace || (logprobs && !tokens) || (n_top > 0 && (!top_ids || !top_logprobs)))
    return refuse(SPEC_E_INVALID, "spec_token_logprobs: null pointer");
  if (misaligned(logits, 4) || misaligned(workspace, 16))
    return refuse(SPEC_E_INVALID, "spec_token_logprobs: misaligned logits or workspace");
  const LogprobPlan p = logprob_plan(rows, V, n_top);
  if (workspace_bytes < logprob_ws_bytes(p)) return refuse(SPEC_E_INVALID, "spec_token_logprobs: workspace too small");
  return launched(launch_logprobs(p, logits, row_stride, temperature, tokens, logprobs, entropy, top_ids,
                                    top_logprobs, workspace, static_cast<hipStream_t>(stream)), "spec_token_logprobs");
}

// ---------------------------------------------------------------------------
// cache pages

size_t spec_op_kv_copy_pages_workspace_bytes(int32_t n) { return n <= 0 ? 0 : align_up(sizeof(int2) * n); }

spec_status spec_op_kv_copy_pages(int32_t n_planes, int32_t num_pages, size_t page_bytes, void* pool, int32_t n,
                                  const int32_t* src_pages, const int32_t* dst_pages, void* workspace,
                                  size_t workspace_bytes, void* stream) try {
  if (n_planes < 0 || num_pages < 0 || n < 0) return refuse(SPEC_E_INVALID, "spec_op_kv_copy_pages: negative size");
  if (n == 0 || n_planes == 0) return SPEC_OK;
  if (!pool || !src_pages || !dst_pages || !workspace) return refuse(SPEC_E_INVALID, "spec_op_kv_copy_pages: null pointer");
  if (page_bytes == 0 || page_bytes % 16 || n_planes > 65535)
    return refuse(SPEC_E_UNSUPPORTED, "spec_op_kv_copy_pages: page_bytes must be a multiple of 16, n_planes at most 65535");
  if (misaligned(pool, 16) || misaligned(workspace, 16) || workspace_bytes < spec_op_kv_copy_pages_workspace_bytes(n))
    return refuse(SPEC_E_INVALID, "spec_op_kv_copy_pages: misaligned pool or workspace, or workspace too small");
  std::vector<uint64_t> is_dst((static_cast<size_t>(num_pages) + 63) / 64, 0);
  std::vector<int2> pairs(n);
  for (int i = 0; i < n; ++i) {
    const int32_t s = src_pages[i], d = dst_pages[i];
    if (s < 0 || s >= num_pages || d < 0 || d >= num_pages)
      return refuse(SPEC_E_INVALID, "spec_op_kv_copy_pages: page outside the pool");
    if (is_dst[d / 64] >> (d % 64) & 1) return refuse(SPEC_E_INVALID, "spec_op_kv_copy_pages: a page is a destination twice");
    is_dst[d / 64] |= uint64_t{1} << (d % 64);
    pairs[i] = make_int2(s, d);
  }
  for (int i = 0; i < n; ++i)
    if (is_dst[src_pages[i] / 64] >> (src_pages[i] % 64) & 1)
      return refuse(SPEC_E_INVALID, "spec_op_kv_copy_pages: a destination is also a source");
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool in_args = sizeof(int2) * n <= kUploadInline;
  if (!in_args) {
    MetaBlock mb;
    mb.add(pairs);
    const spec_status s = upload_tables(workspace, mb, "spec_op_kv_copy_pages: more pairs than a captured call takes", st);
    if (s != SPEC_OK) return s;
  }
  return launched(launch_kv_copy_pages(in_args ? pairs.data() : static_cast<const int2*>(workspace), n, in_args, pool,
                                         n_planes, num_pages, page_bytes, st), "spec_op_kv_copy_pages");
} catch (const std::exception&) {
  return refuse(SPEC_E_UNSUPPORTED, "spec_op_kv_copy_pages: out of host memory");
}

// ---------------------------------------------------------------------------
// the 4-bit cache

size_t spec_kv4_page_bytes(int32_t n_kv_heads, int32_t head_dim) {
  if (n_kv_heads <= 0 || (head_dim != 64 && head_dim != 128)) return 0;
  return static_cast<size_t>(n_kv_heads) * kv4_block_bytes(head_dim);
}

spec_status spec_op_rope_kv4(int32_t dtype, int32_t R, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                             float theta, const float* qkv, const int32_t* pos, const int32_t* slot,
                             int32_t num_pages, void* q_out, void* k_pages, void* v_pages, void* stream) {
  if ((dtype != SPEC_F32 && dtype != SPEC_BF16) || R < 0 || n_heads <= 0 || n_heads > kMaxHeads || n_kv_heads <= 0 ||
      n_kv_heads > kMaxHeads || !(theta > 0.f) || num_pages < 0 || num_pages > kMaxSlotPages)
    return refuse(SPEC_E_INVALID, "spec_op_rope_kv4: bad dtype or size");
  if (head_dim != 64 && head_dim != 128) return refuse(SPEC_E_UNSUPPORTED, "spec_op_rope_kv4: head_dim must be 64 or 128");
  if (R == 0) return SPEC_OK;
  if (!qkv || !pos || !slot || !q_out || (num_pages > 0 && (!k_pages || !v_pages)))
    return refuse(SPEC_E_INVALID, "spec_op_rope_kv4: null pointer");
  if (misaligned(qkv, 16) || misaligned(q_out, 16) || misaligned(k_pages, 16) || misaligned(v_pages, 16))
    return refuse(SPEC_E_INVALID, "spec_op_rope_kv4: qkv, q_out and the pages must be 16-byte aligned");
  return launched(launch_rope_kv4(dtype == SPEC_F32 ? 0 : 1, R, n_heads, n_kv_heads, head_dim, theta, qkv, pos, slot,
                                    num_pages, q_out, k_pages, v_pages, static_cast<hipStream_t>(stream)), "spec_op_rope_kv4");
}

spec_status spec_op_kv4_read(int32_t dtype, int32_t R, int32_t n_kv_heads, int32_t head_dim, const int32_t* slot,
                             int32_t num_pages, const void* k_pages, const void* v_pages, void* k_out, void* v_out,
                             void* stream) {
  if ((dtype != SPEC_F32 && dtype != SPEC_BF16) || R < 0 || n_kv_heads <= 0 || n_kv_heads > kMaxHeads ||
      num_pages < 0 || num_pages > kMaxSlotPages)
    return refuse(SPEC_E_INVALID, "spec_op_kv4_read: bad dtype or size");
  if (head_dim != 64 && head_dim != 128) return refuse(SPEC_E_UNSUPPORTED, "spec_op_kv4_read: head_dim must be 64 or 128");
  if (R == 0 || num_pages == 0) return SPEC_OK;
  if (!slot || !k_pages || !v_pages || !k_out || !v_out) return refuse(SPEC_E_INVALID, "spec_op_kv4_read: null pointer");
  if (misaligned(k_pages, 16) || misaligned(v_pages, 16) || misaligned(k_out, 16) || misaligned(v_out, 16))
    return refuse(SPEC_E_INVALID, "spec_op_kv4_read: the pages and outputs must be 16-byte aligned");
  return launched(launch_kv4_read(dtype == SPEC_F32 ? 0 : 1, R, n_kv_heads, head_dim, slot, num_pages, k_pages,
                                    v_pages, k_out, v_out, static_cast<hipStream_t>(stream)), "spec_op_kv4_read");
}

namespace {

// One spec_op_attention_kv4 call: its work and the layout of its workspace.
struct Kv4Call {
  spec_status status = SPEC_E_INVALID;
  const char* why = "";
  int R = 0;
  int64_t pages = 0;  // of all sequences (expanded form)
  AttnPlan plan;
  size_t tables = 0, o_part = 0, o_ml = 0, o_k = 0, o_v = 0, bytes = 0;
};

Kv4Call kv4_call(int32_t dtype, int32_t n_seqs, const int32_t* rows, const int32_t* pos0, int32_t max_pages,
                 int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
  Kv4Call c;
  auto fail = [&](spec_status s, const char* why) {
    c.status = s;
    c.why = why;
    return c;
  };
  if ((dtype != SPEC_F32 && dtype != SPEC_BF16) || n_seqs < 0 || max_pages <= 0 || n_heads <= 0 || n_heads > kMaxHeads ||
      n_kv_heads <= 0 || n_heads % n_kv_heads)
    return fail(SPEC_E_INVALID, "spec_op_attention_kv4: bad dtype or size");
  const int G = n_heads / n_kv_heads, dt = dtype == SPEC_F32 ? 0 : 1;
  if (head_dim != 64 && head_dim != 128) return fail(SPEC_E_UNSUPPORTED, "spec_op_attention_kv4: head_dim must be 64 or 128");
  if (G > 16 * (dt == 0 ? kKv4MaxNtF32 : kKv4MaxNt))
    return fail(SPEC_E_UNSUPPORTED, "spec_op_attention_kv4: more query heads per kv head than a tile holds (64 for bf16, 32 for fp32)");
  if (n_seqs > 0 && (!rows || !pos0)) return fail(SPEC_E_INVALID, "spec_op_attention_kv4: null pointer");
  std::vector<AttnSegment> segs;
  int64_t R = 0;
  for (int i = 0; i < n_seqs; ++i) {
    const int64_t len = static_cast<int64_t>(pos0[i]) + rows[i];
    if (rows[i] < 0 || pos0[i] < 0 || len > kMaxExtent || (len + 15) / 16 > max_pages)
      return fail(SPEC_E_INVALID, "spec_op_attention_kv4: rows beyond the page table or 2^30 positions, or a negative length");
    if (R + rows[i] > INT32_MAX) return fail(SPEC_E_INVALID, "spec_op_attention_kv4: too many rows");
    if (rows[i] > 0) segs.push_back(AttnSegment{i, static_cast<int32_t>(R), rows[i], pos0[i]});
    if (rows[i] > 0) c.pages += (len + 15) / 16;
    R += rows[i];
  }
  if (c.pages > INT32_MAX) return fail(SPEC_E_INVALID, "spec_op_attention_kv4: too many pages");
  c.R = static_cast<int>(R);
  c.status = SPEC_OK;
  if (R == 0) return c;
  c.plan = plan_kv4(segs, G, n_kv_heads, kOpMaxParts, dt == 0);
  // the page ids that the call reads, one sequence after the other: an item finds
  // its sequence's at it.seq (the kernels' max_pages is 1)
  std::vector<int32_t> first(n_seqs, 0);
  int64_t pages = 0;
  for (const AttnSegment& s : segs) {
    first[s.seq] = static_cast<int32_t>(pages);
    pages += (static_cast<int64_t>(s.pos0) + s.nrows + 15) / 16;
  }
  for (AttnItem& it : c.plan.items) it.seq = first[it.seq];
  c.tables = align_up(sizeof(int32_t) * c.pages) + align_up(sizeof(AttnItem) * c.plan.items.size()) +
             align_up(sizeof(AttnGroup) * c.plan.groups.size()) +
             (c.plan.prefill ? align_up(sizeof(int32_t) * c.pages) : 0);
  c.o_part = c.tables;
  c.o_ml = c.o_part + align_up(sizeof(float) * static_cast<size_t>(c.plan.n_parts) * n_kv_heads * 64 * head_dim);
  c.o_k = c.o_ml + align_up(sizeof(float) * static_cast<size_t>(c.plan.n_parts) * n_kv_heads * 64 * 2);
  const size_t pool = c.plan.prefill ? align_up(size_t{2} * c.pages * n_kv_heads * 16 * head_dim) : 0;
  c.o_v = c.o_k + pool;
  c.bytes = c.o_v + pool;
  return c;
}

}  // namespace

size_t spec_op_attention_kv4_workspace_bytes(int32_t dtype, int32_t n_seqs, const int32_t* rows, const int32_t* pos0,
                                             int32_t max_pages, int32_t n_heads, int32_t n_kv_heads,
                                             int32_t head_dim) try {
  const Kv4Call c = kv4_call(dtype, n_seqs, rows, pos0, max_pages, n_heads, n_kv_heads, head_dim);
  if (c.status != SPEC_OK) set_global_error(c.why);
  return c.status == SPEC_OK ? c.bytes : 0;
} catch (const std::exception&) {
  set_global_error("spec_op_attention_kv4: out of host memory");
  return 0;
}

spec_status spec_op_attention_kv4(int32_t dtype, int32_t n_seqs, const int32_t* rows, const int32_t* pos0,
                                  const int32_t* page_table, int32_t max_pages, int32_t num_pages, int32_t n_heads,
                                  int32_t n_kv_heads, int32_t head_dim, const void* q, const void* k_pages,
                                  const void* v_pages, void* out, void* workspace, size_t workspace_bytes,
                                  void* stream) try {
  Kv4Call c = kv4_call(dtype, n_seqs, rows, pos0, max_pages, n_heads, n_kv_heads, head_dim);
  if (c.status != SPEC_OK) return refuse(c.status, c.why);
  if (c.R == 0) return SPEC_OK;
  if (!page_table || !q || !k_pages || !v_pages || !out || !workspace)
    return refuse(SPEC_E_INVALID, "spec_op_attention_kv4: null pointer");
  if (misaligned(q, 16) || misaligned(k_pages, 16) || misaligned(v_pages, 16) || misaligned(out, 16) ||
      misaligned(workspace, 256) || workspace_bytes < c.bytes)
    return refuse(SPEC_E_INVALID,
                  "spec_op_attention_kv4: buffers must be 16-byte aligned, the workspace 256-byte aligned and large enough");
  std::vector<int32_t> table, src;
  table.reserve(c.pages);
  for (int i = 0; i < n_seqs; ++i) {
    const int n = rows[i] > 0 ? static_cast<int>((static_cast<int64_t>(pos0[i]) + rows[i] + 15) / 16) : 0;
    const int32_t* from = page_table + static_cast<size_t>(i) * max_pages;
    for (int j = 0; j < n; ++j)
      if (from[j] < 0 || from[j] >= num_pages)
        return refuse(SPEC_E_INVALID, "spec_op_attention_kv4: page outside the pool");
    table.insert(table.end(), from, from + n);
  }
  if (c.plan.prefill) {  // the prompt kernel reads expanded pages, numbered as they are listed
    src.swap(table);
    table.resize(src.size());
    for (size_t j = 0; j < table.size(); ++j) table[j] = static_cast<int32_t>(j);
  }
  MetaBlock mb;
  const size_t opt = mb.add(table), oit = mb.add(c.plan.items), ogr = mb.add(c.plan.groups), osr = mb.add(src);
  char* ws = static_cast<char*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  // small tables of a call that is one kernel travel in its arguments
  int max_item_pages = 0, max_parts = 0;
  for (const AttnItem& it : c.plan.items) max_item_pages = std::max(max_item_pages, (it.t1 + 15) / 16 - it.t0 / 16);
  for (const AttnGroup& g : c.plan.groups) max_parts = std::max(max_parts, g.nparts);
  const bool in_args = !c.plan.prefill && c.plan.groups.empty() && mb.size() <= kUploadInline &&
                       max_item_pages <= kKv4StagedPages;
  if (!in_args) {
    const spec_status s = upload_tables(ws, mb, "spec_op_attention_kv4: larger tables than a captured call takes", st);
    if (s != SPEC_OK) return s;
  }
  AttnArgs a;
  a.dtype = dtype == SPEC_F32 ? 0 : 1;
  a.Hq = n_heads;
  a.Hkv = n_kv_heads;
  a.hd = head_dim;
  a.q = q;
  a.kpool = k_pages;
  a.vpool = v_pages;
  a.page_table = reinterpret_cast<const int32_t*>(ws + opt);
  a.max_pages = 1;
  a.out = out;
  a.part_o = reinterpret_cast<float*>(ws + c.o_part);
  a.part_ml = reinterpret_cast<float*>(ws + c.o_ml);
  const AttnItem* items = reinterpret_cast<const AttnItem*>(ws + oit);
  const int n_items = static_cast<int>(c.plan.items.size());
  if (c.plan.prefill) {
    const hipError_t e = launch_kv4_expand(static_cast<int>(src.size()), reinterpret_cast<const int32_t*>(ws + osr),
                                           n_kv_heads, head_dim, k_pages, v_pages, ws + c.o_k, ws + c.o_v, st);
    if (e != hipSuccess) return launched(e, "spec_op_attention_kv4");
    a.kpool = ws + c.o_k;
    a.vpool = ws + c.o_v;
    return launched(launch_attention_prefill_bf16(a, items, n_items, c.plan.few_keys, st, true), "spec_op_attention_kv4");
  }
  Kv4Tables t;
  t.tables = in_args ? mb.data() : ws;
  t.inline_bytes = in_args ? mb.size() : 0;
  t.o_pt = opt;
  t.o_it = oit;
  t.o_gr = ogr;
  return launched(launch_attention_kv4(a, t, n_items, static_cast<int>(c.plan.groups.size()), max_parts, c.plan.nt,
                                         c.plan.w, st), "spec_op_attention_kv4");
} catch (const std::exception&) {
  return refuse(SPEC_E_UNSUPPORTED, "spec_op_attention_kv4: out of host memory");
}

// ---------------------------------------------------------------------------
// the latent cache

namespace {

// Sizes of a latent cache's heads and entries that the kernels are built for.
bool latent_sizes(int32_t nope_dim, int32_t rope_dim, int32_t rank) {
  return (nope_dim == 64 || nope_dim == 128) && (rope_dim == 32 || rope_dim == 64) && (rank == 256 || rank == 512);
}

}  // namespace

spec_status spec_op_rope_latent(int32_t dtype, int32_t R, int32_t n_heads, int32_t nope_dim, int32_t rope_dim,
                                int32_t rank, float theta, float eps, const float* q, const float* kv,
                                const void* norm_w, const int32_t* pos, const int32_t* slot, int32_t num_pages,
                                void* q_out, void* pages, void* stream) {
  if ((dtype != SPEC_F32 && dtype != SPEC_BF16) || R < 0 || n_heads <= 0 || n_heads > kMaxHeads || !(theta > 0.f) ||
      !(theta <= FLT_MAX) || !(eps >= 0.f) || num_pages < 0 || num_pages > kMaxSlotPages)
    return refuse(SPEC_E_INVALID, "spec_op_rope_latent: bad dtype or size");
  if (!latent_sizes(nope_dim, rope_dim, rank))
    return refuse(SPEC_E_UNSUPPORTED, "spec_op_rope_latent: nope_dim must be 64 or 128, rope_dim 32 or 64, rank 256 or 512");
  if (R == 0) return SPEC_OK;
  if (!q || !kv || !norm_w || !pos || !slot || !q_out || (num_pages > 0 && !pages))
    return refuse(SPEC_E_INVALID, "spec_op_rope_latent: null pointer");
  if (misaligned(q, 16) || misaligned(kv, 16) || misaligned(norm_w, 16) || misaligned(q_out, 16) || misaligned(pages, 16))
    return refuse(SPEC_E_INVALID, "spec_op_rope_latent: q, kv, norm_w, q_out and the pages must be 16-byte aligned");
  return launched(launch_rope_latent(dtype == SPEC_F32 ? 0 : 1, R, n_heads, nope_dim, rope_dim, rank, theta, eps, q, kv,
                                     norm_w, pos, slot, num_pages, q_out, pages, static_cast<hipStream_t>(stream)),
                  "spec_op_rope_latent");
}

namespace {

// One spec_op_attention_latent call: its work and the layout of its workspace.
struct LatentCall {
  spec_status status = SPEC_E_INVALID;
  const char* why = "";
  int64_t rows = 0;
  int64_t pages = 0, x_pages = 0;  // of the sequences in the absorbed and the expanded form
  std::vector<int> first, second;  // those sequences
  std::vector<int32_t> row_list;   // the absorbed form's rows, where both are taken
  int R = 0;                       // their number
  LatentPlan plan;
  LatentPromptPlan x;
  size_t o_q = 0, o_o = 0, o_part = 0, o_ml = 0, o_k = 0, o_v = 0, o_key = 0, o_xpart = 0, o_xml = 0, bytes = 0;
};

// Most bytes of expanded keys and values: beyond it (131072 keys of 32 heads of 128
// dims take 2 GiB) the absorbed form reads the cache itself.
constexpr int64_t kLatentMaxExpanded = int64_t{1} << 32;

LatentCall latent_call(int32_t dtype, int32_t n_seqs, const int32_t* rows, const int32_t* pos0, int32_t max_pages,
                       int32_t n_heads, int32_t nope_dim, int32_t rope_dim, int32_t rank, int32_t v_dim) {
  LatentCall c;
  auto fail = [&](spec_status s, const char* why) {
    c.status = s;
    c.why = why;
    return c;
  };
  if ((dtype != SPEC_F32 && dtype != SPEC_BF16) || n_seqs < 0 || max_pages <= 0 || n_heads <= 0 || n_heads > kMaxHeads)
    return fail(SPEC_E_INVALID, "spec_op_attention_latent: bad dtype or size");
  if (!latent_sizes(nope_dim, rope_dim, rank) || (v_dim != 64 && v_dim != 128))
    return fail(SPEC_E_UNSUPPORTED,
                "spec_op_attention_latent: nope_dim and v_dim must be 64 or 128, rope_dim 32 or 64, rank 256 or 512");
  if (n_seqs > 0 && (!rows || !pos0)) return fail(SPEC_E_INVALID, "spec_op_attention_latent: null pointer");
  const int64_t x_page = int64_t{32} * (static_cast<int64_t>(n_heads) * (nope_dim + v_dim) + rope_dim);  // bytes
  const int64_t weights = static_cast<int64_t>(n_heads) * (nope_dim + v_dim) * rank;
  std::vector<LatentSegment> segs, x_segs;
  for (int i = 0; i < n_seqs; ++i) {
    const int64_t len = static_cast<int64_t>(pos0[i]) + rows[i], pages = (len + 15) / 16;
    if (rows[i] < 0 || pos0[i] < 0 || len > kMaxExtent || pages > max_pages)
      return fail(SPEC_E_INVALID, "spec_op_attention_latent: rows beyond the page table or 2^30 positions, or a negative length");
    if ((c.rows + rows[i]) * n_heads > kMaxExtent)
      return fail(SPEC_E_INVALID, "spec_op_attention_latent: more than 2^30 rows x heads");
    if (rows[i] == 0) continue;
    if (c.pages + pages > kMaxExtent) return fail(SPEC_E_INVALID, "spec_op_attention_latent: too many pages");
    const int32_t row = static_cast<int32_t>(c.rows);
    if (dtype == SPEC_BF16 && latent_expands(rows[i], pos0[i], weights) && (c.x_pages + pages) * x_page <= kLatentMaxExpanded) {
      x_segs.push_back(LatentSegment{0, rows[i], pos0[i], static_cast<int32_t>(c.x_pages), row});
      c.second.push_back(i);
      c.x_pages += pages;
    } else {
      segs.push_back(LatentSegment{c.R, rows[i], pos0[i], static_cast<int32_t>(c.pages), row - c.R});
      c.first.push_back(i);
      c.pages += pages;
      c.R += rows[i];
    }
    c.rows += rows[i];
  }
  c.status = SPEC_OK;
  if (c.rows == 0) return c;
  const int waves = dtype == SPEC_F32 ? latent_f32_waves(rank) : 0;
  // (the expanded form's launches stay far below: 4 GiB of keys and values hold under 2^20 blocks x heads)
  if (latent_tiles(segs, n_heads, waves) > latent_max_items(waves))
    return fail(SPEC_E_UNSUPPORTED, "spec_op_attention_latent: more workgroups than a launch holds");
  if (c.R) c.plan = plan_latent(segs, n_heads, waves);
  c.x = plan_latent_prompt(x_segs, n_heads);
  if (c.R && c.R < c.rows)
    for (const LatentSegment& s : segs)
      for (int r = 0; r < s.nrows; ++r) c.row_list.push_back(s.row0 + s.qoff + r);
  const size_t elem = dtype == SPEC_F32 ? 4 : 2, lat = align_up(elem * c.R * n_heads * rank);
  c.o_q = align_up(sizeof(int32_t) * (c.pages + c.x_pages)) + align_up(sizeof(LatentItem) * c.plan.items.size()) +
          align_up(sizeof(LatentGroup) * c.plan.groups.size()) + align_up(sizeof(LatentItem) * c.x.items.size()) +
          align_up(sizeof(LatentGroup) * c.x.groups.size()) + align_up(sizeof(int32_t) * c.row_list.size());
  c.o_o = c.o_q + lat;
  c.o_part = c.o_o + lat;
  c.o_ml = c.o_part + align_up(sizeof(float) * static_cast<size_t>(c.plan.n_parts) * c.plan.tile * rank);
  c.o_k = c.o_ml + align_up(sizeof(float) * static_cast<size_t>(c.plan.n_parts) * c.plan.tile * 2);
  c.o_v = c.o_k + align_up(size_t{32} * c.x_pages * n_heads * nope_dim);
  c.o_key = c.o_v + align_up(size_t{32} * c.x_pages * n_heads * v_dim);
  // (the prompt kernel loads four pages at a time: up to three past the last)
  c.o_xpart = c.o_key + align_up(size_t{32} * c.x_pages * rope_dim) + (c.x_pages ? align_up(size_t{96} * n_heads * std::max(nope_dim, v_dim)) : 0);
  const size_t x_rows = static_cast<size_t>(c.x.n_parts) * c.x.rows * n_heads;
  c.o_xml = c.o_xpart + align_up(sizeof(float) * x_rows * v_dim);
  c.bytes = c.o_xml + align_up(sizeof(float) * x_rows * 2);
  return c;
}

}  // namespace

size_t spec_op_attention_latent_workspace_bytes(int32_t dtype, int32_t n_seqs, const int32_t* rows, const int32_t* pos0,
                                                int32_t max_pages, int32_t n_heads, int32_t nope_dim, int32_t rope_dim,
                                                int32_t rank, int32_t v_dim) try {
  const LatentCall c = latent_call(dtype, n_seqs, rows, pos0, max_pages, n_heads, nope_dim, rope_dim, rank, v_dim);
  if (c.status != SPEC_OK) set_global_error(c.why);
  return c.status == SPEC_OK ? c.bytes : 0;
} catch (const std::exception&) {
  set_global_error("spec_op_attention_latent: out of host memory");
  return 0;
}

spec_status spec_op_attention_latent(int32_t dtype, int32_t n_seqs, const int32_t* rows, const int32_t* pos0,
                                     const int32_t* page_table, int32_t max_pages, int32_t num_pages, int32_t n_heads,
                                     int32_t nope_dim, int32_t rope_dim, int32_t rank, int32_t v_dim, float scale,
                                     const void* q, const void* pages, const void* w_k, int64_t w_k_stride,
                                     const void* w_v, int64_t w_v_stride, void* out, void* workspace,
                                     size_t workspace_bytes, void* stream) try {
  const LatentCall c = latent_call(dtype, n_seqs, rows, pos0, max_pages, n_heads, nope_dim, rope_dim, rank, v_dim);
  if (c.status != SPEC_OK) return refuse(c.status, c.why);
  if (!(scale > 0.f) || !(scale <= 1e30f)) return refuse(SPEC_E_INVALID, "spec_op_attention_latent: scale must be positive and finite");
  if (c.rows == 0) return SPEC_OK;
  if (!page_table || !q || !pages || !w_k || !w_v || !out || !workspace)
    return refuse(SPEC_E_INVALID, "spec_op_attention_latent: null pointer");
  const int64_t unit = dtype == SPEC_F32 ? 4 : 8;  // elements in 16 bytes
  if (w_k_stride < static_cast<int64_t>(nope_dim) * rank || w_v_stride < static_cast<int64_t>(v_dim) * rank ||
      w_k_stride % unit || w_v_stride % unit || w_k_stride > (int64_t{1} << 40) || w_v_stride > (int64_t{1} << 40))
    return refuse(SPEC_E_INVALID, "spec_op_attention_latent: a head stride that is short, odd or beyond 2^40");
  if (misaligned(q, 16) || misaligned(pages, 16) || misaligned(w_k, 16) || misaligned(w_v, 16) || misaligned(out, 16) ||
      misaligned(workspace, 256) || workspace_bytes < c.bytes)
    return refuse(SPEC_E_INVALID,
                  "spec_op_attention_latent: buffers must be 16-byte aligned, the workspace 256-byte aligned and large enough");
  // the page ids that the call reads, one sequence after the other: the absorbed form's, then the expanded one's
  std::vector<int32_t> table;
  table.reserve(c.pages + c.x_pages);
  for (const std::vector<int>* seqs : {&c.first, &c.second})
    for (const int i : *seqs) {
      const int n = static_cast<int>((static_cast<int64_t>(pos0[i]) + rows[i] + 15) / 16);
      const int32_t* from = page_table + static_cast<size_t>(i) * max_pages;
      for (int j = 0; j < n; ++j)
        if (from[j] < 0 || from[j] >= num_pages)
          return refuse(SPEC_E_INVALID, "spec_op_attention_latent: page outside the pool");
      table.insert(table.end(), from, from + n);
    }
  MetaBlock mb;
  const size_t opt = mb.add(table), oit = mb.add(c.plan.items), ogr = mb.add(c.plan.groups), oxi = mb.add(c.x.items),
               oxg = mb.add(c.x.groups), orl = mb.add(c.row_list);
  char* ws = static_cast<char*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  // small tables of the absorbed form alone travel with its first kernel
  const size_t n_inline = align_up(mb.size(), 16);
  const bool in_args = c.x.items.empty() && n_inline <= kLatentInline;
  if (in_args) {
    mb.pad(n_inline);
  } else {
    const spec_status up = upload_tables(ws, mb, "spec_op_attention_latent: larger tables than a captured call takes", st);
    if (up != SPEC_OK) return up;
  }
  LatentArgs a;
  a.dtype = dtype == SPEC_F32 ? 0 : 1;
  a.H = n_heads;
  a.nope = nope_dim;
  a.rope = rope_dim;
  a.rank = rank;
  a.vdim = v_dim;
  a.R = c.R;
  a.row_list = c.row_list.empty() ? nullptr : reinterpret_cast<const int32_t*>(ws + orl);
  a.scale = scale * 1.4426950408889634f;
  a.q = q;
  a.pages = pages;
  a.w_k = w_k;
  a.w_v = w_v;
  a.k_stride = w_k_stride;
  a.v_stride = w_v_stride;
  a.page_list = reinterpret_cast<const int32_t*>(ws + opt);
  a.out = out;
  a.q_lat = ws + c.o_q;
  a.o_lat = ws + c.o_o;
  a.part_o = reinterpret_cast<float*>(ws + c.o_part);
  a.part_ml = reinterpret_cast<float*>(ws + c.o_ml);
  hipError_t e = hipSuccess;
  if (!c.x.items.empty()) {
    const LatentExpanded x{ws + c.o_k, ws + c.o_v, ws + c.o_key, reinterpret_cast<float*>(ws + c.o_xpart),
                           reinterpret_cast<float*>(ws + c.o_xml)};
    e = launch_latent_expand(a, a.page_list + c.pages, static_cast<int>(c.x_pages), x, st);
    if (e == hipSuccess)
      e = launch_latent_prompt(a, reinterpret_cast<const LatentItem*>(ws + oxi), static_cast<int>(c.x.items.size()), c.x.rows, x, st);
    if (e == hipSuccess)
      e = launch_latent_prompt_combine(a, reinterpret_cast<const LatentGroup*>(ws + oxg), static_cast<int>(c.x.groups.size()), c.x.rows, x, st);
  }
  if (c.R) {
    int max_parts = 0;
    for (const LatentGroup& g : c.plan.groups) max_parts = std::max(max_parts, g.nparts);
    if (e == hipSuccess) e = in_args ? launch_latent_absorb(a, st, ws, mb.data(), mb.size()) : launch_latent_absorb(a, st);
    if (e == hipSuccess)
      e = launch_latent_attention(a, reinterpret_cast<const LatentItem*>(ws + oit), static_cast<int>(c.plan.items.size()),
                                  c.plan.tile, st);
    if (e == hipSuccess)
      e = launch_latent_combine(a, reinterpret_cast<const LatentGroup*>(ws + ogr), static_cast<int>(c.plan.groups.size()),
                                c.plan.tile, max_parts, st);
    if (e == hipSuccess) e = launch_latent_values(a, st);
  }
  return launched(e, "spec_op_attention_latent");
} catch (const std::exception&) {
  return refuse(SPEC_E_UNSUPPORTED, "spec_op_attention_latent: out of host memory");
}

}  // extern "C"
