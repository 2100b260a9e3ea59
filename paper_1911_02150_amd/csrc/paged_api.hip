// C-ABI layer of the paged caches and of the verification of drafted tokens: arguments are checked on the host before anything is enqueued.
#include "../../include/mqa.h"
#include "paged.hpp"

using namespace mqa;

namespace {

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// Sizes of a paged cache; rows of the pool are counted in 32 bits, and positions as the contiguous caches' are.
bool cache_sizes_ok(int b, int h_kv, int num_pages, int page_size, int max_pages, int k, int v) {
  if (b <= 0 || h_kv <= 0 || num_pages <= 0 || page_size <= 0 || max_pages <= 0 || k <= 0 || v <= 0) return false;
  if ((k & 7) || (v & 7) || k > 256 || v > 256) return false;
  const long long positions = (long long)max_pages * page_size;
  if (positions > (1ll << 24) || (long long)b * h_kv > (1ll << 24) || (long long)b * h_kv * (positions < 256 ? 256 : positions) > (1ll << 31)) return false;
  return (long long)num_pages * h_kv <= (1ll << 31) / page_size - 1;
}

PagedCache cache_of(const void* K, const void* V, const int32_t* table, int h_kv, int num_pages, int page_size, int max_pages, int k, int v) {
  PagedCache c;
  c.K = const_cast<void*>(K);
  c.V = const_cast<void*>(V);
  c.table = table;
  c.num_pages = num_pages; c.page_size = page_size; c.max_pages = max_pages; c.h_kv = h_kv;
  c.k = k; c.v = v;
  return c;
}

bool decode_sizes_ok(int b, int n, int h, int h_kv, int page_size, int max_pages, int k, int v) {
  if (n <= 0 || h <= 0 || !cache_sizes_ok(b, h_kv, 1, page_size, max_pages, k, v) || h % h_kv) return false;
  return (long long)n * (h / h_kv) <= kPagedMaxRows && (long long)b * n * h <= (1ll << 22);
}

}  // namespace

extern "C" {

int mqa_paged_append_kv_rows(const float* k_new, const float* v_new, const int32_t* counts, void* K_pages, void* V_pages, const int32_t* table,
                             const int32_t* lens_in, int32_t* lens_out, int b, int n, int h_kv, int num_pages, int page_size, int max_pages,
                             int k, int v, mqa_dtype dt, void* stream) {
  if (!k_new || !v_new || !K_pages || !V_pages || !table || !lens_in || !lens_out) return MQA_ERR_NULL;
  if (dt != MQA_F32 && dt != MQA_BF16) return MQA_ERR_DTYPE;
  if (n <= 0 || !cache_sizes_ok(b, h_kv, num_pages, page_size, max_pages, k, v) || n > max_pages * page_size) return MQA_ERR_SHAPE;
  if ((long long)b * n > (1ll << 30) / h_kv / ((k + v) >> 3)) return MQA_ERR_SHAPE;
  if (lens_in == lens_out || counts == lens_out) return MQA_ERR_SHAPE;      // (read by workgroups that come after one that has written)
  if (misaligned(k_new) || misaligned(v_new) || misaligned(K_pages) || misaligned(V_pages) || misaligned(table) || misaligned(lens_in) ||
      misaligned(lens_out) || (counts && misaligned(counts)))
    return MQA_ERR_ALIGN;
  PagedAppend p;
  p.c = cache_of(K_pages, V_pages, table, h_kv, num_pages, page_size, max_pages, k, v);
  p.k_new = k_new; p.v_new = v_new; p.counts = counts; p.lens_in = lens_in; p.lens_out = lens_out;
  p.b = b; p.n = n;
  return launch_paged_append(p, dt == MQA_BF16, static_cast<hipStream_t>(stream)) == hipSuccess ? MQA_OK : MQA_ERR_LAUNCH;
}

size_t mqa_paged_decode_workspace_bytes(int b, int n, int h, int h_kv, int page_size, int max_pages, int k, int v, mqa_dtype dt, int with_scores) {
  if ((dt != MQA_F32 && dt != MQA_BF16) || !decode_sizes_ok(b, n, h, h_kv, page_size, max_pages, k, v)) return 0;
  return paged_plan(b, n, h, h_kv, page_size, max_pages, k, v, dt == MQA_BF16, with_scores).bytes;
}

int mqa_paged_decode_step(const float* q, const void* K_pages, const void* V_pages, const int32_t* table, const int32_t* lens, float* o,
                          const float* scores_in, float* scores_out, int b, int n, int h, int h_kv, int num_pages, int page_size, int max_pages,
                          int k, int v, mqa_dtype dt, float scale, void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !K_pages || !V_pages || !table || !lens || !o || (scores_in && !scores_out)) return MQA_ERR_NULL;
  if (dt != MQA_F32 && dt != MQA_BF16) return MQA_ERR_DTYPE;
  if (!decode_sizes_ok(b, n, h, h_kv, page_size, max_pages, k, v) || !cache_sizes_ok(b, h_kv, num_pages, page_size, max_pages, k, v)) return MQA_ERR_SHAPE;
  if (misaligned(q) || misaligned(K_pages) || misaligned(V_pages) || misaligned(table) || misaligned(lens) || misaligned(o) ||
      (scores_in && misaligned(scores_in)) || (scores_out && misaligned(scores_out)))
    return MQA_ERR_ALIGN;
  const PagedPlan pl = paged_plan(b, n, h, h_kv, page_size, max_pages, k, v, dt == MQA_BF16, scores_out != nullptr);
  if (pl.bytes) {
    if (!workspace || workspace_bytes < pl.bytes) return MQA_ERR_WORKSPACE;
    if (misaligned(workspace)) return MQA_ERR_ALIGN;
  }
  PagedDecode p = {};
  p.c = cache_of(K_pages, V_pages, table, h_kv, num_pages, page_size, max_pages, k, v);
  p.q = q; p.lens = lens; p.o = o; p.scores_in = scores_in; p.scores_out = scores_out;
  p.b = b; p.n = n; p.h = h; p.R = n * (h / h_kv);
  p.block_rows = pl.block_rows; p.blocks = pl.blocks; p.split = pl.split;
  p.qscale = scale * kLog2e;      // (rounded, and once more with q: a logit is off by a step of its own size, as float32's scale * (q . k) and its exponential's base are)
  paged_workspace(&p, pl, workspace);
  return launch_paged_decode(p, pl, dt == MQA_BF16, static_cast<hipStream_t>(stream)) == hipSuccess ? MQA_OK : MQA_ERR_LAUNCH;
}

int mqa_paged_evict_kv(void* K_pages, void* V_pages, const int32_t* table_in, const int32_t* lens_in, const float* scores_in, const int32_t* table_out,
                       int32_t* lens_out, float* scores_out, int32_t* kept, int b, int h_kv, int num_pages, int page_size, int max_pages_in,
                       int max_pages_out, int k, int v, mqa_dtype dt, int budget, int recent, void* stream) {
  if (!K_pages || !V_pages || !table_in || !lens_in || !scores_in || !table_out || !lens_out || !scores_out || !kept) return MQA_ERR_NULL;
  if (dt != MQA_F32 && dt != MQA_BF16) return MQA_ERR_DTYPE;
  if (!cache_sizes_ok(b, h_kv, num_pages, page_size, max_pages_in, k, v) || !cache_sizes_ok(b, h_kv, num_pages, page_size, max_pages_out, k, v)) return MQA_ERR_SHAPE;
  if (budget <= 0 || recent < 0 || recent > budget || budget > max_pages_out * page_size) return MQA_ERR_SHAPE;
  if ((long long)b * h_kv >= (1 << 22) || (long long)b * h_kv * (budget + 15ll) >= (1 << 28)) return MQA_ERR_SHAPE;      // (grids of less than 2^32 threads)
  if (table_in == table_out || lens_in == lens_out || scores_in == scores_out) return MQA_ERR_SHAPE;      // not an in-place operation
  if (misaligned(K_pages) || misaligned(V_pages) || misaligned(table_in) || misaligned(lens_in) || misaligned(scores_in) || misaligned(table_out) ||
      misaligned(lens_out) || misaligned(scores_out) || misaligned(kept))
    return MQA_ERR_ALIGN;
  PagedEvict p;
  p.c = cache_of(K_pages, V_pages, table_in, h_kv, num_pages, page_size, max_pages_in, k, v);
  p.lens_in = lens_in; p.scores_in = scores_in; p.table_out = table_out; p.max_pages_out = max_pages_out;
  p.lens_out = lens_out; p.scores_out = scores_out; p.kept = kept;
  p.b = b; p.budget = budget; p.recent = recent;
  return launch_paged_evict(p, dt == MQA_BF16, static_cast<hipStream_t>(stream)) == hipSuccess ? MQA_OK : MQA_ERR_LAUNCH;
}

static bool verify_sizes_ok(int b, int n, int vocab) {
  return b > 0 && n >= 0 && vocab > 0 && n <= (1 << 16) && vocab <= (1 << 24) && (long long)b * (2 * n + 1) * ((vocab + 4095) / 4096) <= (1ll << 23);
}

size_t mqa_stack_verify_workspace_bytes(int b, int n, int vocab) { return verify_sizes_ok(b, n, vocab) ? verify_workspace_bytes(b, n, vocab) : 0; }

int mqa_stack_verify_drafts(const float* logits, const float* draft_logits, const int32_t* drafts, const int32_t* counts, const float* u,
                            int32_t* tokens, int32_t* accepted, int b, int n, int vocab, float temperature, void* workspace, size_t workspace_bytes,
                            void* stream) {
  if (!logits || (n > 0 && !drafts) || (temperature > 0.f && !u) || !tokens || !accepted) return MQA_ERR_NULL;
  if (!verify_sizes_ok(b, n, vocab) || !(temperature >= 0.f) || temperature > 1e30f) return MQA_ERR_SHAPE;
  if (!workspace || workspace_bytes < verify_workspace_bytes(b, n, vocab)) return MQA_ERR_WORKSPACE;
  if (misaligned(logits) || (draft_logits && misaligned(draft_logits)) || (drafts && misaligned(drafts)) || (counts && misaligned(counts)) ||
      (u && misaligned(u)) || misaligned(tokens) || misaligned(accepted) || misaligned(workspace))
    return MQA_ERR_ALIGN;
  Verify p;
  p.logits = logits; p.draft_logits = n > 0 ? draft_logits : nullptr; p.drafts = drafts; p.counts = counts; p.u = u; p.tokens = tokens; p.accepted = accepted;
  p.b = b; p.n = n; p.vocab = vocab; p.temperature = temperature;
  return launch_verify(p, workspace, static_cast<hipStream_t>(stream)) == hipSuccess ? MQA_OK : MQA_ERR_LAUNCH;
}

}  // extern "C"
