// Paged caches: parameter blocks, the launchers that the C-ABI layer calls, and what their kernels share.
//
// K and V rows live in pools of pages, K [num_pages, h_kv, page_size, k] and V [num_pages, h_kv, page_size, v]; table [b, max_pages] names the pages of a
// sequence in order.  Position p of sequence i and head e is row (table[i, p / page_size] * h_kv + e) * page_size + p % page_size of the pool; an entry
// outside [0, num_pages) is a page that holds nothing: its rows are neither read nor written.
#pragma once
#include "common.hpp"

namespace mqa {

struct PagedCache {
  void* K;
  void* V;
  const int32_t* table;
  int num_pages, page_size, max_pages, h_kv;
  int k, v;
  __host__ __device__ int positions() const { return max_pages * page_size; }        // (at most 2^24)
};

struct PagedAppend {
  PagedCache c;
  const float* k_new;      // [b, n, h_kv, k]
  const float* v_new;      // [b, n, h_kv, v]
  const int32_t* counts;   // [b], or null: n rows each
  const int32_t* lens_in;
  int32_t* lens_out;
  int b, n;
};

// A decode launch's work is cut into pieces: every group (sequence, K/V head) into as many, of equal length, as make them no longer than a share of all groups'
// tiles of 32 positions; `blocks` workgroups have a piece, one for every block of query rows.  A group in one piece is finished by it; the others' pieces leave
// partial softmax states, which a second launch merges.  (Pieces that run on from one group into the next, all of the same length, were slower: a
// workgroup's start and end, 5 us, are then paid twice in a row.)
struct PagedDecode {
  PagedCache c;
  const float* q;          // [b, n, h, k]
  const int32_t* lens;
  float* o;                // [b, n, h, v]
  const float* scores_in;  // [b, h_kv, positions], or null: zeros
  float* scores_out;       // the same, or null
  float* part_o;           // [pieces, R, v]
  float* part_m;           // [pieces, R], log2 domain
  float* part_l;
  int2* spans;             // [b, h_kv]: a group's first piece, and how many it has
  int4* work;              // [1 + pieces of one head], or null: the list of paged_list_kernel
  float* logits;           // with scores: [b, h_kv, R, positions rounded up to 32], log2 domain
  float2* stats;           // with scores: [b, h_kv, R]: maximum, 1 / sum, of groups in one piece
  int b, n, h;
  int R;                   // query rows of a group: n * h / h_kv, query-major
  int block_rows, blocks;  // R in blocks
  int split;               // 0: piece g is group g
  float qscale;            // scale * log2(e)
  const float* K_scales;   // caches of 8 bits: [num_pages, h_kv, page_size / block]
  const float* V_scales;
  int block;               // positions of a scale
};

struct PagedEvict {
  PagedCache c;
  const int32_t* lens_in;
  const float* scores_in;  // [b, h_kv, positions]
  const int32_t* table_out;
  int max_pages_out;
  int32_t* lens_out;
  float* scores_out;       // [b, h_kv, max_pages_out * page_size]
  int32_t* kept;           // [b, h_kv, budget]
  int b, budget, recent;
};

struct PagedPlan {
  int form;                // the matrix kernel's widths: 64 or 128; -64, -128, -256: up to that
  int block_rows, blocks, split, pieces;      // pieces: at most
  int listed;              // so many sequences that their pieces are listed first
  size_t bytes;
};
constexpr int kPagedTile = 32;
constexpr int kPagedMaxRows = 1024;     // query rows of a K/V head

hipError_t launch_paged_append(const PagedAppend& p, int is_bf16, hipStream_t st);
// scaled: a cache of 8 bits
PagedPlan paged_plan(int b, int n, int h, int h_kv, int page_size, int max_pages, int k, int v, int is_bf16, int with_scores, bool scaled = false);
void paged_workspace(PagedDecode* p, const PagedPlan& plan, void* workspace);        // where its parts are
hipError_t launch_paged_decode(const PagedDecode& p, const PagedPlan& plan, int is_bf16, hipStream_t st);
hipError_t launch_paged_evict(const PagedEvict& p, int is_bf16, hipStream_t st);

// ---- caches of 8 bits (scaled_append.hip, scaled_decode.hip): `type` is MQA_E4M3 or MQA_INT8
struct ScaledAppend {
  PagedAppend a;
  float* K_scales;         // [num_pages, h_kv, page_size / block]
  float* V_scales;
  int block;               // positions of a scale; divides page_size
};
hipError_t launch_scaled_append(const ScaledAppend& p, int is_e4m3, hipStream_t st);
PagedPlan scaled_plan(int b, int n, int h, int h_kv, int page_size, int max_pages, int k, int v);
hipError_t launch_scaled_decode(const PagedDecode& p, const PagedPlan& plan, int is_e4m3, hipStream_t st);

// ---- who holds which page (pages.hip)
struct PageFork {
  const int32_t* table_in;  // [b_in, max_pages]
  const int32_t* lens_in;   // [b_in]
  const int32_t* parents;   // [b_out]
  int32_t* table_out;       // [b_out, max_pages]
  int32_t* lens_out;        // [b_out]
  int32_t* refs;            // [num_pages]
  int b_in, b_out, num_pages, page_size, max_pages;
};
struct PageFree {
  int32_t* table;           // [b, max_pages]
  const int32_t* lens;      // [b]
  int32_t* refs;
  int b, num_pages, page_size, max_pages;
};
struct PageReserve {
  int32_t* table;           // [b, max_pages]
  const int32_t* lens;      // [b]
  const int32_t* counts;    // [b], or null: n each
  int32_t* refs;
  int32_t* granted;         // [b]
  int32_t* moves;           // [b, 2]
  int b, n, num_pages, page_size, max_pages;
};
struct PageCompact {
  const int32_t* table_in;  // [b, max_pages]
  const int32_t* refs_in;   // [num_pages]
  int32_t* table_out;
  int32_t* refs_out;
  int32_t* moves;           // [moves_size, 2]
  int32_t* used;            // [1]
  int b, num_pages, max_pages, moves_size;
};
constexpr int kCopyPools = 16;          // of a launch
struct PageCopy {
  void* pool[kCopyPools];
  uint32_t page_bytes[kCopyPools];
  const int32_t* moves;     // [m, 2]
  int pools, m, num_pages;
};
hipError_t launch_fork(const PageFork& p, hipStream_t st);
hipError_t launch_free(const PageFree& p, hipStream_t st);
size_t reserve_workspace_bytes(int b, int n, int num_pages, int page_size);
hipError_t launch_reserve(const PageReserve& p, void* workspace, hipStream_t st);
size_t compact_workspace_bytes(int num_pages);
hipError_t launch_compact(const PageCompact& p, void* workspace, hipStream_t st);
hipError_t launch_copy_pages(const PageCopy& p, hipStream_t st);

// adjust_logits.hip
struct AdjustLogits {
  const float* logits;        // [b, n + 1, vocab]
  float* out;                 // the same, perhaps the same array
  const int32_t* history;     // [b, cap]
  const int32_t* lens;        // [b]
  const int32_t* prompts;     // [b], or null: 0 each
  const int32_t* drafts;      // [b, n]
  const float* repetition;    // [b], or null: 1
  const float* frequency;     // [b], or null: 0
  const float* presence;      // [b], or null: 0
  const int32_t* bias_tokens; // [b, biases]
  const float* bias_values;   // [b, biases]
  const uint32_t* allowed;    // [b, n + 1, ceil(vocab / 32)], or null: all
  int b, n, vocab, cap, biases;
};
hipError_t launch_adjust(const AdjustLogits& p, hipStream_t st);

// verify.hip
struct Verify {
  const float* logits;        // [b, n + 1, vocab]
  const float* draft_logits;  // [b, n, vocab], or null: a draft's distribution is the drafted token alone
  const int32_t* drafts;      // [b, n]
  const int32_t* counts;      // [b], or null: n each
  const float* u;             // [b, n + 1]
  int32_t* tokens;            // [b, n + 1]
  int32_t* accepted;          // [b]
  int b, n, vocab;
  float temperature;
};
size_t verify_workspace_bytes(int b, int n, int vocab);
hipError_t launch_verify(const Verify& p, void* workspace, hipStream_t st);

// ---------------------------------------------------------------- device helpers
// The row of a pool that position pos of head e is, or -1: it is on a page that holds nothing.
__device__ __forceinline__ int paged_row(const PagedCache& c, const int32_t* table, int e, int pos) {
  const unsigned page = (unsigned)pos / (unsigned)c.page_size;
  const int entry = table[page];
  return (unsigned)entry < (unsigned)c.num_pages ? (entry * c.h_kv + e) * c.page_size + (pos - (int)page * c.page_size) : -1;
}

__device__ __forceinline__ int paged_length(const PagedCache& c, int len) { return len < 0 ? 0 : min(len, c.positions()); }

}  // namespace mqa
