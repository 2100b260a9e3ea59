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
PagedPlan paged_plan(int b, int n, int h, int h_kv, int page_size, int max_pages, int k, int v, int is_bf16, int with_scores);
void paged_workspace(PagedDecode* p, const PagedPlan& plan, void* workspace);        // where its parts are
hipError_t launch_paged_decode(const PagedDecode& p, const PagedPlan& plan, int is_bf16, hipStream_t st);
hipError_t launch_paged_evict(const PagedEvict& p, int is_bf16, hipStream_t st);

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
