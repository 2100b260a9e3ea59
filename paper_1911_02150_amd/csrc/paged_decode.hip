// Attention over paged caches of float32 and bfloat16: the launch plan, the workspace and the launches.
#include "paged_decode.hpp"

namespace mqa {

// The parts of a call's workspace, each on 16 bytes; their size in all.
static size_t lay_out(PagedDecode* p, const PagedPlan& pl, float* at) {
  size_t floats = 0;
  auto take = [&](size_t count) {
    float* const here = at ? at + floats : nullptr;
    floats += (count + 3) & ~(size_t)3;
    return here;
  };
  const size_t states = (size_t)pl.pieces * p->R, groups = (size_t)p->b * p->c.h_kv;
  if (pl.split) {
    p->part_o = take(states * p->c.v);
    p->part_m = take(states);
    p->part_l = take(states);
    p->spans = reinterpret_cast<int2*>(take(groups * 2));
    if (pl.listed) p->work = reinterpret_cast<int4*>(take(4 * ((size_t)p->b + kShares + 1)));
  }
  if (p->scores_out) {
    p->stats = reinterpret_cast<float2*>(take(groups * p->R * 2));
    p->logits = take(groups * p->R * (((size_t)p->c.positions() + kPagedTile - 1) / kPagedTile * kPagedTile));
  }
  return floats * sizeof(float);
}

PagedPlan paged_plan(int b, int n, int h, int h_kv, int page_size, int max_pages, int k, int v, int is_bf16, int with_scores, bool scaled) {
  PagedPlan pl = {};
  const long long R = (long long)n * (h / h_kv), positions = (long long)max_pages * page_size, tiles = (positions + kPagedTile - 1) / kPagedTile;
  const int wide = k > v ? k : v;
  pl.form = k == v && (k == 64 || k == 128) ? k : wide <= 64 ? -64 : wide <= 128 ? -128 : -256;
  const long long groups = (long long)b * h_kv;
  // 16 query rows to a workgroup where the work is so little that its latency counts, else 32, whose tiles are read half as often: 16 sequences of 2048, 32 heads
  // 15.0 us against 19.1, 48 of them 22.7 and 23.2, 512 of up to 4096 with 64 heads 249 and 190; 8 sequences of 200, 64 heads 7.8 and 11.0; 256 wide, 32 heads, 16
  // sequences of 2048 24.4 and 28.5, 32 of them 32.5 and 32.0.
  // And only where a compute unit can hold them all, two each, three of 64 wide: 200 sequences of up to 100, 64 heads, 15.5 and 13.5; 64 wide 150 of 40 7.4 and 8.7.
  // (float32 rows of more than 64: 32 query rows do not fit a wave's registers beside a tile.)
  const bool little = groups * tiles * R * (pl.form == -256 ? 4 : 2) <= 3 << 16 && groups * ((R + 15) / 16) <= (wide <= 64 ? 3 : 2) * kComputeUnits;
  pl.block_rows = R <= 16 || little || (!is_bf16 && wide > 64) ? 16 : 32;
  pl.blocks = (int)((R + pl.block_rows - 1) / pl.block_rows);
  // One launch, a workgroup to a group, where cutting and merging would take longer (8 heads, 32 sequences of 500: 10.3 us, in pieces 12.0; of 640 12.9 and 12.3, of 800 15.7
  // and 12.6; one of 500 9.2 and 11.1, of 800 12.0 and 11.1; float32, one of 380 13.6 both, of 500 15.9 and 13.6), and to greater lengths where there is one for
  // every compute unit (256 of up to 1000, 32 heads: 25, in pieces 32).  8 bits: longer ones (8 heads, 32 of 640 11.7, in pieces 13.1, of 800 13.2 and 13.4; one of 640 11.5 and 12.3, of 1100 15.8 and
  // 12.5), and where there are 64 workgroups too (16 of up to 1000, 8 K/V heads of 64, 12.1 and 14.2; 64 of up to 800, 32 heads, 14.3 and 16.7); 300 of 1500, 32 heads, 37.5 and 56, of up to 1500 36.4
  // and 35.0, 512 of up to 2000 44.8 and 49.6.
  const bool heavy = wide > 128 || (!is_bf16 && wide > 64);
  const long long one = groups * pl.blocks;
  const int whole = scaled ? (one >= kComputeUnits ? 64 : heavy ? 12 : one >= 64 ? 32 : 24) : one >= kComputeUnits ? 32 : heavy ? 12 : 16;
  pl.split = tiles > whole;
  pl.listed = pl.split && b > kLookedFor;
  const long long least = groups * ((tiles + 3) / 4), most = groups + kShares;      // (pieces of four tiles; a last, shorter one in every group)
  pl.pieces = (int)(!pl.split ? groups : least < most ? least : most);
  PagedDecode p = {};
  p.b = b; p.R = (int)R;
  p.c.h_kv = h_kv; p.c.v = v; p.c.page_size = page_size; p.c.max_pages = max_pages;
  p.scores_out = with_scores ? reinterpret_cast<float*>(1) : nullptr;
  pl.bytes = lay_out(&p, pl, nullptr);
  return pl;
}

void paged_workspace(PagedDecode* p, const PagedPlan& pl, void* workspace) { lay_out(p, pl, static_cast<float*>(workspace)); }

template <typename T, int D, int HB, bool CACHED, bool EXACT>
static hipError_t launch_matrix(const PagedDecode& p, const PagedPlan& pl, hipStream_t st) {
  constexpr size_t lds = Lds<T, D, HB>::alone;
  return p.scores_out ? launch_form<paged_matrix_kernel<T, D, HB, true, CACHED, EXACT>>(lds, p, pl, st)
                      : launch_form<paged_matrix_kernel<T, D, HB, false, CACHED, EXACT>>(lds, p, pl, st);
}
template <typename T, int D, bool EXACT>
static hipError_t launch_rows(const PagedDecode& p, const PagedPlan& pl, hipStream_t st) {
  constexpr bool narrow = sizeof(T) == 4 && D > 64;             // (then never 32 rows)
  if constexpr (!EXACT) {
    if constexpr (!narrow)
      if (pl.block_rows == 32) return launch_matrix<T, D, 2, true, false>(p, pl, st);
    return launch_matrix<T, D, 1, true, false>(p, pl, st);
  } else if constexpr (narrow) {
    return pl.blocks > 1 ? launch_matrix<T, D, 1, true, true>(p, pl, st) : launch_matrix<T, D, 1, false, true>(p, pl, st);
  } else {
    if (pl.block_rows == 16) return pl.blocks > 1 ? launch_matrix<T, D, 1, true, true>(p, pl, st) : launch_matrix<T, D, 1, false, true>(p, pl, st);
    return pl.blocks > 1 ? launch_matrix<T, D, 2, true, true>(p, pl, st) : launch_matrix<T, D, 2, false, true>(p, pl, st);
  }
}

hipError_t launch_paged_decode(const PagedDecode& p, const PagedPlan& pl, int is_bf16, hipStream_t st) {
  hipError_t e = launch_list(p, pl, st);
  if (e != hipSuccess) return e;
  switch (pl.form) {
    case 64: e = is_bf16 ? launch_rows<uint16_t, 64, true>(p, pl, st) : launch_rows<float, 64, true>(p, pl, st); break;
    case 128: e = is_bf16 ? launch_rows<uint16_t, 128, true>(p, pl, st) : launch_rows<float, 128, true>(p, pl, st); break;
    case -64: e = is_bf16 ? launch_rows<uint16_t, 64, false>(p, pl, st) : launch_rows<float, 64, false>(p, pl, st); break;
    case -128: e = is_bf16 ? launch_rows<uint16_t, 128, false>(p, pl, st) : launch_rows<float, 128, false>(p, pl, st); break;
    default: e = is_bf16 ? launch_rows<uint16_t, 256, false>(p, pl, st) : launch_rows<float, 256, false>(p, pl, st); break;
  }
  return e != hipSuccess ? e : launch_finish(p, st);
}

}  // namespace mqa
