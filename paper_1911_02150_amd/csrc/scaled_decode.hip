// Attention over paged caches of 8 bits with a scale for each block of positions and head (the kernels' description: paged_decode.hpp).
#include "paged_decode.hpp"

namespace mqa {

PagedPlan scaled_plan(int b, int n, int h, int h_kv, int page_size, int max_pages, int k, int v, int is_e4m3) {
  return paged_plan(b, n, h, h_kv, page_size, max_pages, k, v, 1, 0);
}

template <typename T, int D, int HB, bool CACHED, bool EXACT>
static hipError_t launch_matrix(const PagedDecode& p, const PagedPlan& pl, hipStream_t st) {
  return launch_form<paged_matrix_kernel<T, D, HB, false, CACHED, EXACT>>(Lds<T, D, HB>::alone, p, pl, st);
}
template <typename T, int D, bool EXACT>
static hipError_t launch_rows(const PagedDecode& p, const PagedPlan& pl, hipStream_t st) {
  if constexpr (!EXACT) return pl.block_rows == 32 ? launch_matrix<T, D, 2, true, false>(p, pl, st) : launch_matrix<T, D, 1, true, false>(p, pl, st);
  else if (pl.block_rows == 16) return pl.blocks > 1 ? launch_matrix<T, D, 1, true, true>(p, pl, st) : launch_matrix<T, D, 1, false, true>(p, pl, st);
  else return pl.blocks > 1 ? launch_matrix<T, D, 2, true, true>(p, pl, st) : launch_matrix<T, D, 2, false, true>(p, pl, st);
}
template <typename T>
static hipError_t launch_widths(const PagedDecode& p, const PagedPlan& pl, hipStream_t st) {
  switch (pl.form) {
    case 64: return launch_rows<T, 64, true>(p, pl, st);
    case 128: return launch_rows<T, 128, true>(p, pl, st);
    case -64: return launch_rows<T, 64, false>(p, pl, st);
    case -128: return launch_rows<T, 128, false>(p, pl, st);
    default: return launch_rows<T, 256, false>(p, pl, st);
  }
}

hipError_t launch_scaled_decode(const PagedDecode& p, const PagedPlan& pl, int is_e4m3, hipStream_t st) {
  hipError_t e = launch_list(p, pl, st);
  if (e != hipSuccess) return e;
  e = is_e4m3 ? launch_widths<E4M3>(p, pl, st) : launch_widths<Int8>(p, pl, st);
  return e != hipSuccess ? e : launch_finish(p, st);
}

}  // namespace mqa
