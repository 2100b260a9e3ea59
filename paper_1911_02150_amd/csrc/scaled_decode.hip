// Attention over paged caches of 8 bits with a scale for each block of positions and head (the kernels' description: paged_decode.hpp).
#include "paged_decode.hpp"

namespace mqa {
namespace {

template <typename T>
__global__ __launch_bounds__(kThreads)
void scaled_plain_kernel(PagedDecode p) {
  extern __shared__ __align__(16) unsigned char smem[];
  Segment s;
  if (!find_segment(p, &s)) return;
  in_plain_form<T>(p, s, p.block_rows, smem);
}

}  // namespace

PagedPlan scaled_plan(int b, int n, int h, int h_kv, int page_size, int max_pages, int k, int v, int is_e4m3) {
  return paged_plan(b, n, h, h_kv, page_size, max_pages, k, v, 1, 0);
}

hipError_t launch_scaled_decode(const PagedDecode& p, const PagedPlan& pl, int is_e4m3, hipStream_t st) {
  hipError_t e = launch_list(p, pl, st);
  if (e != hipSuccess) return e;
  const size_t lds = scalar_lds_floats(p.c.k, p.c.v) * sizeof(float);
  e = is_e4m3 ? launch_form<scaled_plain_kernel<E4M3>>(lds, p, pl, st) : launch_form<scaled_plain_kernel<Int8>>(lds, p, pl, st);
  return e != hipSuccess ? e : launch_finish(p, st);
}

}  // namespace mqa
