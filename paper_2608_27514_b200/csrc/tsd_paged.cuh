// A paged K/V cache as the kernels see it (not part of the C ABI).
#pragma once
#include "tsd_common.cuh"

namespace tsd {

struct PagedView {
  const void *k, *v;
  int64_t ps_p, ps_r, ps_h;  // page, row, head strides in elements
  const float *k_scale, *v_scale;
  const int32_t* table;
  int64_t table_stride;
  int n_pages, shift, cap;  // page_size = 1 << shift; cap = tokens a sequence can have
};

// TSD_OK, or what is wrong with the description of a cache; nothing on the device is looked at.
int check_paged_cache(const tsd_paged_cache* c);
PagedView paged_view(const tsd_paged_cache& c);

#ifdef __CUDACC__
// Page of slot t, or -1 where the table holds no page of the pool.
__device__ __forceinline__ int page_of(const PagedView& c, int64_t s, int t) {
  const int page = c.table[s * c.table_stride + (t >> c.shift)];
  return page >= 0 && page < c.n_pages ? page : -1;
}
#endif

}  // namespace tsd
