// Pages of a K/V cache: where a position's row lies, shared by the kernels that read and write
// paged caches.
#pragma once
#include "common.cuh"

namespace hdsfa {

// A pool of num_pages pages of prow rows (P tokens x n streams), and page tables of max_pages
// entries a sequence: position p of a sequence is row p % prow of page table[p / prow].
struct PageGeom {
  int num_pages, max_pages, prow;
  FastDiv d_prow;
};
inline PageGeom make_page_geom(int num_pages, int max_pages, int prow) {
  return PageGeom{num_pages, max_pages, prow, make_fast_div((uint32_t)prow)};
}

// Pool row of position p >= 0 of the sequence whose page table is `table`; -1 where the table
// names no page of the pool.  Rows of a pool fit 31 bits (checked on the host).
__host__ __device__ inline int page_row(const PageGeom& g, const int32_t* table, int p) {
  const int i = fast_div(p, g.d_prow);
  if (i >= g.max_pages) return -1;
  const int id = table[i];
  return (unsigned)id < (unsigned)g.num_pages ? id * g.prow + (p - i * g.prow) : -1;
}

}  // namespace hdsfa
