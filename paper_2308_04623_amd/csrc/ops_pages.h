// What the operators of ssd_pages.h share: the checks of pools, sequences and rows, and
// the order of a block's bytes.
//
// The order is that of matrix-core operands, so that attention loads 16 bytes a lane,
// 1 KB a wave, straight into registers.  Lane (g, m) = 16 g + m of a wave holds, of 32 rows,
//   keys:   for each product of 16 rows and 32 dims row m's 8 dims,
//   values: for each product of 16 dims and 32 rows dim m's rows 4 g + r and 16 + 4 g + r, r < 4:
// those whose weights the lane has from the product before (the result of 16 rows and 16
// queries leaves rows 4 g + r in lane group g), so weights never change lanes.
#pragma once

#include "../../include/ssd_pages.h"
#include "ops_common.h"

namespace ssd {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

constexpr int kMaxPages = 1 << 20;

// bytes of a page's keys (or values) of one head
inline __host__ __device__ int block_bytes(const ssd_page_pool& p) { return p.page_rows * p.head_dim; }

inline ssd_status check_pool(const ssd_page_pool* p) {
  OP_REQUIRE(p, SSD_E_INVALID_ARG, "null pool");
  OP_REQUIRE(p->code == SSD_PAGE_INT8 || p->code == SSD_PAGE_E4M3, SSD_E_INVALID_ARG,
             "code must be SSD_PAGE_INT8 or SSD_PAGE_E4M3");
  OP_REQUIRE(p->page_rows == 32 || p->page_rows == 64 || p->page_rows == 128, SSD_E_UNSUPPORTED,
             "page_rows must be 32, 64 or 128");
  OP_REQUIRE(p->head_dim == 32 || p->head_dim == 64 || p->head_dim == 128, SSD_E_UNSUPPORTED,
             "head_dim must be 32, 64 or 128");
  OP_REQUIRE(p->n_layer >= 1 && p->n_layer <= 4096, SSD_E_INVALID_ARG, "n_layer outside [1, 4096]");
  OP_REQUIRE(p->n_page >= 1 && p->n_page <= kMaxPages, SSD_E_INVALID_ARG, "n_page outside [1, 2^20]");
  OP_REQUIRE(p->n_kv_head >= 1 && p->n_kv_head <= 1024, SSD_E_INVALID_ARG, "n_kv_head outside [1, 1024]");
  OP_REQUIRE(p->data && p->scale, SSD_E_INVALID_ARG, "null pool data");
  OP_REQUIRE((uintptr_t)p->data % 16 == 0 && (uintptr_t)p->scale % 8 == 0, SSD_E_UNSUPPORTED,
             "the pool's data is not 16-byte aligned, or its scales not 8-byte aligned");
  return SSD_OK;
}

inline ssd_status check_seqs(const ssd_page_seqs* s, int page_rows, bool refs) {
  OP_REQUIRE(s, SSD_E_INVALID_ARG, "null sequences");
  OP_REQUIRE(s->n_seq >= 1 && s->n_seq <= 4096, SSD_E_INVALID_ARG, "n_seq outside [1, 4096]");
  OP_REQUIRE(s->n_col >= 0 && (int64_t)s->n_col * page_rows < (1 << 30), SSD_E_INVALID_ARG,
             "n_col is negative, or its pages hold 2^30 rows");
  OP_REQUIRE(s->n_seq == 1 || s->table_ld >= s->n_col, SSD_E_INVALID_ARG, "table_ld below n_col");
  OP_REQUIRE(s->length && (s->table || s->n_col == 0) && (s->refs || !refs), SSD_E_INVALID_ARG,
             "null table, length or refs");
  OP_REQUIRE((uintptr_t)s->length % 4 == 0 && (uintptr_t)s->table % 4 == 0 && (uintptr_t)s->refs % 4 == 0,
             SSD_E_INVALID_ARG, "table, length or refs is not aligned to its elements");
  return SSD_OK;
}

// Rows of [n0][n1][n2][n3] with the desc's strides (layer, seq, and the two behind them)
struct RowDim {
  int64_t n, step;  // in elements
};
inline ssd_status check_rows(ssd_dtype dtype, const RowDim (&dims)[4], int head_dim, bool written,
                             const void* a, const void* b) {
  OP_REQUIRE(op_dtype(dtype), SSD_E_INVALID_ARG, "dtype must be SSD_F32 or SSD_BF16");
  OP_REQUIRE(a && b, SSD_E_INVALID_ARG, "null rows");
  OP_REQUIRE((uintptr_t)a % 16 == 0 && (uintptr_t)b % 16 == 0, SSD_E_UNSUPPORTED, "a pointer is not 16-byte aligned");
  const int unit = 16 / op_size(dtype);
  RowDim d[4];
  int n = 0;
  for (const RowDim& x : dims) {
    OP_REQUIRE(x.step >= 0, SSD_E_INVALID_ARG, "a stride is negative");
    OP_REQUIRE(x.step % unit == 0, SSD_E_UNSUPPORTED, "a stride is not a multiple of 16 bytes");
    if (x.n > 1) d[n++] = x;
  }
  if (!written) return SSD_OK;
  for (int i = 0; i < n; ++i)
    for (int j = i + 1; j < n; ++j)
      if (d[j].step < d[i].step) {
        const RowDim t = d[i];
        d[i] = d[j];
        d[j] = t;
      }
  int64_t reach = head_dim;
  for (int i = 0; i < n; ++i) {
    OP_REQUIRE(d[i].step >= reach, SSD_E_INVALID_ARG, "rows that are written overlap");
    reach += (d[i].n - 1) * d[i].step;
  }
  return SSD_OK;
}
// bytes from the first element to past the last
inline size_t rows_extent(ssd_dtype dtype, const RowDim (&dims)[4], int head_dim) {
  int64_t e = head_dim;
  for (const RowDim& x : dims) {
    if (x.n <= 0) return 0;
    e += (x.n - 1) * x.step;
  }
  return (size_t)e * op_size(dtype);
}

}  // namespace ssd
