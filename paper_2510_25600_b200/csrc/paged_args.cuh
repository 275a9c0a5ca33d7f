// Checks of a purekv_pages descriptor, shared by the paged calls, and the kernels' view of it.
#pragma once
#include "common.cuh"
#include "paged.cuh"

namespace purekv {

inline int64_t bytes_of(purekv_dtype t) { return t == PUREKV_E4M3 ? 1 : t == PUREKV_BF16 ? 2 : 4; }

// `dtype` is that of the rows that come and go: bf16 with pools of bf16 or e4m3, fp32 with pools of fp32.
inline purekv_status check_pages(const purekv_pages* p, purekv_dtype dtype, const char* where) {
  PK_REQUIRE(p->n_req >= 0 && p->max_pages >= 0 && p->n_pages >= 0 && p->page_size >= 1 && p->n_kv_heads >= 1 && p->head_dim >= 1,
             PUREKV_ERR_INVALID_ARG, "%s: bad sizes of the paged cache", where);
  PK_REQUIRE(p->n_kv_heads <= 65536 && p->head_dim <= 65536, PUREKV_ERR_UNSUPPORTED, "%s: too many heads, or too large ones", where);
  PK_REQUIRE(p->dtype == PUREKV_BF16 || p->dtype == PUREKV_FP32 || p->dtype == PUREKV_E4M3, PUREKV_ERR_INVALID_ARG,
             "%s: unknown dtype of the pools", where);
  PK_REQUIRE(p->dtype == dtype || (p->dtype == PUREKV_E4M3 && dtype == PUREKV_BF16), PUREKV_ERR_UNSUPPORTED,
             "%s: bf16 goes with pools of bf16 or e4m3, fp32 with pools of fp32", where);
  PK_REQUIRE(p->dtype == PUREKV_E4M3 || (!p->k_scale && !p->v_scale), PUREKV_ERR_INVALID_ARG, "%s: only e4m3 pools have scales", where);
  if (p->n_req == 0) return PUREKV_OK;
  PK_REQUIRE((p->block_table || p->max_pages == 0) && p->seq_lens, PUREKV_ERR_INVALID_ARG, "%s: null block_table or seq_lens", where);
  PK_REQUIRE(p->n_req == 1 || p->table_stride >= p->max_pages, PUREKV_ERR_INVALID_ARG, "%s: rows of the block table overlap", where);
  PK_REQUIRE(p->n_pages == 0 || (p->k && p->v), PUREKV_ERR_INVALID_ARG, "%s: null pool", where);
  PK_REQUIRE(((uintptr_t)p->k | (uintptr_t)p->v) % 16 == 0, PUREKV_ERR_INVALID_ARG, "%s: pools must be 16-byte aligned", where);
  const int64_t e = bytes_of(p->dtype), row = (int64_t)p->head_dim;
  const struct { int64_t stride; int32_t n; } dims[] = {{p->page_stride, p->n_pages}, {p->token_stride, p->page_size}, {p->head_stride, p->n_kv_heads}};
  for (const auto& d : dims)
    PK_REQUIRE(d.n <= 1 || (d.stride >= row && d.stride * e % 16 == 0), PUREKV_ERR_INVALID_ARG,
               "%s: the pools' strides must be multiples of 16 bytes and at least a row", where);
  PK_REQUIRE(row * e % 16 == 0, PUREKV_ERR_UNSUPPORTED, "%s: rows must be whole 16 bytes", where);
  return PUREKV_OK;
}

inline PagedView view_of(const purekv_pages* p) {
  const int64_t e = bytes_of(p->dtype);
  PagedView v;
  v.table = p->block_table;
  v.seq_lens = p->seq_lens;
  v.table_stride = p->n_req > 1 ? p->table_stride : 0;
  v.page_stride = p->n_pages > 1 ? p->page_stride * e : 0;
  v.token_stride = p->page_size > 1 ? p->token_stride * e : 0;
  v.head_stride = p->n_kv_heads > 1 ? p->head_stride * e : 0;
  v.n_pages = p->n_pages;
  v.max_pages = p->max_pages;
  v.page_size = FastDiv::of(p->page_size);
  return v;
}

}  // namespace purekv
