// C ABI of the paged per-head cache in 8 bits: argument checks and launches. See include/sgdkv.h for the contract
// of every entry point.
#include "paged_host_common.h"

namespace {

using namespace sgdkv;

sgdkv_status check_pool(const sgdkv_page_pool_fp8* p) {
  if (!p) return fail(SGDKV_ERR_INVALID_ARG, "NULL pool");
  if (p->reserved != 0) return fail(SGDKV_ERR_INVALID_ARG, "pool reserved must be 0");
  if (sgdkv_status st = check_dtype(p->row_dtype, "pool row_dtype")) return st;
  if (sgdkv_status st = check_head_dim(p->head_dim)) return st;
  if (sgdkv_status st = check_pages(p->num_pages, p->page_size)) return st;
  return check_ptrs({{p->k_pages, "k_pages"},
                     {p->v_pages, "v_pages"},
                     {p->k_scales, "k_scales"},
                     {p->v_scales, "v_scales"}});
}

uint8_t* bytes_of(void* p) { return static_cast<uint8_t*>(p); }

sgdkv_status plan(const sgdkv_page_pool_fp8* pool, const sgdkv_paged_desc* d, PagedAttnArgs& a, size_t& bytes) {
  if (!pool) return fail(SGDKV_ERR_INVALID_ARG, "NULL pool");
  if (pool->reserved != 0) return fail(SGDKV_ERR_INVALID_ARG, "pool reserved must be 0");
  if (sgdkv_status st = check_dtype(pool->row_dtype, "pool row_dtype")) return st;
  if (sgdkv_status st = check_head_dim(pool->head_dim)) return st;
  const auto shape = pool->head_dim == 128 ? paged_attn_fp8_shape_128 : paged_attn_fp8_shape_64;
  return plan_paged(pool->row_dtype, pool->head_dim, shape, d, a, bytes);
}

}  // namespace

extern "C" {

sgdkv_status sgdkv_paged_store_fp8(const sgdkv_page_pool_fp8* pool, const void* k_rows, const void* v_rows,
                                   const int32_t* slots, int64_t n, void* stream) {
  if (sgdkv_status st = check_pool(pool)) return st;
  if (n < 0 || n > (int64_t(1) << 40) / pool->head_dim)
    return fail(SGDKV_ERR_INVALID_ARG, "n = %lld rows out of range", (long long)n);
  if (n > 0)
    if (sgdkv_status st = check_ptrs({{k_rows, "k_rows"}, {v_rows, "v_rows"}, {slots, "slots"}})) return st;
  if (sgdkv_status st = host_check_device(nullptr)) return st;
  StoreFp8Args a{};
  a.D = pool->head_dim;
  a.dtype = pool->row_dtype;
  a.n = n;
  a.total_slots = pool->num_pages * pool->page_size;
  a.k = k_rows;
  a.v = v_rows;
  a.slots = slots;
  a.k_pages = bytes_of(pool->k_pages);
  a.v_pages = bytes_of(pool->v_pages);
  a.k_scales = bytes_of(pool->k_scales);
  a.v_scales = bytes_of(pool->v_scales);
  (void)hipGetLastError();
  return launched(launch_paged_store_fp8(a, stream_of(stream)), "paged store in 8 bits");
}

sgdkv_status sgdkv_norm_rope_store_fp8(const sgdkv_page_pool_fp8* pool, const sgdkv_norm_rope_desc* desc,
                                       float rope_factor, const void* q, const void* k, const void* v,
                                       const int32_t* positions, const int32_t* slots, const float* inv_freq,
                                       const void* q_weight, const void* k_weight, void* q_out, void* stream) {
  if (sgdkv_status st = check_pool(pool)) return st;
  if (!std::isfinite(rope_factor)) return fail(SGDKV_ERR_INVALID_ARG, "rope_factor must be finite");
  NormRopeArgs a;
  const NormRopePtrs x = {q, k, v, positions, slots, inv_freq, q_weight, k_weight, q_out};
  if (sgdkv_status st = plan_norm_rope(pool->row_dtype, pool->head_dim, desc, x, a)) return st;
  if (sgdkv_status st = host_check_device(nullptr)) return st;
  a.factor = rope_factor;
  a.total_slots = pool->num_pages * pool->page_size;
  a.k_pages = pool->k_pages;
  a.v_pages = pool->v_pages;
  a.k_scales = bytes_of(pool->k_scales);
  a.v_scales = bytes_of(pool->v_scales);
  (void)hipGetLastError();
  return launched(launch_norm_rope_fp8(a, stream_of(stream)), "norm, rotation and store in 8 bits");
}

sgdkv_status sgdkv_paged_attention_fp8_workspace_size(const sgdkv_page_pool_fp8* pool, const sgdkv_paged_desc* desc,
                                                      size_t* bytes) {
  if (!bytes) return fail(SGDKV_ERR_INVALID_ARG, "NULL bytes");
  PagedAttnArgs a;
  size_t n = 0;
  if (sgdkv_status st = plan(pool, desc, a, n)) return st;
  *bytes = n;
  return host_ok();
}

sgdkv_status sgdkv_paged_attention_fp8(const sgdkv_page_pool_fp8* pool, const sgdkv_paged_desc* desc, const void* q,
                                       const int32_t* tables, const int32_t* rows, const int32_t* cu_new, void* out,
                                       float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  PagedAttnArgs a;
  size_t bytes = 0;
  if (sgdkv_status st = plan(pool, desc, a, bytes)) return st;
  if (sgdkv_status st = check_pool(pool)) return st;
  AttnPtrs x = {q, tables, rows, cu_new, out, lse_out, workspace, workspace_bytes};
  if (sgdkv_status st = check_attention(desc, pool->page_size, x, bytes, a)) return st;
  if (sgdkv_status st = host_check_device(nullptr)) return st;
  if (a.T == 0) return host_ok();
  a.num_pages = pool->num_pages;
  a.k_pages = pool->k_pages;
  a.v_pages = pool->v_pages;
  a.k_scales = bytes_of(pool->k_scales);
  a.v_scales = bytes_of(pool->v_scales);
  (void)hipGetLastError();
  return launched(launch_paged_attention_fp8(a, stream_of(stream)), "paged attention in 8 bits");
}

}  // extern "C"
