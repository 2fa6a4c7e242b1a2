// C ABI of the paged per-head cache: argument checks and launches. See include/sgdkv.h for the contract
// of every entry point.
#include "paged_host_common.h"

namespace {

using namespace sgdkv;

// The pool without its pointers.
sgdkv_status check_pool_shape(const sgdkv_page_pool* p) {
  if (!p) return fail(SGDKV_ERR_INVALID_ARG, "NULL pool");
  if (p->reserved != 0) return fail(SGDKV_ERR_INVALID_ARG, "pool reserved must be 0");
  if (sgdkv_status st = check_dtype(p->dtype, "pool dtype")) return st;
  return check_head_dim(p->head_dim);
}

sgdkv_status check_pool(const sgdkv_page_pool* p) {
  if (sgdkv_status st = check_pool_shape(p)) return st;
  if (sgdkv_status st = check_pages(p->num_pages, p->page_size)) return st;
  return check_ptrs({{p->k_pages, "k_pages"}, {p->v_pages, "v_pages"}});
}

sgdkv_status plan(const sgdkv_page_pool* pool, const sgdkv_paged_desc* d, PagedAttnArgs& a, size_t& bytes) {
  if (sgdkv_status st = check_pool_shape(pool)) return st;
  return plan_paged(pool->dtype, pool->head_dim, paged_attn_shape, d, a, bytes);
}

}  // namespace

extern "C" {

sgdkv_status sgdkv_page_update(const sgdkv_page_desc* desc, const int32_t* rows, const int32_t* add, int32_t* tables,
                               int32_t* free_pages, const int32_t* head, int32_t* rows_out, int32_t* head_out,
                               int32_t* cu_out, int32_t* slots, int32_t* status, void* stream) {
  if (!desc) return fail(SGDKV_ERR_INVALID_ARG, "NULL descriptor");
  if (desc->reserved != 0) return fail(SGDKV_ERR_INVALID_ARG, "reserved must be 0");
  if (desc->batch < 1 || desc->num_kv_heads < 1)
    return fail(SGDKV_ERR_INVALID_ARG, "batch and num_kv_heads must be >= 1");
  const int64_t nseg = (int64_t)desc->batch * desc->num_kv_heads;
  if (nseg > kMaxPageSegs)
    return fail(SGDKV_ERR_UNSUPPORTED, "batch * num_kv_heads = %lld > %d", (long long)nseg, kMaxPageSegs);
  if (sgdkv_status st = check_page_size(desc->page_size)) return st;
  if (sgdkv_status st = check_max_pages(desc->max_pages, desc->page_size)) return st;
  if (nseg * desc->max_pages > kMaxInt)
    return fail(SGDKV_ERR_UNSUPPORTED, "%lld segments of %d table columns", (long long)nseg, desc->max_pages);
  if (desc->by_segment != 0 && desc->by_segment != 1)
    return fail(SGDKV_ERR_INVALID_ARG, "by_segment %d is not 0 or 1", desc->by_segment);
  if (desc->num_free < 1 || desc->num_free > kMaxInt)
    return fail(SGDKV_ERR_INVALID_ARG, "num_free %lld outside [1, 2^31 - 1]", (long long)desc->num_free);
  const int64_t per_row = desc->by_segment ? 1 : desc->num_kv_heads;
  if (desc->num_slots < 0 || desc->num_slots > kMaxInt / per_row)
    return fail(SGDKV_ERR_INVALID_ARG, "num_slots %lld out of range", (long long)desc->num_slots);
  if (sgdkv_status st = check_ptrs({{rows, "rows"},
                                    {add, "add"},
                                    {tables, "tables"},
                                    {free_pages, "free_pages"},
                                    {head, "head"},
                                    {rows_out, "rows_out"},
                                    {head_out, "head_out"},
                                    {cu_out, "cu_out"},
                                    {status, "status"}}))
    return st;
  if (desc->num_slots > 0)
    if (sgdkv_status st = check_ptrs({{slots, "slots"}})) return st;
  int cus = 0;
  if (sgdkv_status st = host_check_device(&cus)) return st;
  PageArgs a{};
  a.B = desc->batch;
  a.Hkv = desc->num_kv_heads;
  a.S = (int)nseg;
  a.page_shift = log2_of(desc->page_size);
  a.max_pages = desc->max_pages;
  a.by_segment = desc->by_segment;
  a.num_free = desc->num_free;
  a.num_slots = desc->num_slots;
  a.rows = rows;
  a.add = add;
  a.tables = tables;
  a.free_pages = free_pages;
  a.head = head;
  a.rows_out = rows_out;
  a.head_out = head_out;
  a.cu_out = cu_out;
  a.slots = slots;
  a.status = status;
  (void)hipGetLastError();
  return launched(launch_page_update(a, cus, stream_of(stream)), "page update");
}

sgdkv_status sgdkv_paged_store(const sgdkv_page_pool* pool, const void* k_rows, const void* v_rows,
                               const int32_t* slots, int64_t n, void* stream) {
  if (sgdkv_status st = check_pool(pool)) return st;
  if (n < 0 || n > (int64_t(1) << 40) / pool->head_dim)
    return fail(SGDKV_ERR_INVALID_ARG, "n = %lld rows out of range", (long long)n);
  if (n > 0)
    if (sgdkv_status st = check_ptrs({{k_rows, "k_rows"}, {v_rows, "v_rows"}, {slots, "slots"}})) return st;
  if (sgdkv_status st = host_check_device(nullptr)) return st;
  PagedStoreArgs a{};
  a.row_shift = log2_of(pool->head_dim * elt_bytes(pool->dtype) / 16);
  a.n = n;
  a.total_slots = pool->num_pages * pool->page_size;
  a.k = k_rows;
  a.v = v_rows;
  a.slots = slots;
  a.k_pages = pool->k_pages;
  a.v_pages = pool->v_pages;
  (void)hipGetLastError();
  return launched(launch_paged_store(a, stream_of(stream)), "paged store");
}

sgdkv_status sgdkv_norm_rope_store(const sgdkv_page_pool* pool, const sgdkv_norm_rope_desc* desc, const void* q,
                                   const void* k, const void* v, const int32_t* positions, const int32_t* slots,
                                   const float* inv_freq, const void* q_weight, const void* k_weight, void* q_out,
                                   void* stream) {
  if (sgdkv_status st = check_pool(pool)) return st;
  NormRopeArgs a;
  const NormRopePtrs x = {q, k, v, positions, slots, inv_freq, q_weight, k_weight, q_out};
  if (sgdkv_status st = plan_norm_rope(pool->dtype, pool->head_dim, desc, x, a)) return st;
  if (sgdkv_status st = host_check_device(nullptr)) return st;
  a.total_slots = pool->num_pages * pool->page_size;
  a.k_pages = pool->k_pages;
  a.v_pages = pool->v_pages;
  (void)hipGetLastError();
  return launched(launch_norm_rope(a, stream_of(stream)), "norm, rotation and store");
}

sgdkv_status sgdkv_paged_attention_workspace_size(const sgdkv_page_pool* pool, const sgdkv_paged_desc* desc,
                                                  size_t* bytes) {
  if (!bytes) return fail(SGDKV_ERR_INVALID_ARG, "NULL bytes");
  PagedAttnArgs a;
  size_t n = 0;
  if (sgdkv_status st = plan(pool, desc, a, n)) return st;
  *bytes = n;
  return host_ok();
}

sgdkv_status sgdkv_paged_attention(const sgdkv_page_pool* pool, const sgdkv_paged_desc* desc, const void* q,
                                   const int32_t* tables, const int32_t* rows, const int32_t* cu_new, void* out,
                                   float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  PagedAttnArgs a;
  size_t bytes = 0;
  if (sgdkv_status st = plan(pool, desc, a, bytes)) return st;
  if (sgdkv_status st = check_pool(pool)) return st;
  const AttnPtrs x = {q, tables, rows, cu_new, out, lse_out, workspace, workspace_bytes};
  if (sgdkv_status st = check_attention(desc, pool->page_size, x, bytes, a)) return st;
  if (sgdkv_status st = host_check_device(nullptr)) return st;
  if (a.T == 0) return host_ok();
  a.num_pages = pool->num_pages;
  a.k_pages = pool->k_pages;
  a.v_pages = pool->v_pages;
  (void)hipGetLastError();
  return launched(launch_paged_attention(a, stream_of(stream)), "paged attention");
}

}  // extern "C"
