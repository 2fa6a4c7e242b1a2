// C ABI of the paged per-head cache: argument checks and launches. See include/sgdkv.h for the contract
// of every entry point.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "host_common.h"
#include "paged_internal.h"
#include "sgdkv.h"

namespace {

using sgdkv::host_check_device;
using sgdkv::host_ok;

constexpr int64_t kMaxInt = 0x7FFFFFFF;
// Rows of a segment: the kernels' row numbers may run a few tiles past the last one.
constexpr int64_t kMaxRows = kMaxInt - 2048;

sgdkv_status fail(sgdkv_status code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return sgdkv::host_fail(code, buf);
}

struct NamedPtr {
  const void* p;
  const char* name;
};

// Every pointer is set and 16-byte aligned.
sgdkv_status check_ptrs(std::initializer_list<NamedPtr> ptrs) {
  for (const NamedPtr& x : ptrs) {
    if (!x.p) return fail(SGDKV_ERR_INVALID_ARG, "NULL %s", x.name);
    if (reinterpret_cast<uintptr_t>(x.p) & 15u)
      return fail(SGDKV_ERR_INVALID_ARG, "%s is not 16-byte aligned", x.name);
  }
  return SGDKV_OK;
}

int log2_of(int x) {
  int n = 0;
  while ((1 << n) < x) ++n;
  return n;
}

sgdkv_status check_page_size(int32_t p) {
  if (p < sgdkv::kMinPage || p > sgdkv::kMaxPage || (p & (p - 1)))
    return fail(SGDKV_ERR_INVALID_ARG, "page_size %d is not a power of two from %d to %d", p, sgdkv::kMinPage,
                sgdkv::kMaxPage);
  return SGDKV_OK;
}

int elt_bytes(int32_t dtype) { return dtype == SGDKV_DTYPE_BF16 ? 2 : 4; }

// The pool without its pointers.
sgdkv_status check_pool_shape(const sgdkv_page_pool* p) {
  if (!p) return fail(SGDKV_ERR_INVALID_ARG, "NULL pool");
  if (p->reserved != 0) return fail(SGDKV_ERR_INVALID_ARG, "pool reserved must be 0");
  if (p->dtype != SGDKV_DTYPE_F32 && p->dtype != SGDKV_DTYPE_BF16)
    return fail(SGDKV_ERR_INVALID_ARG, "pool dtype %d", p->dtype);
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(SGDKV_ERR_UNSUPPORTED, "head_dim %d (built: 64, 128)", p->head_dim);
  return SGDKV_OK;
}

sgdkv_status check_pool(const sgdkv_page_pool* p) {
  if (sgdkv_status st = check_pool_shape(p)) return st;
  if (sgdkv_status st = check_page_size(p->page_size)) return st;
  if (p->num_pages < 1 || p->num_pages > kMaxInt / p->page_size)
    return fail(SGDKV_ERR_INVALID_ARG, "num_pages %lld outside [1, (2^31 - 1) / page_size]", (long long)p->num_pages);
  return check_ptrs({{p->k_pages, "k_pages"}, {p->v_pages, "v_pages"}});
}

hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }

sgdkv_status launched(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(SGDKV_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return host_ok();
}

// ------------------------------------------------------------- attention plan
sgdkv_status plan_paged(const sgdkv_page_pool* pool, const sgdkv_paged_desc* d, sgdkv::PagedAttnArgs& a,
                        size_t& bytes) {
  if (sgdkv_status st = check_pool_shape(pool)) return st;
  if (!d) return fail(SGDKV_ERR_INVALID_ARG, "NULL descriptor");
  if (d->batch < 1 || d->num_q_heads < 1 || d->num_kv_heads < 1)
    return fail(SGDKV_ERR_INVALID_ARG, "batch, num_q_heads, num_kv_heads must be >= 1");
  if (d->num_q_heads % d->num_kv_heads)
    return fail(SGDKV_ERR_INVALID_ARG, "num_q_heads %d is not a multiple of num_kv_heads %d", d->num_q_heads,
                d->num_kv_heads);
  const int G = d->num_q_heads / d->num_kv_heads;
  if (G > sgdkv::kMaxPagedGroup)
    return fail(SGDKV_ERR_UNSUPPORTED, "%d query heads per KV head > %d", G, sgdkv::kMaxPagedGroup);
  if (d->num_q_heads > 8192) return fail(SGDKV_ERR_UNSUPPORTED, "num_q_heads %d > 8192", d->num_q_heads);
  const int64_t nseg = (int64_t)d->batch * d->num_kv_heads;
  if (nseg > 65535) return fail(SGDKV_ERR_UNSUPPORTED, "batch * num_kv_heads = %lld > 65535", (long long)nseg);
  if (d->out_dtype != SGDKV_DTYPE_F32 && d->out_dtype != SGDKV_DTYPE_BF16)
    return fail(SGDKV_ERR_INVALID_ARG, "out_dtype %d", d->out_dtype);
  if (d->num_tokens < 0 || d->num_tokens > (kMaxInt - 128) / d->num_q_heads)  // a tile past the end still counts
    return fail(SGDKV_ERR_INVALID_ARG, "num_tokens %lld outside [0, (2^31 - 129) / num_q_heads]",
                (long long)d->num_tokens);
  if (d->max_new < 1) return fail(SGDKV_ERR_INVALID_ARG, "max_new %d < 1", d->max_new);
  if (d->causal != 0 && d->causal != 1) return fail(SGDKV_ERR_INVALID_ARG, "causal %d is not 0 or 1", d->causal);
  a = sgdkv::PagedAttnArgs{};
  a.B = d->batch;
  a.Hq = d->num_q_heads;
  a.Hkv = d->num_kv_heads;
  a.G = G;
  a.D = pool->head_dim;
  a.S = (int)nseg;
  a.inv_hkv = ((uint64_t(1) << 32) + a.Hkv - 1) / a.Hkv;
  a.T = (int)d->num_tokens;
  a.dtype = pool->dtype;
  a.out_dtype = d->out_dtype;
  a.causal = d->causal;
  a.max_pages = d->max_pages;
  a.max_new = (int)std::min<int64_t>(d->max_new, std::max<int64_t>(d->num_tokens, 1));
  const double scale = d->scale == 0.f ? 1.0 / std::sqrt((double)a.D) : (double)d->scale;
  const double c2 = scale * 1.4426950408889634074;
  if (!(std::fabs(c2) <= (double)FLT_MAX))
    return fail(SGDKV_ERR_INVALID_ARG, "scale %g: scale * log2(e) is not finite in fp32", d->scale);
  a.c2 = (float)c2;
  const sgdkv::PagedAttnShape shape = sgdkv::paged_attn_shape(a.dtype, G, a.max_new);
  a.tile_rows = shape.rows;
  a.key_tile = shape.key_tile;
  a.tokens = shape.rows / G;
  a.max_tiles = (a.max_new + a.tokens - 1) / a.tokens;
  a.by_tile = nseg * a.max_tiles <= sgdkv::kPagedWorkers;
  // What a tile takes beside its keys is as much as so many keys. (128 query rows of bf16: prompts of 800 tokens with
  // 64 / 8 heads 464 us with 128, 441 with 256, 455 with 512. fp32, whose keys take longer: 3 x 50 tokens over 1K
  // 22.5 us with 64, 30 with 128.)
  a.min_shift = log2_of(shape.rows < 128 ? 128 : (a.dtype ? 4 : 2) * shape.key_tile);
  // The workspace follows the bound the caller gave, whatever the tokens of this call.
  const int most_rows = sgdkv::paged_attn_shape(a.dtype, G, d->max_new).rows;
  bytes = (size_t)sgdkv::kPagedWorkers * (sizeof(int4) + 2 * (size_t)most_rows * (a.D + 2) * sizeof(float));
  return SGDKV_OK;
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
  if (nseg > sgdkv::kMaxPageSegs)
    return fail(SGDKV_ERR_UNSUPPORTED, "batch * num_kv_heads = %lld > %d", (long long)nseg, sgdkv::kMaxPageSegs);
  if (sgdkv_status st = check_page_size(desc->page_size)) return st;
  if (desc->max_pages < 1 || desc->max_pages > kMaxRows / desc->page_size)
    return fail(SGDKV_ERR_INVALID_ARG, "max_pages %d outside [1, (2^31 - 2049) / page_size]", desc->max_pages);
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
  sgdkv::PageArgs a{};
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
  return launched(sgdkv::launch_page_update(a, cus, stream_of(stream)), "page update");
}

sgdkv_status sgdkv_paged_store(const sgdkv_page_pool* pool, const void* k_rows, const void* v_rows,
                               const int32_t* slots, int64_t n, void* stream) {
  if (sgdkv_status st = check_pool(pool)) return st;
  if (n < 0 || n > (int64_t(1) << 40) / pool->head_dim)
    return fail(SGDKV_ERR_INVALID_ARG, "n = %lld rows out of range", (long long)n);
  if (n > 0)
    if (sgdkv_status st = check_ptrs({{k_rows, "k_rows"}, {v_rows, "v_rows"}, {slots, "slots"}})) return st;
  if (sgdkv_status st = host_check_device(nullptr)) return st;
  sgdkv::PagedStoreArgs a{};
  a.row_shift = log2_of(pool->head_dim * elt_bytes(pool->dtype) / 16);
  a.n = n;
  a.total_slots = pool->num_pages * pool->page_size;
  a.k = k_rows;
  a.v = v_rows;
  a.slots = slots;
  a.k_pages = pool->k_pages;
  a.v_pages = pool->v_pages;
  (void)hipGetLastError();
  return launched(sgdkv::launch_paged_store(a, stream_of(stream)), "paged store");
}

sgdkv_status sgdkv_norm_rope_store(const sgdkv_page_pool* pool, const sgdkv_norm_rope_desc* desc, const void* q,
                                   const void* k, const void* v, const int32_t* positions, const int32_t* slots,
                                   const float* inv_freq, const void* q_weight, const void* k_weight, void* q_out,
                                   void* stream) {
  if (sgdkv_status st = check_pool(pool)) return st;
  if (!desc) return fail(SGDKV_ERR_INVALID_ARG, "NULL descriptor");
  if (desc->reserved != 0) return fail(SGDKV_ERR_INVALID_ARG, "reserved must be 0");
  if (desc->num_q_heads < 0 || desc->num_kv_heads < 1)
    return fail(SGDKV_ERR_INVALID_ARG, "num_q_heads %d must be >= 0 and num_kv_heads %d >= 1", desc->num_q_heads,
                desc->num_kv_heads);
  if (desc->num_q_heads > 8192 || desc->num_kv_heads > 8192)
    return fail(SGDKV_ERR_UNSUPPORTED, "more than 8192 heads");
  const int64_t most = std::max(desc->num_q_heads, desc->num_kv_heads);
  if (desc->num_tokens < 0 || desc->num_tokens > kMaxInt / most)
    return fail(SGDKV_ERR_INVALID_ARG, "num_tokens %lld outside [0, (2^31 - 1) / heads]", (long long)desc->num_tokens);
  const int d = pool->head_dim, eb = elt_bytes(pool->dtype);
  if (desc->rot_dim < 0 || desc->rot_dim > d || desc->rot_dim % 16)
    return fail(SGDKV_ERR_INVALID_ARG, "rot_dim %d is not a multiple of 16 from 0 to %d", desc->rot_dim, d);
  if (desc->interleaved != 0 && desc->interleaved != 1)
    return fail(SGDKV_ERR_INVALID_ARG, "interleaved %d is not 0 or 1", desc->interleaved);
  if (!(desc->eps >= 0.f) || std::isinf(desc->eps)) return fail(SGDKV_ERR_INVALID_ARG, "eps must be >= 0 and finite");
  const struct {
    int64_t stride;
    int heads;
    const char* name;
  } strides[] = {{desc->q_stride, desc->num_q_heads, "q_stride"},
                 {desc->k_stride, desc->num_kv_heads, "k_stride"},
                 {desc->v_stride, desc->num_kv_heads, "v_stride"}};
  for (const auto& s : strides) {
    if (s.heads == 0) continue;
    if (s.stride < (int64_t)s.heads * d || s.stride > kMaxInt || (s.stride * eb) % 16)
      return fail(SGDKV_ERR_INVALID_ARG, "%s %lld is below heads * head_dim, above 2^31 - 1 or no multiple of 16 bytes",
                  s.name, (long long)s.stride);
  }
  if (desc->num_tokens > 0) {
    if (sgdkv_status st = check_ptrs({{k, "k"}, {v, "v"}, {positions, "positions"}, {slots, "slots"}})) return st;
    if (desc->num_q_heads > 0)
      if (sgdkv_status st = check_ptrs({{q, "q"}, {q_out, "q_out"}})) return st;
    if (desc->rot_dim > 0)
      if (sgdkv_status st = check_ptrs({{inv_freq, "inv_freq"}})) return st;
  }
  if (q_weight)
    if (sgdkv_status st = check_ptrs({{q_weight, "q_weight"}})) return st;
  if (k_weight)
    if (sgdkv_status st = check_ptrs({{k_weight, "k_weight"}})) return st;
  if (desc->num_q_heads > 0 && q_out && q_out == q && desc->q_stride != (int64_t)desc->num_q_heads * d)
    return fail(SGDKV_ERR_INVALID_ARG, "q_out may be q only where q is dense");
  if (sgdkv_status st = host_check_device(nullptr)) return st;
  sgdkv::NormRopeArgs a{};
  a.T = (int)desc->num_tokens;
  a.Hq = desc->num_q_heads;
  a.Hkv = desc->num_kv_heads;
  a.D = d;
  a.dtype = pool->dtype;
  a.rot = desc->rot_dim;
  a.interleaved = desc->interleaved;
  a.eps = desc->eps;
  a.q_stride = desc->q_stride * eb;
  a.k_stride = desc->k_stride * eb;
  a.v_stride = desc->v_stride * eb;
  a.total_slots = pool->num_pages * pool->page_size;
  a.q = q;
  a.k = k;
  a.v = v;
  a.positions = positions;
  a.slots = slots;
  a.inv_freq = inv_freq;
  a.q_weight = q_weight;
  a.k_weight = k_weight;
  a.q_out = q_out;
  a.k_pages = pool->k_pages;
  a.v_pages = pool->v_pages;
  (void)hipGetLastError();
  return launched(sgdkv::launch_norm_rope(a, stream_of(stream)), "norm, rotation and store");
}

sgdkv_status sgdkv_paged_attention_workspace_size(const sgdkv_page_pool* pool, const sgdkv_paged_desc* desc,
                                                  size_t* bytes) {
  if (!bytes) return fail(SGDKV_ERR_INVALID_ARG, "NULL bytes");
  sgdkv::PagedAttnArgs a;
  size_t n = 0;
  if (sgdkv_status st = plan_paged(pool, desc, a, n)) return st;
  *bytes = n;
  return host_ok();
}

sgdkv_status sgdkv_paged_attention(const sgdkv_page_pool* pool, const sgdkv_paged_desc* desc, const void* q,
                                   const int32_t* tables, const int32_t* rows, const int32_t* cu_new, void* out,
                                   float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  sgdkv::PagedAttnArgs a;
  size_t bytes = 0;
  if (sgdkv_status st = plan_paged(pool, desc, a, bytes)) return st;
  if (sgdkv_status st = check_pool(pool)) return st;
  if (desc->max_pages < 1 || desc->max_pages > kMaxRows / pool->page_size)
    return fail(SGDKV_ERR_INVALID_ARG, "max_pages %d outside [1, (2^31 - 2049) / page_size]", desc->max_pages);
  if (a.T > 0)
    if (sgdkv_status st =
            check_ptrs({{q, "q"}, {tables, "tables"}, {rows, "rows"}, {cu_new, "cu_new"}, {out, "out"}}))
      return st;
  if (lse_out)
    if (sgdkv_status st = check_ptrs({{lse_out, "lse_out"}})) return st;
  if (!workspace) return fail(SGDKV_ERR_WORKSPACE, "NULL workspace (%zu bytes needed)", bytes);
  if (reinterpret_cast<uintptr_t>(workspace) & 255u)
    return fail(SGDKV_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  if (workspace_bytes < bytes)
    return fail(SGDKV_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", workspace_bytes, bytes);
  if (sgdkv_status st = host_check_device(nullptr)) return st;
  if (a.T == 0) return host_ok();
  a.page_shift = log2_of(pool->page_size);
  a.num_pages = pool->num_pages;
  a.q = q;
  a.k_pages = pool->k_pages;
  a.v_pages = pool->v_pages;
  a.tables = tables;
  a.rows = rows;
  a.cu = cu_new;
  a.out = out;
  a.lse = lse_out;
  a.shared = static_cast<int4*>(workspace);
  a.part = reinterpret_cast<float*>(a.shared + sgdkv::kPagedWorkers);
  a.part_ms = a.part + 2 * (size_t)sgdkv::kPagedWorkers * a.tile_rows * a.D;
  (void)hipGetLastError();
  return launched(sgdkv::launch_paged_attention(a, stream_of(stream)), "paged attention");
}

}  // extern "C"
