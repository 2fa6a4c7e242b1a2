// Argument checks and the attention plan of the paged cache's C ABI, shared by its host files.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>

#include "host_common.h"
#include "paged_internal.h"
#include "sgdkv.h"

namespace sgdkv {

constexpr int64_t kMaxInt = 0x7FFFFFFF;
// Rows of a segment: the kernels' row numbers may run a few tiles past the last one.
constexpr int64_t kMaxRows = kMaxInt - 2048;

inline sgdkv_status fail(sgdkv_status code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return host_fail(code, buf);
}

struct NamedPtr {
  const void* p;
  const char* name;
};

// Every pointer is set and 16-byte aligned.
inline sgdkv_status check_ptrs(std::initializer_list<NamedPtr> ptrs) {
  for (const NamedPtr& x : ptrs) {
    if (!x.p) return fail(SGDKV_ERR_INVALID_ARG, "NULL %s", x.name);
    if (reinterpret_cast<uintptr_t>(x.p) & 15u)
      return fail(SGDKV_ERR_INVALID_ARG, "%s is not 16-byte aligned", x.name);
  }
  return SGDKV_OK;
}

inline int log2_of(int x) {
  int n = 0;
  while ((1 << n) < x) ++n;
  return n;
}

inline sgdkv_status check_page_size(int32_t p) {
  if (p < kMinPage || p > kMaxPage || (p & (p - 1)))
    return fail(SGDKV_ERR_INVALID_ARG, "page_size %d is not a power of two from %d to %d", p, kMinPage, kMaxPage);
  return SGDKV_OK;
}

inline int elt_bytes(int32_t dtype) { return dtype == SGDKV_DTYPE_BF16 ? 2 : 4; }

inline sgdkv_status check_dtype(int32_t dtype, const char* what) {
  if (dtype != SGDKV_DTYPE_F32 && dtype != SGDKV_DTYPE_BF16)
    return fail(SGDKV_ERR_INVALID_ARG, "%s %d", what, dtype);
  return SGDKV_OK;
}

inline sgdkv_status check_head_dim(int32_t d) {
  if (d != 64 && d != 128) return fail(SGDKV_ERR_UNSUPPORTED, "head_dim %d (built: 64, 128)", d);
  return SGDKV_OK;
}

inline sgdkv_status check_pages(int64_t num_pages, int32_t page_size) {
  if (sgdkv_status st = check_page_size(page_size)) return st;
  if (num_pages < 1 || num_pages > kMaxInt / page_size)
    return fail(SGDKV_ERR_INVALID_ARG, "num_pages %lld outside [1, (2^31 - 1) / page_size]", (long long)num_pages);
  return SGDKV_OK;
}

inline sgdkv_status check_max_pages(int32_t max_pages, int32_t page_size) {
  if (max_pages < 1 || max_pages > kMaxRows / page_size)
    return fail(SGDKV_ERR_INVALID_ARG, "max_pages %d outside [1, (2^31 - 2049) / page_size]", max_pages);
  return SGDKV_OK;
}

inline hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }

inline sgdkv_status launched(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(SGDKV_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return host_ok();
}

// ------------------------------------------------------------- attention plan
// For queries of `dtype` and a cache whose kernel instances `shape_of` knows.
inline sgdkv_status plan_paged(int dtype, int head_dim, PagedAttnShape (*shape_of)(int, int, int),
                               const sgdkv_paged_desc* d, PagedAttnArgs& a, size_t& bytes) {
  if (!d) return fail(SGDKV_ERR_INVALID_ARG, "NULL descriptor");
  if (d->batch < 1 || d->num_q_heads < 1 || d->num_kv_heads < 1)
    return fail(SGDKV_ERR_INVALID_ARG, "batch, num_q_heads, num_kv_heads must be >= 1");
  if (d->num_q_heads % d->num_kv_heads)
    return fail(SGDKV_ERR_INVALID_ARG, "num_q_heads %d is not a multiple of num_kv_heads %d", d->num_q_heads,
                d->num_kv_heads);
  const int G = d->num_q_heads / d->num_kv_heads;
  if (G > kMaxPagedGroup)
    return fail(SGDKV_ERR_UNSUPPORTED, "%d query heads per KV head > %d", G, kMaxPagedGroup);
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
  a = PagedAttnArgs{};
  a.B = d->batch;
  a.Hq = d->num_q_heads;
  a.Hkv = d->num_kv_heads;
  a.G = G;
  a.D = head_dim;
  a.S = (int)nseg;
  a.inv_hkv = ((uint64_t(1) << 32) + a.Hkv - 1) / a.Hkv;
  a.T = (int)d->num_tokens;
  a.dtype = dtype;
  a.out_dtype = d->out_dtype;
  a.causal = d->causal;
  a.max_pages = d->max_pages;
  a.max_new = (int)std::min<int64_t>(d->max_new, std::max<int64_t>(d->num_tokens, 1));
  const double scale = d->scale == 0.f ? 1.0 / std::sqrt((double)a.D) : (double)d->scale;
  const double c2 = scale * 1.4426950408889634074;
  if (!(std::fabs(c2) <= (double)FLT_MAX))
    return fail(SGDKV_ERR_INVALID_ARG, "scale %g: scale * log2(e) is not finite in fp32", d->scale);
  a.c2 = (float)c2;
  const PagedAttnShape shape = shape_of(a.dtype, G, a.max_new);
  a.tile_rows = shape.rows;
  a.key_tile = shape.key_tile;
  a.tokens = shape.rows / G;
  a.max_tiles = (a.max_new + a.tokens - 1) / a.tokens;
  a.by_tile = nseg * a.max_tiles <= kPagedWorkers;
  // What a tile takes beside its keys is as much as so many keys. (128 query rows of bf16: prompts of 800 tokens with
  // 64 / 8 heads 464 us with 128, 441 with 256, 455 with 512. fp32, whose keys take longer: 3 x 50 tokens over 1K
  // 22.5 us with 64, 30 with 128.)
  a.min_shift = log2_of(shape.rows < 128 ? 128 : (a.dtype ? 4 : 2) * shape.key_tile);
  // The workspace follows the bound the caller gave, whatever the tokens of this call.
  const int most_rows = shape_of(a.dtype, G, d->max_new).rows;
  bytes = (size_t)kPagedWorkers * (sizeof(int4) + 2 * (size_t)most_rows * (a.D + 2) * sizeof(float));
  return SGDKV_OK;
}

struct AttnPtrs {
  const void* q;
  const int32_t* tables;
  const int32_t* rows;
  const int32_t* cu_new;
  void* out;
  float* lse_out;
  void* workspace;
  size_t workspace_bytes;
};

// The checks of a planned call's pointers and pages, and the arguments but for the pool's.
inline sgdkv_status check_attention(const sgdkv_paged_desc* desc, int32_t page_size, const AttnPtrs& x, size_t bytes,
                                    PagedAttnArgs& a) {
  if (sgdkv_status st = check_max_pages(desc->max_pages, page_size)) return st;
  if (a.T > 0)
    if (sgdkv_status st = check_ptrs(
            {{x.q, "q"}, {x.tables, "tables"}, {x.rows, "rows"}, {x.cu_new, "cu_new"}, {x.out, "out"}}))
      return st;
  if (x.lse_out)
    if (sgdkv_status st = check_ptrs({{x.lse_out, "lse_out"}})) return st;
  if (!x.workspace) return fail(SGDKV_ERR_WORKSPACE, "NULL workspace (%zu bytes needed)", bytes);
  if (reinterpret_cast<uintptr_t>(x.workspace) & 255u)
    return fail(SGDKV_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  if (x.workspace_bytes < bytes)
    return fail(SGDKV_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", x.workspace_bytes, bytes);
  a.page_shift = log2_of(page_size);
  a.q = x.q;
  a.tables = x.tables;
  a.rows = x.rows;
  a.cu = x.cu_new;
  a.out = x.out;
  a.lse = x.lse_out;
  a.shared = static_cast<int4*>(x.workspace);
  a.part = reinterpret_cast<float*>(a.shared + kPagedWorkers);
  a.part_ms = a.part + 2 * (size_t)kPagedWorkers * a.tile_rows * a.D;
  return SGDKV_OK;
}

struct NormRopePtrs {
  const void* q;
  const void* k;
  const void* v;
  const int32_t* positions;
  const int32_t* slots;
  const float* inv_freq;
  const void* q_weight;
  const void* k_weight;
  void* q_out;
};

// The checks of norm_rope_store's descriptor and pointers, and the arguments but for the pool's.
inline sgdkv_status plan_norm_rope(int dtype, int d, const sgdkv_norm_rope_desc* desc, const NormRopePtrs& x,
                                   NormRopeArgs& a) {
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
  const int eb = elt_bytes(dtype);
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
    if (sgdkv_status st = check_ptrs({{x.k, "k"}, {x.v, "v"}, {x.positions, "positions"}, {x.slots, "slots"}}))
      return st;
    if (desc->num_q_heads > 0)
      if (sgdkv_status st = check_ptrs({{x.q, "q"}, {x.q_out, "q_out"}})) return st;
    if (desc->rot_dim > 0)
      if (sgdkv_status st = check_ptrs({{x.inv_freq, "inv_freq"}})) return st;
  }
  if (x.q_weight)
    if (sgdkv_status st = check_ptrs({{x.q_weight, "q_weight"}})) return st;
  if (x.k_weight)
    if (sgdkv_status st = check_ptrs({{x.k_weight, "k_weight"}})) return st;
  if (desc->num_q_heads > 0 && x.q_out && x.q_out == x.q && desc->q_stride != (int64_t)desc->num_q_heads * d)
    return fail(SGDKV_ERR_INVALID_ARG, "q_out may be q only where q is dense");
  a = NormRopeArgs{};
  a.T = (int)desc->num_tokens;
  a.Hq = desc->num_q_heads;
  a.Hkv = desc->num_kv_heads;
  a.D = d;
  a.dtype = dtype;
  a.rot = desc->rot_dim;
  a.interleaved = desc->interleaved;
  a.eps = desc->eps;
  a.q_stride = desc->q_stride * eb;
  a.k_stride = desc->k_stride * eb;
  a.v_stride = desc->v_stride * eb;
  a.q = x.q;
  a.k = x.k;
  a.v = x.v;
  a.positions = x.positions;
  a.slots = x.slots;
  a.inv_freq = x.inv_freq;
  a.q_weight = x.q_weight;
  a.k_weight = x.k_weight;
  a.q_out = x.q_out;
  return SGDKV_OK;
}

}  // namespace sgdkv
