// Internal interface between the C-ABI layer of the paged cache (paged_host.cpp) and its HIP
// kernels (paged_cache.hip, paged_few.hip, paged_many.hip). Not installed; not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sgdkv {

constexpr int kPageBlock = 256;       // threads per workgroup of the page and row kernels
constexpr int kMaxPageSegs = 4096;    // segments of one page update (their lengths and prefix sums fill 64 KB of LDS)
constexpr int kMinPage = 16;          // rows per page: every 16-row group of a segment lies in one page
constexpr int kMaxPage = 1024;
// Workgroups that share an attention call: two per compute unit of the MI355X. A constant, so that results do not
// depend on the device.
constexpr int kPagedWorkers = 512;
constexpr int kMaxPagedGroup = 16;    // query heads per KV head

// ------------------------------------------------------------- page update
struct PageArgs {
  int B, Hkv, S;           // S = B * Hkv segments
  int page_shift, max_pages;
  int by_segment;          // add and slots per segment; otherwise per sequence and token
  int64_t num_free;        // entries of free_pages
  int64_t num_slots;       // rows of slots
  const int32_t* rows;     // [S]
  const int32_t* add;      // [S] or [B]
  int32_t* tables;         // [S][max_pages]
  int32_t* free_pages;     // [num_free]
  const int32_t* head;     // [1]
  int32_t* rows_out;       // [S]
  int32_t* head_out;       // [1]
  int32_t* cu_out;         // [S + 1] or [B + 1]
  int32_t* slots;          // [num_slots] or [num_slots][Hkv]
  int32_t* status;         // [1]
};
hipError_t launch_page_update(const PageArgs& a, int cus, hipStream_t stream);

// ------------------------------------------------------------- rows into pages
struct PagedStoreArgs {
  int row_shift;        // log2 of a row's 16-byte pieces
  int64_t n;            // rows
  int64_t total_slots;  // rows of the pool
  const void* k;
  const void* v;
  const int32_t* slots;  // [n]
  void* k_pages;
  void* v_pages;
};
hipError_t launch_paged_store(const PagedStoreArgs& a, hipStream_t stream);

struct NormRopeArgs {
  int T, Hq, Hkv, D, dtype;
  int rot;          // rotated elements per head (0: none)
  int interleaved;  // pairs (2i, 2i + 1) instead of (i, i + rot / 2)
  float eps;
  int64_t q_stride, k_stride, v_stride;  // bytes between tokens
  int64_t total_slots;
  const void* q;
  const void* k;
  const void* v;
  const int32_t* positions;  // [T]
  const int32_t* slots;      // [T][Hkv]
  const float* inv_freq;     // [rot / 2]
  const void* q_weight;      // [D] or NULL
  const void* k_weight;
  void* q_out;  // [T][Hq][D]
  void* k_pages;
  void* v_pages;
  int parts;    // waves that share a token's heads (set at the launch)
};
hipError_t launch_norm_rope(const NormRopeArgs& a, hipStream_t stream);

// ------------------------------------------------------------- attention
struct PagedAttnArgs {
  int B, Hq, Hkv, G, D, S, T;
  int dtype, out_dtype, causal;
  int page_shift, max_pages, max_new;
  int64_t num_pages;
  float c2;          // scale * log2(e)
  uint64_t inv_hkv;  // ceil(2^32 / Hkv): seg * inv_hkv >> 32 is seg / Hkv for seg below 65536
  int tile_rows;     // query rows per tile (M)
  int key_tile;      // key rows per step of a workgroup (KT)
  int tokens;        // new tokens per query tile
  int max_tiles;     // query tiles of a segment with max_new tokens
  int by_tile;
  int min_shift;     // log2 of the key rows a worker takes at least (whole key tiles)
  const void* q;
  const void* k_pages;
  const void* v_pages;
  const int32_t* tables;
  const int32_t* rows;
  const int32_t* cu;
  void* out;
  float* lse;        // optional
  // workspace
  // Query tiles that a worker began: segment, tile, 2 * that worker (+ 1 if the tile starts after the worker's
  // share does), and the last worker that has a part of it (-1: no other). [S * max_tiles], an entry per tile, where
  // that is at most kPagedWorkers (by_tile); otherwise [kPagedWorkers], the tile each worker left to the next ones.
  int4* shared;
  float* part;       // [2 * kPagedWorkers][M][D]: o of a query tile that several workers share
  float* part_ms;    // [2 * kPagedWorkers][M][2]
};
// The kernel instance for a shape: query rows per tile and key rows per step.
struct PagedAttnShape {
  int rows;      // M
  int key_tile;  // KT
};
PagedAttnShape paged_attn_shape(int dtype, int G, int max_new);
hipError_t launch_paged_attention(const PagedAttnArgs& a, hipStream_t stream);

}  // namespace sgdkv
