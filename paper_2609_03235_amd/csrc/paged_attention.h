// Attention of new tokens over a paged per-head KV cache (gfx950): shared by the instances for few query
// rows (paged_few.hip, paged_few_fp8.hip for pools in 8 bits) and for many (paged_many.hip).
//
// Segment (b, h) holds the rows of KV head h of sequence b, the new tokens' own rows last. Token i of the n
// new ones sees rows 0 .. rows - n + i; the G query heads of the group see the same rows, so the n * G query
// rows are cut into tiles of whole tokens (`tokens` of them, the G heads of a token together) and every key
// row is read once per tile. S^T = K Q^T is computed rather than S: a lane then holds one query row's logits
// (keys down the accumulator registers), so the softmax statistics need no cross-lane work until the end, and
// the probabilities are already the B operand of O^T = V^T P^T, with the keys of a step in the order the
// accumulator left them. V^T takes the same key order and comes out of LDS through the transposing read.
//
// Work is shared by cost, not by tile: the tiles in (segment, tile) order form one line whose length is the
// key rows each has to see, cut into equal pieces, one per workgroup. A piece covers whole tiles and at most
// two part ones, whose partial results (m, s, o) go to the workspace; the merge kernel joins them in order.
// The lengths are read on the device, so a captured call replays with whatever they have become.
#pragma once

#include "device_common.h"
#include "fp8_rows.h"
#include "mfma_frag.h"
#include "paged_internal.h"
#include "sgdkv_internal.h"

namespace sgdkv {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr int kAttnBlock = 256;
constexpr int kAttnWaves = kAttnBlock / 64;
// Most query rows per KV head of the instances for few: what leaves room for two workgroups in a compute unit's
// registers and LDS.
constexpr int kFewRowsBf16 = 48, kFewRowsF32 = 32;

// A segment as a workgroup sees it. Lengths that do not fit the buffers are cut to them.
struct PagedSeg {
  int t0;      // first token
  int n;       // tokens computed
  int rows;    // rows of the segment
  int base;    // token i sees base + i + 1 rows (clamped to [0, rows])
  int tiles;   // query tiles
};

__device__ __forceinline__ PagedSeg paged_seg(const PagedAttnArgs& a, int seg) {
  PagedSeg s;
  const int b = (int)((uint32_t)seg * a.inv_hkv >> 32);
  int c0 = a.cu[b], c1 = a.cu[b + 1];
  c0 = min(max(c0, 0), a.T);
  c1 = min(max(c1, c0), a.T);
  const int64_t most = (int64_t)a.max_pages << a.page_shift;
  const int r = max(a.rows[seg], 0);
  s.rows = r > most ? (int)most : r;
  s.t0 = c0;
  s.n = min(c1 - c0, a.max_new);
  s.base = s.rows - (c1 - c0);
  s.tiles = (int)(((uint32_t)s.n + a.tokens - 1) / (uint32_t)a.tokens);
  return s;
}

// Rows that token i sees, and those that query tile t sees (its last token's).
__device__ __forceinline__ int seen_by(const PagedAttnArgs& a, const PagedSeg& s, int i) {
  return a.causal ? max(s.base + i + 1, 0) : s.rows;
}
__device__ __forceinline__ int tile_rows(const PagedAttnArgs& a, const PagedSeg& s, int t) {
  return seen_by(a, s, min((t + 1) * a.tokens, s.n) - 1);
}
// A tile takes as many places of the line as it sees rows, at least one (its results are written all the same),
// and 2^min_shift more for what every tile takes however short it is: 16 tiles of a few rows each, all one worker's
// by their rows alone, took 118 us so and 9 with it. The rows of the first m tiles:
__device__ __forceinline__ int64_t cost_of(const PagedAttnArgs& a, const PagedSeg& s, int m) {
  if (!a.causal) return (int64_t)m * max(s.rows, 1);
  if (m <= 0) return 0;
  const int64_t full = m < s.tiles ? m : s.tiles - 1;  // tiles whose last token is number (t + 1) * tokens
  int64_t blind = s.base < 0 ? (int)((uint32_t)-s.base / (uint32_t)a.tokens) : 0;  // those that see nothing
  if (blind > full) blind = full;
  int64_t sum = blind + (full - blind) * s.base + (int64_t)a.tokens * (full * (full + 1) - blind * (blind + 1)) / 2;
  if (m == s.tiles) sum += max(s.base + s.n, 1);
  return sum;
}

// The places of the first m tiles.
__device__ __forceinline__ int64_t places_of(const PagedAttnArgs& a, const PagedSeg& s, int m) {
  return cost_of(a, s, m) + ((int64_t)m << a.min_shift);
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// A place on the line: a tile, its segment, and where it starts.
struct LineTile {
  int seg, tile;
  int64_t start;
  PagedSeg g;
};

struct LineScratch {
  int64_t wave_sum[kAttnWaves];
  int64_t start;
  int seg;
  PagedSeg g;
};

__device__ __forceinline__ PagedSeg uniform(const PagedSeg& g) {
  return PagedSeg{uniform(g.t0), uniform(g.n), uniform(g.rows), uniform(g.base), uniform(g.tiles)};
}

// Exclusive prefix sum over the workgroup; total = the sum. Two barriers where it is used twice in a row.
template <typename I>
__device__ __forceinline__ I block_prefix(I mine, int64_t* wave_sum, I& total) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  I x = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const I y = sizeof(I) == 8 ? (I)__shfl_up((long long)x, o, 64) : (I)__shfl_up((int)x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) wave_sum[wid] = x;
  __syncthreads();
  I before = x - mine;
  total = 0;
#pragma unroll
  for (int i = 0; i < kAttnWaves; ++i) {
    const I y = (I)wave_sum[i];
    if (i < wid) before += y;
    total += y;
  }
  return before;
}

// The whole workgroup adds the segments up and finds worker w's piece of the line, [share * w, end): false if
// there is none. share receives the pieces' length: an equal part, at least 2^min_shift.
// PAD (segments of one tile): where all workers' least pieces cover the segments rounded up to whole pieces,
// the line is that, and no worker has parts of two tiles. Short calls are bound by latency: one token over four
// segments of 8K rows took 14.9 us with, 10.4 without the three workers that had two.
// ONE: every call's segments have one tile at most.
template <bool PAD, bool ONE = true>
__device__ __forceinline__ bool find_piece(const PagedAttnArgs& a, LineScratch& sc, int w, int64_t& share,
                                           int64_t& end, bool& padded, LineTile& at) {
  const int tid = threadIdx.x;
  const int per = (a.S + kAttnBlock - 1) / kAttnBlock;
  const int s0 = min(tid * per, a.S), s1 = min(s0 + per, a.S);
  const int64_t least = (int64_t)1 << a.min_shift;
  int64_t mine = 0;
  int pieces = 0;  // of the least length, cut off where there are too many for all workers
  PagedSeg g{};
  auto pieces_of = [&](int64_t c) { return (int)min((c + least - 1) >> a.min_shift, (int64_t)kPagedWorkers + 1); };
  for (int s = s0; s < s1; ++s) {
    g = paged_seg(a, s);
    mine += places_of(a, g, g.tiles);
    if (PAD) pieces += pieces_of(cost_of(a, g, g.tiles));
  }
  padded = false;
  int64_t run = 0, all = 0;
  if constexpr (PAD) {
    int n;
    run = (int64_t)block_prefix(pieces, sc.wave_sum, n) << a.min_shift;
    padded = uniform(n) <= kPagedWorkers;
    if constexpr (!ONE) padded &= a.max_tiles == 1;
    all = (int64_t)uniform(n) << a.min_shift;
    if (!padded) __syncthreads();
  }
  if (!padded) {
    run = block_prefix(mine, sc.wave_sum, all);
    all = uniform(all);
  }
  share = padded ? least : max((all + kPagedWorkers - 1) / kPagedWorkers, least);
  const int64_t want = share * w;
  if (want >= all) return false;
  end = min(want + share, all);
  if (want >= run && want < run + (padded ? (int64_t)pieces << a.min_shift : mine)) {
    for (int s = s0; s < s1; ++s) {
      if (per > 1) g = paged_seg(a, s);
      const int64_t c =
          padded ? (int64_t)pieces_of(cost_of(a, g, g.tiles)) << a.min_shift : places_of(a, g, g.tiles);
      if (want < run + c) {
        sc.seg = s;
        sc.start = run;
        sc.g = g;
        break;
      }
      run += c;
    }
  }
  __syncthreads();
  at.seg = uniform(sc.seg);
  at.g = uniform(sc.g);
  const int64_t seg_start = uniform(sc.start);
  // The last tile that starts at or before `want`: every lane looks at one place in 64.
  const int lane = tid & 63;
  int lo = 0;
  for (int n = at.g.tiles; n > 1;) {
    const int step = (n + 63) >> 6, m = lo + lane * step;
    const int upto = __popcll(__ballot(lane * step < n && seg_start + places_of(a, at.g, m) <= want));
    lo += (upto - 1) * step;
    n = min(step, n - (upto - 1) * step);
  }
  at.tile = uniform(lo);
  at.start = uniform(seg_start + places_of(a, at.g, lo));
  return true;
}

// What a worker leaves for the merge (see PagedAttnArgs::shared) about a tile of nkt key tiles.
__device__ __forceinline__ void leave_shared(const PagedAttnArgs& a, int w, int64_t share, const LineTile& at,
                                             int nkt, bool unshared) {
  const int64_t own = share * w;
  if (threadIdx.x != 0 || at.start < own) return;  // begun by a worker before
  const int64_t past = at.start - own + (int64_t)(nkt - 1) * a.key_tile - share;  // the last key's place, from w + 1's
  const int last = unshared || past < 0 ? -1 : w + 1 + (past < share ? 0 : (int)((uint32_t)past / (uint32_t)share));
  if (a.by_tile) a.shared[at.seg * a.max_tiles + at.tile] = make_int4(at.seg, at.tile, 2 * w + (at.start > own), last);
  else if (last >= 0) a.shared[w] = make_int4(at.seg, at.tile, 2 * w + (at.start > own), last);
}

// Neighbouring workers on one XCD (workgroups go to the eight XCDs in turn): they read the same segment's
// rows, from one L2.
__device__ __forceinline__ int worker_of() {
  static_assert(kPagedWorkers % 8 == 0, "workers per XCD");
  return (blockIdx.x & 7) * (kPagedWorkers / 8) + (blockIdx.x >> 3);
}

// Buffer over the 16-row group of a segment that starts at row r0, `valid` rows of it (0 or fewer: none).
// A table entry outside the pool gives an empty buffer, whose reads are zeros.
__device__ __forceinline__ int group_page(const PagedAttnArgs& a, const int32_t* table, int r0, int limit) {
  return r0 < limit ? table[r0 >> a.page_shift] : -1;
}
__device__ __forceinline__ rsrc_t rows_rsrc(const PagedAttnArgs& a, const void* pool, int page, int r0, int valid,
                                            int rows, int row_bytes) {
  const bool ok = page >= 0 && page < a.num_pages && valid > 0;
  const int64_t row = ok ? ((int64_t)page << a.page_shift) + (r0 & ((1 << a.page_shift) - 1)) : 0;
  const int n = ok ? min(valid, rows) : 0;
  return make_rsrc(static_cast<const char*>(pool) + row * row_bytes, (uint64_t)(n * row_bytes));
}
__device__ __forceinline__ rsrc_t group_rsrc(const PagedAttnArgs& a, const void* pool, int page, int r0, int valid,
                                             int row_bytes) {
  return rows_rsrc(a, pool, page, r0, valid, 16, row_bytes);
}

// The same buffer as four scalar words.
__device__ __forceinline__ u32x4 group_words(const PagedAttnArgs& a, const void* pool, int page, int r0, int valid,
                                             int rows, int row_bytes) {
  const bool ok = page >= 0 && page < a.num_pages && valid > 0;
  const int64_t row = ok ? ((int64_t)page << a.page_shift) + (r0 & ((1 << a.page_shift) - 1)) : 0;
  const uint64_t p = reinterpret_cast<uint64_t>(pool) + row * row_bytes;
  return u32x4{(uint32_t)uniform((int)p), (uint32_t)uniform((int)(p >> 32)),
               (uint32_t)uniform(ok ? min(valid, rows) * row_bytes : 0), (uint32_t)kRsrcWord3};
}

// The codes of the same rows (8-bit pools), one byte each. A code may mean NaN where no row is, and NaN times the zeros
// read there is NaN: none past the last row is read (zero, a power that zeros do not mind).
__device__ __forceinline__ rsrc_t code_rsrc(const PagedAttnArgs& a, const uint8_t* codes, int page, int r0, int valid,
                                            int rows) {
  const bool ok = page >= 0 && page < a.num_pages && valid > 0;
  const int64_t row = ok ? ((int64_t)page << a.page_shift) + (r0 & ((1 << a.page_shift) - 1)) : 0;
  return make_rsrc(codes + row, ok ? min(valid, rows) : 0);
}

// 64 x 16 bytes from a buffer into LDS at lds + 16 * lane; out-of-range lanes write zeros. The compiler does not
// see that these loads are under way: wait_loads() before the data is read (and a barrier, if by other waves).
// There is no destination register that could be reused too early. m0 is a reserved register, which cannot be named as
// clobbered; nothing else in these kernels uses it, and each load sets it for itself.
__device__ __forceinline__ uint32_t lds_address(const char* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
__device__ __forceinline__ void load_to_lds(u32x4 rsrc, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(rsrc)
               : "memory");
}
__device__ __forceinline__ void load_to_lds_nt(u32x4 rsrc, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(lds), "v"(off),
               "s"(rsrc)
               : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
  f32x2 v = {x, y};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
// x and y as sums of N bf16 terms each, of which three hold all 24 bits: word e of each term.
template <int N>
__device__ __forceinline__ void split_bf16(float x, float y, u32x4 (&to)[N], int e) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const uint32_t w = pack_bf16(x, y);
    to[k][e] = w;
    x -= bf16_lo(w);
    y -= bf16_hi(w);
  }
}

// Four keys (rows) by the wave's 16-lane groups' columns, transposed: lane i of a group receives column i of
// the four rows whose pieces the group's lanes point at (lane 4r + c at row r, columns 4c .. 4c + 3).
__device__ __forceinline__ u32x2 lds_transposed(const char* p) {
  typedef __attribute__((address_space(3))) bf16x4* lds_ptr;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_ptr)(p)));
}
// Eight keys of bytes likewise: lane i receives column i of the eight rows that the group's lanes point at (lane
// 2r + c at row r, columns 8c .. 8c + 7).
__device__ __forceinline__ u32x2 lds_transposed8(const char* p) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) i32x2* lds_ptr;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_ptr)(p)));
}

// Masked keys have probability zero, and zero times a value that is not finite is NaN. Keys past every row's last
// one are loaded as zeros. In a tile with keys that some rows see and others do not, clean_values sets values that
// are not finite to zero in LDS, and notes the first such key of each column: as a row sees the keys up to some
// key, it sees such a value exactly if it sees the first, and its output is then NaN. (The same in registers, where
// the products are made, cost the tiles without masks up to a third of their time.)
// Rows [r0, r1) of those from key0 on, the ones that not all see, whose 16-byte pieces lie where `swizzle` says; by
// every wave that uses them.
template <int EB, int RB, typename F>
__device__ __forceinline__ void clean_values(char* vals, int key0, int r0, int r1, int* first_odd, F swizzle) {
  constexpr int VPR = RB / 16;
  constexpr uint32_t kOdd = 0x7F800000u;  // the exponent of infinities and NaN; bf16 in each half
#pragma unroll 2
  for (int i = r0 * VPR + (threadIdx.x & 63); i < r1 * VPR; i += 64) {
    const int r = i / VPR, col = ((i % VPR) ^ swizzle(r)) * (16 / EB);
    u32x4* at = reinterpret_cast<u32x4*>(vals + i * 16);
    u32x4 v = *at;
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, EB == 2 ? max(v[e] & kOdd, v[e] << 16 & kOdd) : v[e] & kOdd);
    if (top != kOdd) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if ((v[e] & kOdd) == kOdd) {
        atomicMin(&first_odd[col + (EB == 2 ? 2 * e + 1 : e)], key0 + r);
        v[e] &= EB == 2 ? 0xFFFFu : 0u;
      }
      if (EB == 2 && (v[e] << 16 & kOdd) == kOdd) {
        atomicMin(&first_odd[col + 2 * e], key0 + r);
        v[e] &= 0xFFFF0000u;
      }
    }
    *at = v;
  }
}
// The same for rows of e4m3 numbers, whose only values that are not finite are the bytes 0x7F and 0xFF.
template <int RB, typename F>
__device__ __forceinline__ void clean_values8(char* vals, int key0, int r0, int r1, int* first_odd, F swizzle) {
  constexpr int VPR = RB / 16;
#pragma unroll 2
  for (int i = r0 * VPR + (threadIdx.x & 63); i < r1 * VPR; i += 64) {
    const int r = i / VPR, col = ((i % VPR) ^ swizzle(r)) * 16;
    u32x4* at = reinterpret_cast<u32x4*>(vals + i * 16);
    u32x4 v = *at;
    uint32_t any = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) any |= (v[e] & 0x7F7F7F7Fu) + 0x01010101u;
    if (!(any & 0x80808080u)) continue;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if ((v[e / 4] >> (8 * (e % 4)) & 0x7F) != 0x7F) continue;
      atomicMin(&first_odd[col + e], key0 + r);
      v[e / 4] &= ~(0xFFu << (8 * (e % 4)));
    }
    *at = v;
  }
}
// Columns col .. col + 3 of a row that sees `seen` keys.
__device__ __forceinline__ f32x4 lose_odd(f32x4 o, const int* first_odd, int col, int seen) {
  const int4 odd = *reinterpret_cast<const int4*>(first_odd + col);
  return f32x4{odd.x < seen ? NAN : o[0], odd.y < seen ? NAN : o[1], odd.z < seen ? NAN : o[2],
               odd.w < seen ? NAN : o[3]};
}

// Four consecutive columns of an output row.
__device__ __forceinline__ void store_out4(const PagedAttnArgs& a, int64_t row, int D, int col, f32x4 v) {
  if (a.out_dtype) {
    u32x2 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    *reinterpret_cast<u32x2*>(static_cast<char*>(a.out) + (row * D + col) * 2) = w;
  } else {
    *reinterpret_cast<f32x4*>(static_cast<char*>(a.out) + (row * D + col) * 4) = v;
  }
}

constexpr float kLn2 = 0.693147180559945309f;
__device__ __forceinline__ float lse_of(float m, float s) {
  return s > 0.f ? (m + fast_log2(s)) * kLn2 : (s == 0.f ? -INFINITY : s);
}

hipError_t launch_paged_few(const PagedAttnArgs& a, hipStream_t stream);
hipError_t launch_paged_many(const PagedAttnArgs& a, hipStream_t stream);
hipError_t launch_paged_few_fp8(const PagedAttnArgs& a, hipStream_t stream);
hipError_t launch_paged_many_fp8(const PagedAttnArgs& a, hipStream_t stream);
// Joins the parts of shared tiles after an attention kernel.
hipError_t launch_paged_merge(const PagedAttnArgs& a, hipStream_t stream);

}  // namespace sgdkv
