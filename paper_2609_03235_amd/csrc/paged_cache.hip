// The paged per-head KV cache (gfx950): pages taken and given back, slots, and rows written to them.
//
// After compression every KV head of every sequence (a segment) holds its own number of rows, so the
// cache is paged per segment: a table row per segment lists the pages (of P rows each) that hold its
// rows in order, and row p of segment s lies in slot tables[s][p / P] * P + p % P of the pool.
//
//   page_update      rows gained or lost per segment -> pages from or to the free stack, new table
//                    entries, the slot of every new row
//   paged_store      rows copied to their slots
//   norm_rope_store  new tokens: norm and rotation per head, q to a dense tensor, k and v to their slots
//
// All three are bound by latency or by HBM. The pools may pass 4 GiB, so their rows are addressed with
// 64-bit pointers; every slot is compared with the pool's size first.
#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "paged_internal.h"
#include "sgdkv_internal.h"

namespace sgdkv {

namespace {

constexpr int kWavesPerBlock = kPageBlock / 64;

// ------------------------------------------------------------------ page update
// Pages of a segment of `rows` rows, cut to the table's width (more is reported as a failure).
__device__ __forceinline__ int pages_of(const PageArgs& a, int64_t rows) {
  const int64_t p = (rows + ((int64_t)1 << a.page_shift) - 1) >> a.page_shift;
  return p > a.max_pages ? a.max_pages : (int)p;
}

// Exclusive prefix sums over the workgroup's threads of new rows, pages taken and pages given back.
struct Gains {
  int64_t fresh;
  int taken, given;
};
__device__ __forceinline__ Gains block_prefix(Gains v, Gains* tmp, Gains& total) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  Gains x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t f = __shfl_up((long long)x.fresh, o, 64);
    const int t = __shfl_up(x.taken, o, 64), g = __shfl_up(x.given, o, 64);
    if (lane >= o) {
      x.fresh += f;
      x.taken += t;
      x.given += g;
    }
  }
  if (lane == 63) tmp[wid] = x;
  __syncthreads();
  Gains before{x.fresh - v.fresh, x.taken - v.taken, x.given - v.given};
  total = Gains{0, 0, 0};
#pragma unroll
  for (int w = 0; w < kPageBlock / 64; ++w) {
    const Gains y = tmp[w];
    if (w < wid) before = Gains{before.fresh + y.fresh, before.taken + y.taken, before.given + y.given};
    total = Gains{total.fresh + y.fresh, total.taken + y.taken, total.given + y.given};
  }
  return before;
}

// The last entry of the ascending prefix p[0 .. n) that is <= i, where empty pieces share a value.
__device__ __forceinline__ int piece_of(const int32_t* p, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Every workgroup reads the segments' lengths and computes the same prefix sums into LDS (they are few
// beside the slots), then does its share of the table entries and slots: one launch, no scan before it. Bound
// by latency: about four dependent memory reads and the scan; one more token for 512 segments takes 6 us, the 2.1 M
// slots of 64 segments 13 (the first with one workgroup and the lengths read again at every use 24, with the first
// workgroup's threads at four slots each 10).
// Nothing that one workgroup writes is read by another: table entries past a segment's old pages are written
// and those within them read; the stack is written below its head (the pages given back, looked up in their
// tables by those who take them in the same call) and read from its head on. rows_out and head_out may be the
// inputs themselves: where several workgroups read those, a second launch of one workgroup writes them (FINAL).
template <bool FINAL>
__global__ __launch_bounds__(kPageBlock) void page_update_kernel(PageArgs a, int write_rows) {
  extern __shared__ int32_t lds[];
  const int pieces = a.by_segment ? a.S : a.B;
  int32_t* taken = lds;              // [S + 1] pages taken before a segment
  int32_t* given = taken + a.S + 1;  // [S + 1] pages given back before a segment
  int32_t* rows = given + a.S + 1;   // [S]
  int32_t* cu = rows + a.S;          // [pieces + 1] new rows before a segment (a sequence)
  __shared__ Gains tmp[kPageBlock / 64];
  const int tid = threadIdx.x;
  const int64_t head = a.head[0];

  // A thread takes consecutive segments (and, by token, the sequences that begin among them).
  const int per = (a.S + kPageBlock - 1) / kPageBlock;
  const int s0 = min(tid * per, a.S), s1 = min(s0 + per, a.S);
  const int64_t most = (int64_t)a.max_pages << a.page_shift;
  Gains mine{0, 0, 0};
  int bad = 0;
  for (int s = s0; s < s1; ++s) {
    const int b = a.by_segment ? s : s / a.Hkv;
    const int64_t before = a.rows[s], add = a.add[b], after = max(before + add, (int64_t)0);
    bad |= before < 0 || before > most || after > most;
    rows[s] = (int)before;
    const int d = pages_of(a, after) - pages_of(a, max(before, (int64_t)0));
    mine.taken += max(d, 0);
    mine.given += max(-d, 0);
    if (a.by_segment || s == b * a.Hkv) mine.fresh += max(add, (int64_t)0);
  }
  const int any_bad = __syncthreads_or(bad);
  Gains all;
  Gains run = block_prefix(mine, tmp, all);
  const int64_t base = head - all.given;
  const int status = any_bad                                      ? 2
                     : head < 0 || head > a.num_free || base < 0  ? 3
                     : all.fresh > a.num_slots                    ? 4
                     : base + all.taken > a.num_free              ? 1
                                                                  : 0;
  for (int s = s0; s < s1; ++s) {
    const int b = a.by_segment ? s : s / a.Hkv;
    const int64_t before = rows[s], add = a.add[b], after = max(before + add, (int64_t)0);
    const int d = pages_of(a, after) - pages_of(a, max(before, (int64_t)0));
    taken[s] = run.taken;
    given[s] = run.given;
    run.taken += max(d, 0);
    run.given += max(-d, 0);
    if (a.by_segment || s == b * a.Hkv) {
      cu[b] = (int)run.fresh;
      run.fresh += max(add, (int64_t)0);
    }
    if (write_rows && blockIdx.x == 0) a.rows_out[s] = (int)(status ? before : after);
  }
  if (tid == 0) {
    taken[a.S] = all.taken;
    given[a.S] = all.given;
    cu[pieces] = (int)all.fresh;
    if (write_rows && blockIdx.x == 0) a.head_out[0] = (int)(status ? head : base + all.taken);
  }
  if (FINAL) return;
  __syncthreads();

  const int64_t stride = (int64_t)gridDim.x * kPageBlock, first = (int64_t)blockIdx.x * kPageBlock + tid;
  if (blockIdx.x == 0) {
    for (int i = tid; i <= pieces; i += kPageBlock) a.cu_out[i] = status ? 0 : cu[i];
    if (tid == 0) a.status[0] = status;
  }
  // where the page at stack index i is found: given back in this call below the old head, else on the stack
  auto page_at = [&](int64_t i) -> const int32_t* {
    if (i >= head) return a.free_pages + i;
    const int at = (int)(i - base), g = piece_of(given, a.S, at);
    const int left = pages_of(a, rows[g]) - (given[g + 1] - given[g]);  // its pages afterwards
    return a.tables + (int64_t)g * a.max_pages + left + (at - given[g]);
  };
  if (status == 0) {
    // from the last workgroup on: the first ones have the slots
    const int64_t from = (int64_t)(gridDim.x - 1 - blockIdx.x) * kPageBlock + tid;
    for (int64_t i = from; i < all.taken; i += stride) {
      const int s = piece_of(taken, a.S, (int)i);
      a.tables[(int64_t)s * a.max_pages + pages_of(a, rows[s]) + ((int)i - taken[s])] = *page_at(base + i);
    }
    for (int64_t i = from; i < all.given; i += stride) a.free_pages[base + i] = *page_at(base + i);
  }
  // slots: a thread takes one, or four consecutive ones where there are more than threads
  const uint32_t per_row = a.by_segment ? 1 : a.Hkv;
  const int64_t n = a.num_slots * per_row;
  const int in_page = (1 << a.page_shift) - 1;
  auto slots = [&](auto count, auto by_segment) {
    constexpr int N = decltype(count)::value;
    constexpr bool BY_SEGMENT = decltype(by_segment)::value;
    for (int64_t at = first * N; at < n; at += stride * N) {
      if (BY_SEGMENT && N == 4 && status == 0 && at + 4 <= all.fresh) {
        const int s = piece_of(cu, pieces, (int)at);
        if (at + 4 <= cu[s + 1]) {  // mostly: four rows of one segment, in one page or two
          const int p0 = rows[s] + ((int)at - cu[s]), had = pages_of(a, rows[s]);
          const int j0 = p0 >> a.page_shift, j3 = (p0 + 3) >> a.page_shift;
          const int32_t* table = a.tables + (int64_t)s * a.max_pages;
          const int64_t base_s = base + taken[s] - had;
          const int32_t* first_page = j0 < had ? table + j0 : page_at(base_s + j0);
          const int32_t* last_page = j3 == j0 ? first_page : j3 < had ? table + j3 : page_at(base_s + j3);
          const int64_t pages[2] = {*first_page, *last_page};
          int slot[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int p = p0 + e;
            const int64_t x = ((p >> a.page_shift == j0 ? pages[0] : pages[1]) << a.page_shift) + (p & in_page);
            slot[e] = x < 0 || x > 0x7FFFFFFF ? -1 : (int)x;
          }
          *reinterpret_cast<int4*>(a.slots + at) = make_int4(slot[0], slot[1], slot[2], slot[3]);
          continue;
        }
      }
      // all places are worked out before the first page is read
      const int32_t* page[N];
      int pos[N];
      uint32_t item = (uint32_t)at / per_row, h = (uint32_t)at - item * per_row;
      int piece = -1, seg = -1, entry = -1;  // neighbours mostly share these
#pragma unroll
      for (int e = 0; e < N; ++e) {
        page[e] = nullptr;
        pos[e] = 0;
        if (status == 0 && item < (uint32_t)all.fresh) {
          if (piece < 0 || (int)item >= cu[piece + 1]) piece = piece_of(cu, pieces, (int)item);
          const int s = BY_SEGMENT ? piece : piece * a.Hkv + (int)h;
          pos[e] = rows[s] + ((int)item - cu[piece]);
          const int j = pos[e] >> a.page_shift;
          if (e > 0 && s == seg && j == entry) {
            page[e] = page[e - 1];
          } else {
            const int had = pages_of(a, rows[s]);
            page[e] = j < had ? a.tables + (int64_t)s * a.max_pages + j : page_at(base + taken[s] + (j - had));
            seg = s;
            entry = j;
          }
        }
        if (++h == per_row) {
          h = 0;
          ++item;
        }
      }
      int64_t out[N];
#pragma unroll
      for (int e = 0; e < N; ++e) out[e] = page[e] ? *page[e] : -1;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int64_t slot = (out[e] << a.page_shift) + (pos[e] & in_page);
        out[e] = slot < 0 || slot > 0x7FFFFFFF ? -1 : slot;
      }
      if (N == 4 && at + 4 <= n) {
        *reinterpret_cast<int4*>(a.slots + at) =
            make_int4((int)out[0], (int)out[N / 4], (int)out[N / 2], (int)out[N - 1]);
      } else {
        for (int e = 0; e < N && at + e < n; ++e) a.slots[at + e] = (int32_t)out[e];
      }
    }
  };
  using One = std::integral_constant<int, 1>;
  using Four = std::integral_constant<int, 4>;
  if (a.by_segment) n <= stride ? slots(One{}, std::true_type{}) : slots(Four{}, std::true_type{});
  else n <= stride ? slots(One{}, std::false_type{}) : slots(Four{}, std::false_type{});
}

// ------------------------------------------------------------------ rows to their slots
// A workgroup takes kStoreVecs * 256 consecutive 16-byte pieces; a thread has all its loads under way before it
// stores. The rows are streamed once, in and out: non-temporal. Bound by HBM: 1 M rows of 128 bf16 values take 206 us,
// 5.3 TB/s in and out (one piece per thread, without the hint, 208).
constexpr int kStoreVecs = 4;
__global__ __launch_bounds__(kPageBlock) void paged_store_kernel(PagedStoreArgs a) {
  const int64_t total = a.n << a.row_shift;
  const int64_t first = (int64_t)blockIdx.x * (kStoreVecs * kPageBlock) + threadIdx.x;
  int64_t to[kStoreVecs];
  u32x4 k[kStoreVecs], v[kStoreVecs];
#pragma unroll
  for (int u = 0; u < kStoreVecs; ++u) {
    const int64_t i = first + u * kPageBlock;
    to[u] = -1;
    if (i >= total) continue;
    const int64_t slot = a.slots[i >> a.row_shift];
    if (slot >= 0 && slot < a.total_slots) to[u] = (slot << a.row_shift) + (i & ((1 << a.row_shift) - 1));
    k[u] = __builtin_nontemporal_load(static_cast<const u32x4*>(a.k) + i);
    v[u] = __builtin_nontemporal_load(static_cast<const u32x4*>(a.v) + i);
  }
#pragma unroll
  for (int u = 0; u < kStoreVecs; ++u) {
    if (to[u] < 0) continue;
    __builtin_nontemporal_store(k[u], static_cast<u32x4*>(a.k_pages) + to[u]);
    __builtin_nontemporal_store(v[u], static_cast<u32x4*>(a.v_pages) + to[u]);
  }
}

// ------------------------------------------------------------------ norm, rotation, store
// sin and cos of position * freq. In turns the angle is position * freq / (2 pi): both products are carried with
// their rounding errors, and the nearest quarter turn is taken off in 64 bits, which leaves an angle x in
// [-pi/4, pi/4] for the Taylor sums (the first terms left out are below 2e-9 and 2e-10 of a radian). So the angle of a
// position of 2^31 is as good as that of a small one. The sums are in 64 bits too, and what they give is rounded once:
// an x rounded to 32 bits alone is off by up to 2^-25, 2^-27.7 turns. (A lane does this once per token, for all heads.)
__device__ __forceinline__ void sincos_at(double position, double freq, float& sin_t, float& cos_t) {
  constexpr double kHi = 0.15915494309189535, kLo = -9.839338337591243e-18;  // 1 / (2 pi)
  const double a0 = position * freq, a1 = fma(position, freq, -a0);
  const double t = a0 * kHi, t1 = fma(a0, kHi, -t) + fma(a0, kLo, a1 * kHi);
  const double n = rint(4.0 * t);
  const double x = (fma(-0.25, n, t) + t1) * 6.283185307179586476925;
  const double z = x * x;
  double s = fma(z, 1.0 / 362880, -1.0 / 5040);
  s = fma(z, s, 1.0 / 120);
  s = fma(z, s, -1.0 / 6);
  s = fma(x * z, s, x);
  double c = fma(z, -1.0 / 3628800, 1.0 / 40320);
  c = fma(z, c, -1.0 / 720);
  c = fma(z, c, 1.0 / 24);
  c = fma(z, c, -0.5);
  c = fma(z, c, 1.0);
  const int quarter = (int)((long long)n & 3);
  const float sx = (float)s, cx = (float)c;
  const float a = quarter & 1 ? cx : sx, b = quarter & 1 ? sx : cx;
  sin_t = quarter & 2 ? -a : a;
  cos_t = quarter == 1 || quarter == 2 ? -b : b;
}

template <typename T>
struct RowPiece;  // a lane's 16 bytes of a row
template <>
struct RowPiece<__bf16> {
  static constexpr int N = 8;
  __device__ static __forceinline__ void widen(const u32x4& w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    }
  }
  __device__ static __forceinline__ u32x4 narrow(const float (&x)[8]) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = f32_to_bf16_bits(x[2 * i]) | (f32_to_bf16_bits(x[2 * i + 1]) << 16);
    return w;
  }
};
template <>
struct RowPiece<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ void widen(const u32x4& w, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
  }
  __device__ static __forceinline__ u32x4 narrow(const float (&x)[4]) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
    return w;
  }
};

// Sum over the LPR lanes of a row, the same in each.
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
  if constexpr (LPR == 32) x += __shfl_xor(x, 16, 64);
  if constexpr (LPR >= 16) return row16_sum(x);
  x += __shfl_xor(x, 4, 64);
  x += __shfl_xor(x, 2, 64);
  return x + __shfl_xor(x, 1, 64);
}

// A wave takes one token (or 1/parts of its heads): LPR lanes hold a head's row, 16 bytes each, so 64/LPR
// heads go at once. Lane l computes the token's angle l; the sines and cosines go through LDS once and stay
// in registers, where every head uses them. Sum of squares, norm and rotation are in 32 bits, rounded once
// at the store. Bound by HBM: four heads' loads ahead of their use and stores that do not displace the inputs from
// the caches (80 heads of 8191 tokens, 168 MB in and out: 95 us without either, 80 and 73 with the first, 60 to 70
// with both; the stores make no difference up to 4096 tokens).
template <typename T, int D>
__global__ __launch_bounds__(kPageBlock) void norm_rope_kernel(NormRopeArgs a) {
  using P = RowPiece<T>;
  constexpr int N = P::N, LPR = D / N, HPW = 64 / LPR;
  __shared__ float sines[kWavesPerBlock][64], cosines[kWavesPerBlock][64];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int64_t unit = (int64_t)blockIdx.x * kWavesPerBlock + wid;
  const int64_t token = unit / a.parts;
  const int part = (int)(unit - token * a.parts);
  const bool live = token < a.T;
  const int col = (lane % LPR) * N, half = a.rot / 2;

  if (live && lane < half) {
    float s, c;
    sincos_at(a.positions[token], a.inv_freq[lane], s, c);
    sines[wid][lane] = s;
    cosines[wid][lane] = c;
  }
  __syncthreads();
  if (!live) return;
  // this lane's columns: y = x * c + partner * s, with the sign of the first of a pair in s
  const bool turns = col < a.rot, first = a.interleaved || col < half;
  float cs[N], sn[N], qw[N], kw[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const int pair = a.interleaved ? (col + e) / 2 : (first ? col + e : col + e - half);
    const bool neg = a.interleaved ? (e & 1) == 0 : first;
    cs[e] = turns ? cosines[wid][pair] : 1.f;
    sn[e] = turns ? (neg ? -sines[wid][pair] : sines[wid][pair]) : 0.f;
    qw[e] = kw[e] = 1.f;
  }
  if (a.q_weight) P::widen(reinterpret_cast<const u32x4*>(a.q_weight)[lane % LPR], qw);
  if (a.k_weight) P::widen(reinterpret_cast<const u32x4*>(a.k_weight)[lane % LPR], kw);
  const int partner = a.interleaved || !turns ? lane : (first ? lane + half / N : lane - half / N);

  const int heads = a.Hq + 2 * a.Hkv;
  const char* qrow = static_cast<const char*>(a.q) + token * a.q_stride + (int64_t)(lane % LPR) * 16;
  const char* krow = static_cast<const char*>(a.k) + token * a.k_stride + (int64_t)(lane % LPR) * 16;
  const char* vrow = static_cast<const char*>(a.v) + token * a.v_stride + (int64_t)(lane % LPR) * 16;
  constexpr int RB = D * (int)sizeof(T);
  // kAhead steps' rows are loaded before the first of them is used
  constexpr int kAhead = 4;
  const int step = a.parts * HPW;
  for (int h0 = part * HPW; h0 < heads; h0 += kAhead * step) {
    u32x4 w[kAhead];
    int64_t slot[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int h = h0 + u * step + lane / LPR;
      slot[u] = -1;
      if (h >= heads) continue;
      const int kv = h < a.Hq + a.Hkv ? h - a.Hq : h - a.Hq - a.Hkv;
      w[u] = *reinterpret_cast<const u32x4*>(h < a.Hq ? qrow + h * RB : (h < a.Hq + a.Hkv ? krow : vrow) + kv * RB);
      if (h >= a.Hq) slot[u] = a.slots[token * a.Hkv + kv];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int h = h0 + u * step + lane / LPR;
      if (h0 + u * step >= heads) break;
      const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
      u32x4 y = w[u];
      float x[N];
      P::widen(y, x);
      if (is_q ? a.q_weight != nullptr : is_k && a.k_weight != nullptr) {
        // every lane of a row takes this branch together
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) ss = fmaf(x[e], x[e], ss);
        ss = row_sum<LPR>(ss);
        const float r = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = x[e] * r * (is_q ? qw[e] : kw[e]);
      }
      if (a.rot) {
        float p[N];
#pragma unroll
        for (int e = 0; e < N; ++e) p[e] = a.interleaved ? x[e ^ 1] : __shfl(x[e], partner, 64);
        if (turns && (is_q || is_k)) {  // columns that do not turn: nothing times zero, which may be infinite
#pragma unroll
          for (int e = 0; e < N; ++e) x[e] = fmaf(p[e], sn[e], x[e] * cs[e]);
        }
      }
      if (is_q || is_k) y = P::narrow(x);
      if (is_q) {
        __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(a.q_out) + (token * a.Hq + h) * LPR + lane % LPR);
      } else if (slot[u] >= 0 && slot[u] < a.total_slots) {
        __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(is_k ? a.k_pages : a.v_pages) + slot[u] * LPR +
                                           lane % LPR);
      }
    }
  }
}

}  // namespace

hipError_t launch_page_update(const PageArgs& a, int cus, hipStream_t stream) {
  const size_t lds = (3 * (size_t)a.S + (a.by_segment ? a.S : a.B) + 3) * sizeof(int32_t);
  // One workgroup per four rounds of slots, up to two per compute unit. How many pages change hands is known
  // on the device only, at most all table entries: one workgroup per 4096 of those, up to 64.
  const int64_t rounds = (a.num_slots * (a.by_segment ? 1 : a.Hkv) + 4 * kPageBlock - 1) / (4 * kPageBlock);
  const int64_t entries = (int64_t)a.S * a.max_pages;
  const int wgs = (int)std::max({(int64_t)1, std::min<int64_t>((rounds + 3) / 4, 2 * cus),
                                 std::min<int64_t>(entries / 4096, 64)});
  const bool in_place = a.rows_out == a.rows || a.head_out == a.head;
  const bool second = wgs > 1 && in_place;
  prof_begin("page_update", stream);
  page_update_kernel<false><<<dim3(wgs), dim3(kPageBlock), lds, stream>>>(a, !second);
  if (second) page_update_kernel<true><<<dim3(1), dim3(kPageBlock), lds, stream>>>(a, 1);
  prof_end(stream);
  return hipGetLastError();
}

// A launch holds fewer than 2^32 threads; more rows or tokens than that go in several.
constexpr int64_t kMaxBlocks = (int64_t(1) << 23);

hipError_t launch_paged_store(const PagedStoreArgs& args, hipStream_t stream) {
  const int64_t per = kStoreVecs * kPageBlock, most = (kMaxBlocks * per) >> args.row_shift;
  const int64_t row_bytes = int64_t(16) << args.row_shift;
  if (args.n == 0) return hipSuccess;
  prof_begin("paged_store", stream);
  for (int64_t first = 0; first < args.n; first += most) {
    PagedStoreArgs a = args;
    a.n = std::min(most, args.n - first);
    a.k = static_cast<const char*>(args.k) + first * row_bytes;
    a.v = static_cast<const char*>(args.v) + first * row_bytes;
    a.slots = args.slots + first;
    const int64_t blocks = ((a.n << a.row_shift) + per - 1) / per;
    paged_store_kernel<<<dim3((unsigned)blocks), dim3(kPageBlock), 0, stream>>>(a);
  }
  prof_end(stream);
  return hipGetLastError();
}

namespace {
void launch_norm_rope_part(const NormRopeArgs& a, hipStream_t stream) {
  const int64_t waves = (int64_t)a.T * a.parts;
  const dim3 grid((unsigned)((waves + kWavesPerBlock - 1) / kWavesPerBlock)), block(kPageBlock);
  if (a.dtype) {
    if (a.D == 128) norm_rope_kernel<__bf16, 128><<<grid, block, 0, stream>>>(a);
    else norm_rope_kernel<__bf16, 64><<<grid, block, 0, stream>>>(a);
  } else {
    if (a.D == 128) norm_rope_kernel<float, 128><<<grid, block, 0, stream>>>(a);
    else norm_rope_kernel<float, 64><<<grid, block, 0, stream>>>(a);
  }
}
}  // namespace

hipError_t launch_norm_rope(const NormRopeArgs& args, hipStream_t stream) {
  if (args.T == 0) return hipSuccess;
  // Few tokens share their heads out over several waves, up to about eight waves per compute unit in all.
  const int eb = args.dtype ? 2 : 4, row_lanes = args.D * eb / 16, heads = args.Hq + 2 * args.Hkv;
  const int steps = (heads * row_lanes + 63) / 64;  // steps of a wave that takes all heads
  const int64_t want = (2048 + (int64_t)args.T - 1) / args.T;
  const int64_t most = kMaxBlocks * kWavesPerBlock;  // tokens of a launch: beyond 2048 a token is a wave's
  prof_begin("norm_rope_store", stream);
  for (int64_t first = 0; first < args.T; first += most) {
    NormRopeArgs a = args;
    a.parts = want < steps ? (int)want : steps;
    a.T = (int)std::min(most, args.T - first);
    if (a.Hq) {
      a.q = static_cast<const char*>(args.q) + first * args.q_stride;
      a.q_out = static_cast<char*>(args.q_out) + first * args.Hq * args.D * eb;
    }
    a.k = static_cast<const char*>(args.k) + first * args.k_stride;
    a.v = static_cast<const char*>(args.v) + first * args.v_stride;
    a.positions = args.positions + first;
    a.slots = args.slots + first * args.Hkv;
    launch_norm_rope_part(a, stream);
  }
  prof_end(stream);
  return hipGetLastError();
}

}  // namespace sgdkv
