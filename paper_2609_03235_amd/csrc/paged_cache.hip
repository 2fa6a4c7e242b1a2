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
#include "device_common.h"
#include "paged_internal.h"
#include "sgdkv_internal.h"

namespace sgdkv {

namespace {

constexpr int kWavesPerBlock = kPageBlock / 64;

// ------------------------------------------------------------------ page update
// What one segment gains or loses.
struct Change {
  int64_t before, after;  // rows
  int64_t p0, p1;         // pages before and after
};

__device__ __forceinline__ Change change_of(const PageArgs& a, int s) {
  Change c;
  c.before = a.rows[s];
  const int64_t add = a.add[a.by_segment ? s : s / a.Hkv];
  c.after = c.before + add < 0 ? 0 : c.before + add;
  const int64_t mask = ((int64_t)1 << a.page_shift) - 1;
  c.p0 = (c.before + mask) >> a.page_shift;
  c.p1 = (c.after + mask) >> a.page_shift;
  return c;
}

// Exclusive prefix sum over the workgroup's threads; total receives the sum. tmp: one entry per wave.
__device__ __forceinline__ int64_t block_prefix(int64_t v, int64_t* tmp, int64_t& total) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  int64_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up((long long)x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) tmp[wid] = x;
  __syncthreads();
  int64_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWavesPerBlock; ++w) {
    if (w < wid) before += tmp[w];
    total += tmp[w];
  }
  return before + x - v;
}

// The last entry of the ascending prefix p[0 .. n) that is <= i, where empty pieces share a value.
__device__ __forceinline__ int piece_of(const int32_t* p, int n, int64_t i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Every workgroup computes the same prefix sums over the segments (they are few beside the slots) and
// then does its share of the entries, so one launch does what two with a scan between them would; where
// there are several workgroups a second, one-workgroup launch (FINAL) writes rows_out and head_out, which
// may be the inputs themselves. Nothing that one workgroup writes is read by another: table entries past
// a segment's old pages are written and those within them read; the stack is written below its head (the
// pages given back, looked up in their tables by those who take them in the same call) and read from its
// head on.
template <bool FINAL>
__global__ __launch_bounds__(kPageBlock) void page_update_kernel(PageArgs a, int single) {
  extern __shared__ int32_t lds[];
  int32_t* cu = lds;                // [pieces + 1] new rows before a segment (a sequence)
  const int pieces = a.by_segment ? a.S : a.B;
  int32_t* taken = cu + pieces + 1;  // [S + 1] pages taken before a segment
  int32_t* given = taken + a.S + 1;  // [S + 1] pages given back before a segment
  __shared__ int64_t tmp[kWavesPerBlock];
  const int tid = threadIdx.x;

  // prefix sums; a thread takes consecutive segments
  const int per = (a.S + kPageBlock - 1) / kPageBlock;
  const int s0 = min(tid * per, a.S), s1 = min(s0 + per, a.S);
  const int64_t most = (int64_t)a.max_pages << a.page_shift;
  int64_t n_taken = 0, n_given = 0;
  int bad = 0;
  for (int s = s0; s < s1; ++s) {
    const Change c = change_of(a, s);
    bad |= c.before < 0 || c.before > most || c.after > most;
    n_taken += c.p1 > c.p0 ? c.p1 - c.p0 : 0;
    n_given += c.p0 > c.p1 ? c.p0 - c.p1 : 0;
  }
  int64_t all_taken, all_given, all_new, any_bad;
  int64_t run_t = block_prefix(n_taken, tmp, all_taken);
  int64_t run_g = block_prefix(n_given, tmp, all_given);
  block_prefix(bad, tmp, any_bad);
  for (int s = s0; s < s1; ++s) {
    const Change c = change_of(a, s);
    taken[s] = (int32_t)run_t;
    given[s] = (int32_t)run_g;
    run_t += c.p1 > c.p0 ? c.p1 - c.p0 : 0;
    run_g += c.p0 > c.p1 ? c.p0 - c.p1 : 0;
  }
  const int pper = (pieces + kPageBlock - 1) / kPageBlock;
  const int i0 = min(tid * pper, pieces), i1 = min(i0 + pper, pieces);
  int64_t n_new = 0;
  for (int i = i0; i < i1; ++i) n_new += max(a.add[i], 0);
  int64_t run_n = block_prefix(n_new, tmp, all_new);
  for (int i = i0; i < i1; ++i) {
    cu[i] = (int32_t)run_n;
    run_n += max(a.add[i], 0);
  }
  const int64_t head = a.head[0], base = head - all_given;
  const int status = any_bad                                        ? 2
                     : head < 0 || head > a.num_free || base < 0    ? 3
                     : all_new > a.num_slots                        ? 4
                     : base + all_taken > a.num_free                ? 1
                                                                    : 0;
  if (tid == 0) {
    cu[pieces] = (int32_t)all_new;
    taken[a.S] = (int32_t)all_taken;
    given[a.S] = (int32_t)all_given;
  }
  __syncthreads();

  if (!FINAL) {
    const int64_t stride = (int64_t)gridDim.x * kPageBlock, first = (int64_t)blockIdx.x * kPageBlock + tid;
    if (blockIdx.x == 0) {
      for (int i = tid; i <= pieces; i += kPageBlock) a.cu_out[i] = status ? 0 : cu[i];
      if (tid == 0) a.status[0] = status;
    }
    // the page at stack index i: given back in this call below the old head, else the stack's
    auto page_at = [&](int64_t i) -> int32_t {
      if (i >= head) return a.free_pages[i];
      const int g = piece_of(given, a.S, i - base);
      return a.tables[(int64_t)g * a.max_pages + change_of(a, g).p1 + (i - base - given[g])];
    };
    if (status == 0) {
      for (int64_t i = first; i < all_taken; i += stride) {
        const int s = piece_of(taken, a.S, i);
        a.tables[(int64_t)s * a.max_pages + change_of(a, s).p0 + (i - taken[s])] = page_at(base + i);
      }
      for (int64_t i = first; i < all_given; i += stride) a.free_pages[base + i] = page_at(base + i);
    }
    // slots: a thread takes four consecutive ones
    const int64_t n = a.num_slots * (a.by_segment ? 1 : a.Hkv);
    for (int64_t at = first * 4; at < n; at += stride * 4) {
      int32_t out[4] = {-1, -1, -1, -1};
      int64_t item = a.by_segment ? at : at / a.Hkv;
      int h = a.by_segment ? 0 : (int)(at - item * a.Hkv);
      int piece = -1, seg_of = -1;
      Change c{};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (status == 0 && item < all_new) {
          if (piece < 0 || item >= cu[piece + 1]) piece = piece_of(cu, pieces, item);
          const int s = a.by_segment ? piece : piece * a.Hkv + h;
          if (s != seg_of) {
            c = change_of(a, s);
            seg_of = s;
          }
          const int64_t pos = c.before + (item - cu[piece]), j = pos >> a.page_shift;
          const int32_t page = j < c.p0 ? a.tables[(int64_t)s * a.max_pages + j]
                                        : page_at(base + taken[s] + (j - c.p0));
          const int64_t slot = ((int64_t)page << a.page_shift) + (pos & (((int64_t)1 << a.page_shift) - 1));
          out[e] = slot < 0 || slot > 0x7FFFFFFF ? -1 : (int32_t)slot;
        }
        if (a.by_segment || ++h == a.Hkv) {
          h = 0;
          ++item;
        }
      }
      if (at + 4 <= n) {
        *reinterpret_cast<int4*>(a.slots + at) = make_int4(out[0], out[1], out[2], out[3]);
      } else {
        for (int e = 0; e < 4 && at + e < n; ++e) a.slots[at + e] = out[e];
      }
    }
  }
  if (FINAL || single) {
    // one workgroup: every read of rows and head above is done
    __syncthreads();
    for (int s = tid; s < a.S; s += kPageBlock) {
      const Change c = change_of(a, s);
      a.rows_out[s] = (int32_t)(status ? c.before : c.after);
    }
    if (tid == 0) a.head_out[0] = (int32_t)(status ? head : base + all_taken);
  }
}

// ------------------------------------------------------------------ rows to their slots
__global__ __launch_bounds__(kPageBlock) void paged_store_kernel(PagedStoreArgs a) {
  const int64_t total = a.n * a.row_vecs;
  const int64_t i = (int64_t)blockIdx.x * kPageBlock + threadIdx.x;
  if (i >= total) return;
  const int64_t row = i / a.row_vecs;
  const int64_t slot = a.slots[row];
  if (slot < 0 || slot >= a.total_slots) return;
  const int64_t to = slot * a.row_vecs + (i - row * a.row_vecs);
  const u32x4 k = static_cast<const u32x4*>(a.k)[i];
  const u32x4 v = static_cast<const u32x4*>(a.v)[i];
  static_cast<u32x4*>(a.k_pages)[to] = k;
  static_cast<u32x4*>(a.v_pages)[to] = v;
}

// ------------------------------------------------------------------ norm, rotation, store
// sin and cos of 2 pi t: the quarter turn nearest t is taken off in 64 bits, which leaves an angle x in
// [-pi/4, pi/4] for the Taylor sums (the first terms left out are below 2e-9 and 2e-10), so the angle of a
// position of millions is as good as that of a small one.
__device__ __forceinline__ void sincos_turns(double t, float& sin_t, float& cos_t) {
  const double n = rint(4.0 * t);
  const float x = (float)((t - 0.25 * n) * 6.283185307179586476925);
  const float z = x * x;
  float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
  s = fmaf(z, s, 8.3333333e-3f);
  s = fmaf(z, s, -1.6666667e-1f);
  s = fmaf(x * z, s, x);
  float c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  c = fmaf(z, c, -1.3888889e-3f);
  c = fmaf(z, c, 4.1666667e-2f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.0f);
  const int quarter = (int)((long long)n & 3);
  const float a = quarter & 1 ? c : s, b = quarter & 1 ? s : c;
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

// A wave takes one token (or 1/parts of its heads): LPR lanes hold a head's row, 16 bytes each, so 64/LPR
// heads go at once. Lane l computes the token's angle l; the sines and cosines go through LDS once and stay
// in registers, where every head uses them. Sum of squares, norm and rotation are in 32 bits, rounded once
// at the store.
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
    const double turns = (double)a.positions[token] * ((double)a.inv_freq[lane] * 0.159154943091895335769);
    float s, c;
    sincos_turns(turns, s, c);
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
  for (int h0 = part * HPW; h0 < heads; h0 += a.parts * HPW) {
    const int h = h0 + lane / LPR;
    const bool on = h < heads;
    const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
    const int kv = is_k ? h - a.Hq : h - a.Hq - a.Hkv;
    u32x4 w{};
    if (on) w = *reinterpret_cast<const u32x4*>(is_q ? qrow + h * RB : (is_k ? krow : vrow) + kv * RB);
    u32x4 y = w;
    float x[N];
    P::widen(w, x);
    if (is_q ? a.q_weight != nullptr : is_k && a.k_weight != nullptr) {
      // every lane of a row takes this branch together
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
      for (int o = LPR / 2; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
      const float r = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = x[e] * r * (is_q ? qw[e] : kw[e]);
    }
    if (a.rot) {
      float p[N];
#pragma unroll
      for (int e = 0; e < N; ++e) p[e] = a.interleaved ? x[e ^ 1] : __shfl(x[e], partner, 64);
      if (is_q || is_k) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = fmaf(p[e], sn[e], x[e] * cs[e]);
      }
    }
    if (is_q || is_k) y = P::narrow(x);
    if (!on) continue;
    if (is_q) {
      reinterpret_cast<u32x4*>(a.q_out)[(token * a.Hq + h) * LPR + lane % LPR] = y;
    } else {
      const int64_t slot = a.slots[token * a.Hkv + kv];
      if (slot >= 0 && slot < a.total_slots)
        reinterpret_cast<u32x4*>(is_k ? a.k_pages : a.v_pages)[slot * LPR + lane % LPR] = y;
    }
  }
}

}  // namespace

hipError_t launch_page_update(const PageArgs& a, int cus, hipStream_t stream) {
  const size_t lds = ((size_t)(a.by_segment ? a.S : a.B) + 2 * (size_t)a.S + 3) * sizeof(int32_t);
  const int64_t items = a.num_slots * (a.by_segment ? 1 : a.Hkv);
  // one workgroup up to 4 rounds of slots
  int64_t wgs = (items + 4 * kPageBlock * 4 - 1) / (4 * kPageBlock * 4);
  if (wgs < 1) wgs = 1;
  if (wgs > cus) wgs = cus;
  const int single = wgs == 1;
  prof_begin("page_update", stream);
  page_update_kernel<false><<<dim3((unsigned)wgs), dim3(kPageBlock), lds, stream>>>(a, single);
  if (!single) page_update_kernel<true><<<dim3(1), dim3(kPageBlock), lds, stream>>>(a, 0);
  prof_end(stream);
  return hipGetLastError();
}

hipError_t launch_paged_store(const PagedStoreArgs& a, int cus, hipStream_t stream) {
  (void)cus;
  if (a.n == 0) return hipSuccess;
  const int64_t blocks = (a.n * a.row_vecs + kPageBlock - 1) / kPageBlock;
  prof_begin("paged_store", stream);
  paged_store_kernel<<<dim3((unsigned)blocks), dim3(kPageBlock), 0, stream>>>(a);
  prof_end(stream);
  return hipGetLastError();
}

hipError_t launch_norm_rope(const NormRopeArgs& args, hipStream_t stream) {
  NormRopeArgs a = args;
  if (a.T == 0) return hipSuccess;
  // Few tokens share their heads out over several waves, up to about eight waves per compute unit in all.
  const int row_lanes = a.D * (a.dtype ? 2 : 4) / 16, heads = a.Hq + 2 * a.Hkv;
  const int steps = (heads * row_lanes + 63) / 64;  // steps of a wave that takes all heads
  const int64_t want = (2048 + a.T - 1) / a.T;
  a.parts = want < steps ? (int)want : steps;
  const int64_t waves = (int64_t)a.T * a.parts;
  const dim3 grid((unsigned)((waves + kWavesPerBlock - 1) / kWavesPerBlock)), block(kPageBlock);
  prof_begin("norm_rope_store", stream);
  if (a.dtype) {
    if (a.D == 128) norm_rope_kernel<__bf16, 128><<<grid, block, 0, stream>>>(a);
    else norm_rope_kernel<__bf16, 64><<<grid, block, 0, stream>>>(a);
  } else {
    if (a.D == 128) norm_rope_kernel<float, 128><<<grid, block, 0, stream>>>(a);
    else norm_rope_kernel<float, 64><<<grid, block, 0, stream>>>(a);
  }
  prof_end(stream);
  return hipGetLastError();
}

}  // namespace sgdkv
