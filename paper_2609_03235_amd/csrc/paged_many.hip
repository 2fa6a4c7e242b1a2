// Paged attention for many query rows per KV head (chunks of new tokens). See paged_attention.h.
//
// A workgroup holds 128 query rows, 32 per wave, and walks the keys of its piece of the line in tiles that all four
// waves share through LDS: two buffers, one barrier per tile, and the next tile on its way from memory straight into
// LDS while one is computed (no registers, no LDS writes). A query tile's first keys and its queries are under way
// while the results of the one before are written, whole lines at a time (312 prompts of 64 tokens, 64 / 8 heads: 247
// us with one after the other, 16 bytes of a row at a time; 206 with this, 194 now). Products are 32x32 MFMAs. Every
// row keeps a reference for its exponentials that only moves when a tile's sum shows that it fell too far behind, so a
// logit costs one fma, one exp2 and one add. 32 query rows a wave and two workgroups a compute unit are what the
// registers (o takes 64, the queries 32, a tile's logits 32) and LDS (64 KB each) hold; the second workgroup runs
// while the first waits. Bound by the matrix unit and the vector unit, 29 % of the matrix unit's cycles at once and
// the others one after the other, at the clock that the socket's power leaves (1.64 GHz; 2.36 on zeros): two sequences
// of 8192 tokens over 16K rows, 64 / 8 heads of 128, bf16: 10.3 to 10.7 ms, 0.97 to 1.01 PFLOP/s (0.93 on the slowest
// card seen; 8.5 to 9.0 ms on zeros).
#include <type_traits>

#include "paged_attention.h"

namespace sgdkv {

namespace {

// Rows in LDS have no padding (a load writes its lanes' 16 bytes one after the other); the 16-byte pieces of a
// row change places instead, piece c of row r lying at place c ^ key_swizzle(r) (value_swizzle): reads of one
// piece of 16 rows, or of four pieces of four rows, touch every bank once.
template <typename T, int D>
struct ManyShape {
  static constexpr int EB = sizeof(T), RB = D * EB;
  static constexpr int KT = EB == 2 ? 64 : 32;    // keys per tile
  static constexpr int RPW = KT / kAttnWaves;     // rows a wave loads
  static constexpr int VPR = RB / 16, RPL = 64 / VPR, NL = RPW / RPL;  // rows per load, loads per wave
  static constexpr int NK = KT / 32, ND = D / 32;
  static constexpr int NC = EB == 2 ? D / 16 : D / 8;  // 16-byte operand pieces of a row per lane half
  static constexpr int TILE = KT * RB;
  static __device__ __forceinline__ int key_swizzle(int r) { return RB == 128 ? (r >> 1) & 7 : r & 15; }
  static __device__ __forceinline__ int value_swizzle(int r) {
    return EB == 4 ? ((r >> 2) & 1) << 3 : (RB == 128 ? ((r >> 1) & 1) << 2 : (r & 3) << 2);
  }
};

// A query tile of at most so many keys is one worker's alone where that is at most twice a worker's share: a part
// of a tile costs 64 KB of partial results, as much time as about 400 keys, written and read again (8 sequences of
// 512 tokens with 28 / 4 heads 61 us with 256 for 512, 52 so; 3 of 128 over 600 rows, whose tiles the second half
// leaves shared, 32 and 36).
template <typename T>
constexpr int kUnshared = sizeof(T) == 2 ? 512 : 128;

// Reference kept while a tile's sum of exponentials stays below this.
constexpr float kFar = 1024.f;

// A tile's probabilities of one lane, as the operand of the product with the values. bf16 output of bf16 inputs:
// rounded to bf16, each off by up to 2^-8 of itself. The keys' errors average out: 1 x 1999 tokens over 8K rows, 28 / 4
// heads, are off by 2.00e-3 of the output (rms), of which its own rounding to bf16 makes 1.66e-3. FINE (fp32 output)
// keeps all 24 bits in three terms, 6.6e-7, at three times these products: 445 us for 268, and 18.0 ms for 10.5 with
// two sequences of 8192 tokens over 16K rows, 64 / 8 heads. A caller who wants them asks for fp32 output.
template <typename T, bool FINE, int NK>
struct Probs;
template <int NK>
struct Probs<float, false, NK> {
  float v[NK][16];
  __device__ __forceinline__ void set(int n, int i, float x, float y) {
    v[n][i] = x;
    v[n][i + 1] = y;
  }
};
template <int NK>
struct Probs<__bf16, false, NK> {
  u32x4 hi[2 * NK];  // piece t: keys 16t .. 16t + 15 in the accumulator's order
  __device__ __forceinline__ void set(int n, int i, float x, float y) {
    hi[2 * n + i / 8][(i % 8) / 2] = pack_bf16(x, y);
  }
  __device__ __forceinline__ void pieces(int t, u32x4 (&to)[1]) const { to[0] = hi[t]; }
};
template <int NK>
struct Probs<__bf16, true, NK> : Probs<float, false, NK> {
  __device__ __forceinline__ void pieces(int t, u32x4 (&to)[3]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float* x = &this->v[t / 2][8 * (t % 2) + 2 * e];
      split_bf16(x[0], x[1], to, e);
    }
  }
};

// A tile of the line as its worker does it.
struct ManyTile {
  LineTile at;
  int limit, nkt;  // rows that it sees, in so many key tiles
  int j0, j1;      // the worker's
  bool own;        // not shared
};

template <typename T, int D, bool FINE>
__global__ __launch_bounds__(kAttnBlock, 2) void paged_many_kernel(PagedAttnArgs a) {
  using S = ManyShape<T, D>;
  constexpr int EB = S::EB, RB = S::RB, KT = S::KT, NC = S::NC, NK = S::NK, ND = S::ND, NL = S::NL;
  constexpr int M = 128;
  __shared__ __attribute__((aligned(16))) char lds[2][2][S::TILE];  // two buffers of keys and values
  __shared__ __attribute__((aligned(16))) int odd[2][D];            // first_odd of this tile and of the next
  __shared__ LineScratch sc;

  const int tid = threadIdx.x, wid = uniform(tid >> 6), lane = tid & 63;
  const int lq = lane & 31, half = lane >> 5;
  const int w = worker_of();
  int64_t share, end;
  bool padded;
  LineTile at;
  if (!a.by_tile && tid == 0) a.shared[w] = make_int4(0, 0, 0, -1);
  if (!find_piece<false>(a, sc, w, share, end, padded, at)) return;
  int64_t pos = share * w;

  // where this lane's 16 bytes of each load come from, within the wave's rows
  const int my_row = wid * S::RPW;
  uint32_t koff[NL], voff[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int r = i * S::RPL + lane / S::VPR, c = lane % S::VPR;
    koff[i] = r * RB + (c ^ S::key_swizzle(my_row + r)) * 16;
    voff[i] = r * RB + (c ^ S::value_swizzle(my_row + r)) * 16;
  }
  const uint32_t lds0 = lds_address(&lds[0][0][0]);

  // The next tile of the piece that this worker does, if there is one.
  auto advance = [&](ManyTile& t) {
    while (pos < end) {
      if (at.tile >= at.g.tiles) {  // the next segment
        if (++at.seg >= a.S) return false;
        at.tile = 0;
        at.g = paged_seg(a, at.seg);
        continue;
      }
      t.at = at;
      t.limit = uniform(tile_rows(a, at.g, at.tile));
      t.nkt = max((t.limit + KT - 1) / KT, 1);
      // A tile of few keys is not shared: the worker that it starts with does all of it.
      t.own = t.limit <= kUnshared<T> && t.limit + (1 << a.min_shift) <= 2 * share;
      t.j0 = t.own ? (at.start < share * w ? t.nkt : 0) : (int)((pos - at.start + KT - 1) / KT);
      t.j1 = t.own ? t.nkt : (int)min((int64_t)t.nkt, (end - at.start + KT - 1) / KT);
      at.start = pos = at.start + max(t.limit, 1) + (1 << a.min_shift);
      ++at.tile;
      if (t.j0 < t.j1) return true;
    }
    return false;
  };

  const int r = wid * 32 + lq, tok = r / a.G, hd = r - tok * a.G;  // the lane's row of a tile
  const int32_t* table;
  int page;
  u32x4 q[NC];
  auto load = [&](const ManyTile& t, int j) {
    const int r0 = j * KT + my_row;
    const u32x4 kr = group_words(a, a.k_pages, page, r0, t.limit - r0, S::RPW, RB);
    const u32x4 vr = group_words(a, a.v_pages, page, r0, t.limit - r0, S::RPW, RB);
    const uint32_t to = uniform((int)(lds0 + (j & 1) * 2 * S::TILE + my_row * RB));
#pragma unroll
    for (int i = 0; i < NL; ++i) load_to_lds(kr, koff[i], to + i * 1024);
#pragma unroll
    for (int i = 0; i < NL; ++i) load_to_lds(vr, voff[i], to + S::TILE + i * 1024);
  };
  // Sets a tile's queries and first keys on their way; by then all waves are done with the keys before.
  auto begin = [&](const ManyTile& t, int which) {
    table = a.tables + (int64_t)t.at.seg * a.max_pages;
    // Both pages are read before the loads: a wait for a read waits for all that were sent before it.
    page = group_page(a, table, t.j0 * KT + my_row, t.limit);
    const int page2 = uniform(group_page(a, table, (t.j0 + 1) * KT + my_row, t.limit));
    page = uniform(page);
    load(t, t.j0);
    page = page2;
    const int tok0 = t.at.tile * a.tokens, ntok = min(a.tokens, t.at.g.n - tok0);
    const rsrc_t qr = make_rsrc(
        static_cast<const char*>(a.q) + ((int64_t)(t.at.g.t0 + tok0) * a.Hq + t.at.seg % a.Hkv * a.G) * RB,
        ((uint64_t)(ntok - 1) * a.Hq + a.G) * RB);
    uint32_t from = r < ntok * a.G ? (uint32_t)((tok * a.Hq + hd) * RB + 16 * half) : 0xFFFFF000u;  // or past the end
    asm("" : "+v"(from));  // one path for both: the compiler makes two of every load otherwise
#pragma unroll
    for (int c = 0; c < NC; ++c) q[c] = ld128(qr, from + 32 * c);
    if (tid < D) odd[which][tid] = 0x7FFFFFFF;
  };

  ManyTile now, t;
  bool busy = false;
  int which = 0;
  float m, s;
  f32x16 o[ND];
  for (;;) {
    // The next tile's reads go out before the results of the one before.
    const bool more = advance(t);
    if (more) begin(t, which);
    if (busy) {
      leave_shared(a, w, share, now.at, now.nkt, now.own);
      const PagedSeg& g = now.at.g;
      const int tok0 = now.at.tile * a.tokens, h = now.at.seg % a.Hkv;
      const int nrow = min(a.tokens, g.n - tok0) * a.G;
      const bool on = r < nrow;
      const int seen = on ? seen_by(a, g, tok0 + tok) : 0;
      const int* first_odd = odd[which ^ 1];
      s += __shfl_xor(s, 32, 64);
      auto result = [&](int d, int i) {
        return lose_odd(f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]}, first_odd,
                        32 * d + 8 * i + 4 * half, seen);
      };
      if (now.j0 == 0 && now.j1 == now.nkt) {
        const int64_t row0 = (int64_t)(g.t0 + tok0) * a.Hq + h * a.G;  // the tile's first
        const float inv = s == 0.f ? 0.f : 1.0f / s;
        // Through LDS, in the buffer that the next tile's first keys do not go to, so that whole lines are written:
        // the wave's 32 rows of 2 * D bytes, a bf16 row or half of an fp32 one.
        char* mine = lds[~t.j0 & 1][0] + wid * (S::TILE / 2);
        auto store = [&](auto out) {
          constexpr int OB = sizeof(out), LPR = D / 8, DP = 2 * ND / OB;  // lanes to a row, blocks of 32 columns
          char* to = static_cast<char*>(a.out) + row0 * (D * OB);
#pragma unroll
          for (int d0 = 0; d0 < ND; d0 += DP) {
#pragma unroll
            for (int d = 0; d < DP; ++d)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const f32x4 v = result(d0 + d, i) * inv;
                const int byte = (32 * d + 8 * i + 4 * half) * OB;
                char* place = mine + lq * (2 * D) + (((byte / 16) ^ (lq & (LPR - 1))) * 16) + byte % 16;
                if constexpr (OB == 2)
                  *reinterpret_cast<u32x2*>(place) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
                else
                  *reinterpret_cast<f32x4*>(place) = v;
              }
#pragma unroll 2
            for (int r0 = 0; r0 < 32; r0 += 64 / LPR) {
              const int from = r0 + lane / LPR, c = lane % LPR;
              const u32x4 v = *reinterpret_cast<const u32x4*>(mine + from * (2 * D) + ((c ^ (from & (LPR - 1))) * 16));
              const uint32_t row = __shfl(tok * a.Hq + hd, from, 64);
              if (wid * 32 + from < nrow)
                *reinterpret_cast<u32x4*>(to + (row * (D * OB) + (uint32_t)(d0 * 32 * OB + c * 16))) = v;
            }
          }
        };
        if (FINE || (EB == 4 && !a.out_dtype)) store(float{});
        else store(__bf16{});
        if (on && a.lse && half == 0) a.lse[row0 + tok * a.Hq + hd] = lse_of(m, s);
      } else if (on) {
        const int64_t slot = 2 * (int64_t)w + (now.at.start > share * w ? 1 : 0);
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4*>(a.part + (slot * M + r) * D + 32 * d + 8 * i + 4 * half) = result(d, i);
        if (half == 0) {
          a.part_ms[(slot * M + r) * 2] = m;
          a.part_ms[(slot * M + r) * 2 + 1] = s;
        }
      }
    }
    if (!more) return;
    busy = true;
    now = t;
    const PagedSeg& g = now.at.g;
    const int limit = now.limit, tok0 = now.at.tile * a.tokens;
    const int nrow = min(a.tokens, g.n - tok0) * a.G;
    const bool on = r < nrow;
    const int seen = on ? seen_by(a, g, tok0 + tok) : 0;
    const int first_seen = seen_by(a, g, tok0);
    // the rows of this wave see at most hi keys
    const int hi = wid * 32 < nrow ? uniform(seen_by(a, g, tok0 + (min(nrow, wid * 32 + 32) - 1) / a.G)) : 0;
    int* first_odd = odd[which];
    m = on ? -INFINITY : 0.f;
    s = 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

    // One tile of keys, from key0 on, out of LDS. EDGE: some row does not see all of it; `left` is how many of the
    // keys from 4 * half on this lane's row sees.
    auto attend = [&](char* kb, auto edge, int key0, bool first) {
      constexpr bool EDGE = decltype(edge)::value;
      const int left = seen - key0 - 4 * half;
      char* vb = kb + S::TILE;
      // products first where waves compete: the other waves' exponentials fill in
      __builtin_amdgcn_s_setprio(1);
      f32x16 y[NK];
      const int ksw = S::key_swizzle(lq);  // of every block's row: 32 rows on it repeats
#pragma unroll
      for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) y[n][i] = 0.f;
      auto key = [&](int n, int c) {
        return *reinterpret_cast<const u32x4*>(kb + (32 * n + lq) * RB + (((2 * c + half) ^ ksw) * 16));
      };
      if constexpr (EB == 2) {
        // Four pieces are read while the four before are multiplied. (Left alone, the compiler reads each just before
        // its product and waits: with the same for the values, 8192 tokens over 16K rows took 10.8 ms, and 10.4 so, in
        // turn on one card.)
        u32x4 kf[2][4];
        auto read = [&](int g) {
#pragma unroll
          for (int e = 0; e < 4; ++e) kf[g & 1][e] = key(e % NK, 2 * g + e / NK);
        };
        read(0);
#pragma unroll
        for (int g = 0; g < NK * NC / 4; ++g) {
          if (g + 1 < NK * NC / 4) read(g + 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            y[e % NK] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[g & 1][e]),
                                                                __builtin_bit_cast(bf16x8, q[2 * g + e / NK]),
                                                                y[e % NK], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const u32x4 kf = key(n, c);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              y[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), __uint_as_float(q[c][e]), y[n], 0, 0,
                                                          0);
          }
      }
      __builtin_amdgcn_s_setprio(0);
      // lane: query row lq; register i of block n: key 32n + 8(i / 4) + 4 half + i % 4
      auto sees = [&](int n, int i) { return !EDGE || 32 * n + 8 * (i / 4) + i % 4 < left; };
      float sum;
      Probs<T, FINE, NK> p;
      auto exps = [&](float ref) {
        float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float e0 = fast_exp2(fmaf(y[n][i], a.c2, -ref)), e1 = fast_exp2(fmaf(y[n][i + 1], a.c2, -ref));
            const float p0 = sees(n, i) ? e0 : 0.f, p1 = sees(n, i + 1) ? e1 : 0.f;
            part[(i / 2) & 3] += p0;
            part[(i / 2) & 3] += p1;
            p.set(n, i, p0, p1);
          }
        sum = (part[0] + part[1]) + (part[2] + part[3]);
      };
      // The first keys of a tile have no reference yet: at once to the branch (prompts of 64 tokens 3 % faster; in
      // the tiles that every row sees whole the test costs long calls as much).
      if (EDGE && first) sum = INFINITY;
      else exps(m);
      // All lanes take this branch or none, and none branches in it: so the compiler keeps o in place.
      if (__any(!(sum <= kFar) || m == -INFINITY)) {
        float mx = -INFINITY;
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sees(n, i) ? y[n][i] * a.c2 : -INFINITY);
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float mn = fmaxf(m, mx);
        const float alpha = m == mn ? 1.f : fast_exp2(m - mn);  // before the first key s and o are 0
        s *= alpha;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
        m = mn;
        exps(m == -INFINITY ? 0.f : m);  // nothing seen so far: all are 0
      }
      s += sum;
      if constexpr (EDGE) clean_values<EB, RB>(vb, key0, max(first_seen - key0, 0), min(limit - key0, KT), first_odd,
                                             S::value_swizzle);
      __builtin_amdgcn_s_setprio(1);
      if constexpr (EB == 2) {
        const int l16 = lane & 15;
        const int row = 4 * half + l16 / 4;                        // and 8, 16, ... further on: the same swizzle
        const int place = 2 * ((lane >> 4) & 1) + (l16 & 3) / 2;  // of a block's four pieces
        const char* vp = vb + row * RB + (l16 & 1) * 8;
        auto values = [&](int t, int d) {
          const char* vd = vp + (((4 * d + place) ^ S::value_swizzle(row)) * 16);
          const u32x2 v0 = lds_transposed(vd + 16 * t * RB), v1 = lds_transposed(vd + (16 * t + 8) * RB);
          return u32x4{v0.x, v0.y, v1.x, v1.y};
        };
        u32x4 vf[2][ND];
        auto read = [&](int t) {
#pragma unroll
          for (int d = 0; d < ND; ++d) vf[t & 1][d] = values(t, d);
        };
        read(0);
#pragma unroll
        for (int t = 0; t < KT / 16; ++t) {
          if (t + 1 < KT / 16) read(t + 1);
          u32x4 piece[FINE ? 3 : 1];
          p.pieces(t, piece);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int k = 0; k < (FINE ? 3 : 1); ++k)
#pragma unroll
            for (int d = 0; d < ND; ++d)
              o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[t & 1][d]),
                                                             __builtin_bit_cast(bf16x8, piece[k]), o[d], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
        auto value = [&](int n, int i, int d) {
          const int row = 32 * n + 8 * (i / 4) + 4 * half + i % 4;
          const int at = ((8 * d + lq / 4) ^ S::value_swizzle(4 * half)) * 16 + (lq & 3) * 4;
          return *reinterpret_cast<const float*>(vb + row * RB + at);
        };
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int d = 0; d < ND; ++d)
              o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(value(n, i, d), p.v[n][i], o[d], 0, 0, 0);
      }
      __builtin_amdgcn_s_setprio(0);
    };

    wait_loads();
    // Tells the compiler that the queries are there too: it would wait for them in the loop, and so for its loads.
#pragma unroll
    for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(q[c]));
    __syncthreads();
    // the tiles that every row sees whole, then the others
    int j = now.j0;
    auto tiles = [&](int to, auto edge) {
      for (; j < to; ++j) {
        // the page of the tile after the next, asked for before the next tile's loads and used after them
        const int page2 = group_page(a, table, (j + 2) * KT + my_row, limit);
        if (j + 1 < now.j1) load(now, j + 1);
        if (j * KT < hi) attend(lds[j & 1][0], edge, j * KT, j == now.j0);
        wait_loads();
        page = uniform(page2);
        __syncthreads();
      }
    };
    tiles(min(now.j1, first_seen / KT), std::false_type{});
    tiles(now.j1, std::true_type{});
    which ^= 1;
  }
}

template <typename T, int D>
void launch_many(const PagedAttnArgs& a, hipStream_t stream) {
  if constexpr (sizeof(T) == 2) {
    if (a.out_dtype == 0) {
      paged_many_kernel<T, D, true><<<dim3(kPagedWorkers), dim3(kAttnBlock), 0, stream>>>(a);
      return;
    }
  }
  paged_many_kernel<T, D, false><<<dim3(kPagedWorkers), dim3(kAttnBlock), 0, stream>>>(a);
}

}  // namespace

hipError_t launch_paged_many(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.dtype) a.D == 128 ? launch_many<__bf16, 128>(a, stream) : launch_many<__bf16, 64>(a, stream);
  else a.D == 128 ? launch_many<float, 128>(a, stream) : launch_many<float, 64>(a, stream);
  return hipGetLastError();
}

}  // namespace sgdkv
