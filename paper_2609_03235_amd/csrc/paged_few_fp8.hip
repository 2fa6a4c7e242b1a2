// Paged attention over a pool in 8 bits for few query rows per KV head (single tokens, drafted tokens). See
// paged_attention.h.
//
// Bound by HBM as the instances for wider rows are (paged_few.hip), at half the bytes, so that a byte may cost half as
// many instructions. As there each wave takes its own rows of the workgroup's key tile, keys go from memory into
// registers in the MFMA's A layout and values straight into LDS that only this wave uses. Both are widened to bf16,
// which holds them exactly, two numbers an instruction: keys with their rows' powers, which a lane has one of; values
// without, since a lane has a column of eight rows, whose powers go to the probabilities. The products are bf16 ones
// for fp32 queries too, which go in as three bf16 terms that hold all 24 bits: a third of the bf16 rate is still three
// times fp32's. (The matrix instructions that take e4m3 as it is keep 13 bits of a sum of products of different sizes.)
// 40 x 1 tokens over 4 x 30K rows, 28 / 4 heads of 128, bf16, take 200 us and 5 for the merge, 6.2 TB/s; calls of 16 x
// 2, 4 and 6 tokens over 8 x 25K rows, 64 / 8 heads, fp32 output, 149 to 154, 184 to 187 and 222 to 223, of which the
// loads alone 142 to 158.
#include <type_traits>

#include "paged_attention.h"

namespace sgdkv {

namespace {

constexpr int kFewRows = 48;

// A row's reference for its exponentials moves when a logit passes it by 2^kFar.
constexpr float kFar = 10.f;

constexpr int kKeyTile = 128;  // keys that are one worker's

// Shapes of a wave's rows.
template <int D>
struct FewBytes {
  static constexpr int NC = D / 32, ND = D / 16, NK = D / 64;  // pieces of a row, blocks of columns, loads of a key
  static constexpr int VPR = D / 16, RPL = 64 / VPR, NV = 16 / RPL;  // values: rows per load, loads per group
  // Rows of values in LDS have no padding; piece c of row r lies at place c ^ swizzle(r), so that a transposing read
  // (half of it at a time: 16 rows of a column block, 4 and 4 of each half of 32) touches every bank once.
  static __device__ __forceinline__ int swizzle(int r) {
    return D == 128 ? ((r >> 1) & 3) | ((r >> 4) & 1) << 2 : ((r >> 2) & 1) | ((r >> 4) & 1) << 1;
  }
};

__device__ __forceinline__ rsrc_t rows_buffer(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, bytes, kRsrcWord3);
}

// The same number, for the compiler a new one. What follows from a thread's number alone stays the same over all tiles,
// and is kept for the next one in registers, some 20 of them, which the steps want (16 x 5 tokens over 25K rows 209 us,
// 199 so); before and after the steps it is worked out again instead.
__device__ __forceinline__ int anew(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Eight columns of a query row from `off` on, as QT terms of bf16; `flip` holds the sign bits of a negative scale.
template <int QT>
__device__ __forceinline__ void query_terms(rsrc_t qr, uint32_t off, uint32_t flip, Frag<__bf16> (&to)[QT]) {
  if constexpr (QT == 1) {
    to[0] = gload_frag<__bf16>(qr, off);
  } else {
    const Frag<float> x = gload_frag<float>(qr, off);
    u32x4 w[3];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const u32x4& v = e < 2 ? x.v0 : x.v1;
      split_bf16(__uint_as_float(v[2 * (e % 2)]), __uint_as_float(v[2 * (e % 2) + 1]), w, e);
    }
#pragma unroll
    for (int t = 0; t < 3; ++t) to[t].v = w[t];
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) to[t].v ^= flip;
}

// QT: terms of a query (1: bf16, 3: fp32). QB: 16-row query blocks of a full tile. FINE: the
// probabilities go in as three bf16 terms, all their bits; for bf16 output of bf16 queries as two, off by 2^-16 of each
// (16 x 6 tokens over 25K rows, 64 / 8 heads, 222 to 223 us and 202 to 205).
// A wave's step is U 16-row groups, 2 or UMAX of them: with 4, twice the bytes are under way (40 x 1 tokens over 30K
// rows 222 us, 206 so), and a worker with no more than one key tile has all its waves at work with 2 (1 token over 9K
// rows 15.6 us, 17.2 with 4).
template <int D, int QT, int QB, bool FINE>
__global__ __launch_bounds__(kAttnBlock, 2) void paged_few_fp8_kernel(PagedAttnArgs a) {
  using S = FewBytes<D>;
  constexpr int NC = S::NC, ND = S::ND, NK = S::NK, NV = S::NV;
  constexpr int PT = FINE ? 3 : 2;
  constexpr int UMAX = QB == 1 ? 4 : 2, STAGE = 16 * UMAX * D;
  constexpr int M = 16 * QB, QEB = QT == 1 ? 2 : 4;
  // Query operands read from LDS at each use where their registers are wanted elsewhere. (fp32 queries of one block: 16
  // tokens over 25K rows, 28 / 4 heads, 91 us, in registers, with spills, 105.)
  constexpr bool QLDS = QT > 1 || QB > 2;
  constexpr int QP = D * 2 + 16;  // their pitch
  constexpr int OP = D + 4;  // pitch of a row of o in LDS, in floats: the rows' writes spread over the banks
  constexpr int kMerge = 16 * OP * 4;
  constexpr int kWaveLds = 2 * STAGE > kMerge ? 2 * STAGE : kMerge;
  __shared__ __attribute__((aligned(16))) char lds[kAttnWaves][kWaveLds];
  __shared__ __attribute__((aligned(16))) char qlds[QLDS ? QT * M * QP : 16];
  __shared__ float mws[kAttnWaves][M], sws[kAttnWaves][M];
  __shared__ __attribute__((aligned(16))) int first_odd[D];
  __shared__ LineScratch sc;

  const int tid = threadIdx.x, wid = uniform(tid >> 6), lane = tid & 63;
  const int lr = lane & 15, lg = lane >> 4;
  const int w = worker_of();
  int64_t share, end;
  bool padded;
  LineTile at;
  if (!a.by_tile && tid == 0) a.shared[w] = make_int4(0, 0, 0, -1);
  if (!find_piece<true, QT == 1>(a, sc, w, share, end, padded, at)) return;
  int64_t pos = share * w;
  char* stage = lds[wid];
  const uint32_t stage0 = lds_address(stage);
  uint32_t voff[2][NV];  // where this lane's 16 bytes of each load of values come from, even and odd groups
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int r = i * S::RPL + lane / S::VPR;
      voff[u][i] = r * D + ((lane % S::VPR) ^ S::swizzle(16 * u + r)) * 16;
    }
  // The scale's sign goes to the queries, so that the largest logit is the largest product.
  const float c2 = fabsf(a.c2);
  const uint32_t flip = a.c2 < 0.f ? 0x80008000u : 0u;
  // The 8 columns of a lane's piece c: a lane has 16 bytes of a key at once, two pieces.
  auto piece_col = [&](int c) { return 64 * (c / 2) + 16 * lg + 8 * (c % 2); };

  while (pos < end) {
    if (at.tile >= at.g.tiles) {  // the next segment
      if (++at.seg >= a.S) return;
      at.tile = 0;
      at.g = paged_seg(a, at.seg);
      continue;
    }
    const PagedSeg& g = at.g;
    const int limit = uniform(tile_rows(a, g, at.tile));
    const int nkt = max((limit + kKeyTile - 1) / kKeyTile, 1);
    const int j0 = (int)((pos - at.start + kKeyTile - 1) / kKeyTile);
    const int j1 = (int)min((int64_t)nkt, (end - at.start + kKeyTile - 1) / kKeyTile);

    // The worker's keys of this tile, whose query rows fill NB blocks, in steps of U groups a wave.
    auto attend = [&](auto blocks, auto groups) {
      constexpr int NB = decltype(blocks)::value, U = decltype(groups)::value, STEP = 16 * U;
      const int begin = j0 * kKeyTile, stop = min(limit, j1 * kKeyTile);
      const int steps = max((stop - begin + STEP * kAttnWaves - 1) / (STEP * kAttnWaves), 1);
      const int h = at.seg % a.Hkv;
      const int tok0 = at.tile * a.tokens, ntok = min(a.tokens, g.n - tok0);
      const int nrow = ntok * a.G;
      const int32_t* table = a.tables + (int64_t)at.seg * a.max_pages;
      const int first_seen = min(seen_by(a, g, tok0), stop);
      if (tid < D) first_odd[tid] = 0x7FFFFFFF;
      __syncthreads();  // and the tile before is done with LDS
      auto first_row = [&](int j) { return begin + (j * kAttnWaves + wid) * STEP; };
      // Pages are asked for a step before the loads that need them: a wait for a read waits for all sent before it, so
      // asked for at the step itself each would cost the step a round trip to memory.
      int page[U], next_page[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        page[u] = group_page(a, table, first_row(0) + 16 * u, stop);
        next_page[u] = group_page(a, table, first_row(1) + 16 * u, stop);
      }

      // query rows as B operands: row lr of block qb is head row % G of token row / G
      Frag<__bf16> q[QLDS ? 1 : NB][NC][QT];
      int seen[NB];
      const rsrc_t qr = make_rsrc(
          static_cast<const char*>(a.q) + ((int64_t)(g.t0 + tok0) * a.Hq + h * a.G) * (D * QEB),
          ((uint64_t)(ntok - 1) * a.Hq + a.G) * (D * QEB));
      auto query_off = [&](int r) -> uint32_t {
        const int tok = r / a.G, hd = r - tok * a.G;
        return r < nrow ? (uint32_t)((tok * a.Hq + hd) * (D * QEB)) : 0xFFFF0000u;
      };
#pragma unroll
      for (int qb = 0; qb < NB; ++qb) {
        const int r = 16 * qb + lr;
        seen[qb] = r < nrow ? min(seen_by(a, g, tok0 + r / a.G), stop) : 0;
        if constexpr (!QLDS) {
          const uint32_t off = query_off(r);
#pragma unroll
          for (int c = 0; c < NC; ++c) query_terms<QT>(qr, off + piece_col(c) * QEB, flip, q[qb][c]);
        }
      }
      if constexpr (QLDS) {
        for (int i = anew(tid); i < 16 * NB * (D / 8); i += kAttnBlock) {
          const int r = i / (D / 8), c = i % (D / 8);
          Frag<__bf16> x[QT];
          query_terms<QT>(qr, query_off(r) + c * 8 * QEB, flip, x);
#pragma unroll
          for (int t = 0; t < QT; ++t) *reinterpret_cast<u32x4*>(qlds + (t * M + r) * QP + c * 16) = x[t].v;
        }
        __syncthreads();
      }
      auto query = [&](int qb, int c, int t) {
        if constexpr (QLDS) return lds_frag<__bf16>(qlds, (t * M + 16 * qb + lr) * QP + piece_col(c) * 2);
        else return q[qb][c][t];
      };
      float m[NB], s[NB];
      f32x4 o[NB][ND];
#pragma unroll
      for (int qb = 0; qb < NB; ++qb) {
        m[qb] = -INFINITY;
        s[qb] = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[qb][d] = f32x4{0.f, 0.f, 0.f, 0.f};
      }

      u32x4 raw[U][NK];             // the keys as they come: 16 numbers of row lr
      uint32_t kcode[U], vcode[U];  // the codes of row lr, and of rows 4lg .. 4lg + 3
      auto load = [&](int j, int u) {
        // the group's rows: none of a page outside the pool or past the last one (all scalar, from one row number)
        const int r = first_row(j) + 16 * u, pg = uniform(page[u]);
        const bool ok = (uint32_t)pg < (uint32_t)a.num_pages && r < stop;
        const int n = ok ? min(stop - r, 16) : 0;
        const int64_t row = ok ? ((int64_t)pg << a.page_shift) + (r & ((1 << a.page_shift) - 1)) : 0;
        const uint64_t vp = reinterpret_cast<uint64_t>(a.v_pages) + row * D;
        const u32x4 vr = {(uint32_t)vp, (uint32_t)(vp >> 32), (uint32_t)(n * D), (uint32_t)kRsrcWord3};
        const uint32_t to = uniform((int)(stage0 + (j & 1) * STAGE)) + u * 16 * D;
#pragma unroll
        for (int i = 0; i < NV; ++i) load_to_lds_nt(vr, voff[u % 2][i], to + i * 1024);
        const rsrc_t kr = rows_buffer(static_cast<const char*>(a.k_pages) + row * D, n * D);
#pragma unroll
        for (int c = 0; c < NK; ++c) raw[u][c] = ld128_nt(kr, (uint32_t)(lr * D + 64 * c + 16 * lg));
        // Of the values' codes all 16 are read, four at once; those past the last row go to no result.
        kcode[u] = ld8(rows_buffer(a.k_scales + row, n), lr);
        vcode[u] = ld32(rows_buffer(a.v_scales + row, ok ? 16 : 0), 4 * lg);
      };
#pragma unroll
      for (int u = 0; u < U; ++u) load(0, u);
      for (int j = 0; j < steps; ++j) {
        const int r0 = first_row(j);
        wait_loads();  // this step's keys and values, the next one's pages
        // Where two waves of a SIMD want an instruction the older one has it, and the workgroup that came second takes
        // a third longer for the same keys; so they take turns (16 x 6 tokens over 25K rows 214 us, 211 so; 40 x 1 over
        // 30K 209 and 206).
        if ((j ^ (blockIdx.x / (kPagedWorkers / 2))) & 1) __builtin_amdgcn_s_setprio(2);
        else __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          page[u] = uniform(next_page[u]);
          next_page[u] = group_page(a, table, first_row(j + 2) + 16 * u, stop);
        }
        float vpow[U][4];
        f32x4 y[NB][U];
        Frag<__bf16> k[U][NC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const float kscale = conversion_scale(kcode[u]);
#pragma unroll
          for (int c = 0; c < NC; ++c)
            k[u][c] = widen_piece(raw[u][c / 2][2 * (c % 2)], raw[u][c / 2][2 * (c % 2) + 1], kscale);
#pragma unroll
          for (int i = 0; i < 4; ++i) vpow[u][i] = power_of(vcode[u] >> 8 * i & 0xFF);
#pragma unroll
          for (int qb = 0; qb < NB; ++qb) y[qb][u] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        if (j + 1 < steps) {
#pragma unroll
          for (int u = 0; u < U; ++u) load(j + 1, u);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int qb = 0; qb < NB; ++qb)
#pragma unroll
            for (int t = 0; t < QT; ++t) {
              const Frag<__bf16> qf = query(qb, c, t);
#pragma unroll
              for (int u = 0; u < U; ++u) y[qb][u] = mma(k[u][c], qf, y[qb][u]);
            }
        if (r0 >= stop) continue;  // no rows of this wave's
        char* vals = stage + (j & 1) * STAGE;
        float alpha[NB];
        // The logits become the probabilities that the values take, in place. EDGE: some row does not see all keys.
        auto softmax = [&](auto edge) {
          constexpr bool EDGE = decltype(edge)::value;
#pragma unroll
          for (int qb = 0; qb < NB; ++qb) {
            // lane: query row lr; keys 16u + 4lg + i
            const int left = seen[qb] - r0 - 4 * lg;
            float mx = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i) mx = fmaxf(mx, !EDGE || 16 * u + i < left ? y[qb][u][i] : -INFINITY);
            mx = max_lane_groups(mx) * c2;
            // The reference moves where it is left far behind: few steps rescale o.
            const float mn = mx > m[qb] + kFar ? mx : m[qb];
            const float ref = mn == -INFINITY ? 0.f : mn;
            alpha[qb] = m[qb] == mn ? 1.f : fast_exp2(m[qb] - mn);  // before the first key s and o are 0
            m[qb] = mn;
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float e = fast_exp2(fmaf(y[qb][u][i], c2, -ref)), p = e * vpow[u][i];
                const bool on = !EDGE || 16 * u + i < left;
                sum += on ? e : 0.f;
                y[qb][u][i] = on ? p : 0.f;  // the value's power may be infinite where the key is not seen
              }
            s[qb] = fmaf(s[qb], alpha[qb], sum);
          }
        };
        if (r0 + STEP <= first_seen) {
          softmax(std::false_type{});
        } else {
          clean_values8<D>(vals, r0, max(first_seen - r0, 0), min(stop - r0, STEP), first_odd, S::swizzle);
          softmax(std::true_type{});
        }
        bool moved = false;
#pragma unroll
        for (int qb = 0; qb < NB; ++qb) moved |= alpha[qb] != 1.f;
        if (__any(moved)) {
#pragma unroll
          for (int qb = 0; qb < NB; ++qb)
#pragma unroll
            for (int d = 0; d < ND; ++d) o[qb][d] *= alpha[qb];
        }
        const int row = 4 * lg + (lr & 8) * 2 + lr / 2 % 4;  // of each 32 keys: the operand's order
        const char* vp = vals + row * D + (lr & 1) * 8;
#pragma unroll
        for (int u = 0; u < U; u += 2) {
          u32x4 piece[NB][PT];
#pragma unroll
          for (int qb = 0; qb < NB; ++qb)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              split_bf16(y[qb][u + e / 2][2 * (e % 2)], y[qb][u + e / 2][2 * (e % 2) + 1], piece[qb], e);
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            const u32x2 v = lds_transposed8(vp + u * 16 * D + ((d ^ S::swizzle(row)) * 16));
            const Frag<__bf16> vt = widen_piece(v.x, v.y, 1.f);
#pragma unroll
            for (int k = 0; k < PT; ++k)
#pragma unroll
              for (int qb = 0; qb < NB; ++qb) o[qb][d] = mma(vt, Frag<__bf16>{piece[qb][k]}, o[qb][d]);
          }
        }
      }
      __builtin_amdgcn_s_setprio(0);
      // merge the waves' parts in wave order, 16 rows at a time
      const bool whole = j0 == 0 && j1 == nkt;
      const int64_t slot = 2 * (int64_t)w + (at.start > share * w ? 1 : 0);
#pragma unroll
      for (int qb = 0; qb < NB; ++qb) {
        const float total = sum_lane_groups(s[qb]);
        if (lg == 0) {
          mws[wid][16 * qb + lr] = m[qb];
          sws[wid][16 * qb + lr] = total;
        }
      }
#pragma unroll
      for (int qb = 0; qb < NB; ++qb) {
        const int l = anew(lane);
        __syncthreads();
#pragma unroll
        for (int d = 0; d < ND; ++d)
          *reinterpret_cast<f32x4*>(stage + (l % 16 * OP + 16 * d + 4 * (l / 16)) * 4) = o[qb][d];
        __syncthreads();
        for (int idx = anew(tid); idx < 16 * (D / 4); idx += kAttnBlock) {
          const int lrow = idx / (D / 4), r = 16 * qb + lrow, col = 4 * (idx % (D / 4));
          if (r >= nrow) break;
          float mm = -INFINITY;
#pragma unroll
          for (int x = 0; x < kAttnWaves; ++x) mm = fmaxf(mm, mws[x][r]);
          const float ref = mm == -INFINITY ? 0.f : mm;
          float sum = 0.f;
          f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int x = 0; x < kAttnWaves; ++x) {
            const float f = fast_exp2(mws[x][r] - ref);
            sum = fmaf(sws[x][r], f, sum);
            acc += f * *reinterpret_cast<const f32x4*>(lds[x] + (lrow * OP + col) * 4);
          }
          acc = lose_odd(acc, first_odd, col, seen_by(a, g, tok0 + r / a.G));
          if (whole) {
            const int tok = r / a.G, hd = r - tok * a.G;
            const int64_t out = (int64_t)(g.t0 + tok0 + tok) * a.Hq + h * a.G + hd;
            store_out4(a, out, D, col, acc * (sum == 0.f ? 0.f : 1.0f / sum));
            if (a.lse && col == 0) a.lse[out] = lse_of(mm, sum);
          } else {
            *reinterpret_cast<f32x4*>(a.part + (slot * M + r) * D + col) = acc;
            if (col == 0) {
              a.part_ms[(slot * M + r) * 2] = mm;
              a.part_ms[(slot * M + r) * 2 + 1] = sum;
            }
          }
        }
      }
      __syncthreads();
    };
    if (j0 < j1) {
      // only the blocks that have rows: chunks are of different lengths
      const int blocks = (min(a.tokens, g.n - at.tile * a.tokens) * a.G + 15) / 16;
      using One = std::integral_constant<int, 1>;
      using Two = std::integral_constant<int, 2>;
      if constexpr (QB == 1) {
        if (j1 - j0 > 1) attend(One{}, std::integral_constant<int, UMAX>{});
        else attend(One{}, Two{});
      } else {
        if (QB > 2 && blocks > 2) attend(std::integral_constant<int, QB>{}, Two{});
        else if (blocks > 1) attend(Two{}, Two{});
        else attend(One{}, Two{});
      }
    }
    const int64_t next = padded ? end : at.start + max(limit, 1) + (1 << a.min_shift);
    leave_shared(a, w, share, at, nkt, false);
    at.start = pos = next;
    ++at.tile;
  }
}

template <int D, int QT, int QB>
void launch_few(const PagedAttnArgs& a, hipStream_t stream) {
  const dim3 grid(kPagedWorkers), block(kAttnBlock);
  if constexpr (QT == 1) {
    if (a.out_dtype) {
      paged_few_fp8_kernel<D, QT, QB, false><<<grid, block, 0, stream>>>(a);
      return;
    }
  }
  paged_few_fp8_kernel<D, QT, QB, true><<<grid, block, 0, stream>>>(a);
}

template <int D, int QT>
void launch_few_rows(const PagedAttnArgs& a, hipStream_t stream) {
  switch (a.tile_rows) {
    case 16: return launch_few<D, QT, 1>(a, stream);
    case 32: return launch_few<D, QT, 2>(a, stream);
    default: return launch_few<D, QT, 3>(a, stream);
  }
}

}  // namespace

// More rows than a tile of few holds: tiles of 128 (paged_many.hip) but for fp32 queries of 128 columns, whose three
// terms have no room beside 128 rows' other registers: those take several tiles of few rows. (16 x 16 tokens over 25K
// rows, 64 / 8 heads, 672 to 681 us, 2048 over 8000, 28 / 4, 825 to 838, 3 x 50 over 1000, 4 / 2, 28; with tiles of
// 128 and fp32 products 1575, 1967 and 37.)
PagedAttnShape paged_attn_fp8_shape_64(int, int G, int max_new) {
  const int64_t rows = (int64_t)max_new * G;
  if (rows <= kFewRows) return {16 * (int)((rows + 15) / 16), kKeyTile};
  return {128, 64};
}
PagedAttnShape paged_attn_fp8_shape_128(int dtype, int G, int max_new) {
  const PagedAttnShape s = paged_attn_fp8_shape_64(dtype, G, max_new);
  return dtype || s.rows < 128 ? s : PagedAttnShape{kFewRows, kKeyTile};
}

hipError_t launch_paged_few_fp8(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.dtype) a.D == 128 ? launch_few_rows<128, 1>(a, stream) : launch_few_rows<64, 1>(a, stream);
  else a.D == 128 ? launch_few_rows<128, 3>(a, stream) : launch_few_rows<64, 3>(a, stream);
  return hipGetLastError();
}

hipError_t launch_paged_attention_fp8(const PagedAttnArgs& a, hipStream_t stream) {
  const bool few = a.tile_rows < 128;
  prof_begin("paged_attention_fp8", stream);
  hipError_t e = few ? launch_paged_few_fp8(a, stream) : launch_paged_many_fp8(a, stream);
  prof_end(stream);
  return e != hipSuccess ? e : launch_paged_merge(a, stream);
}

}  // namespace sgdkv
