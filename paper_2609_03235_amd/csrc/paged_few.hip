// Paged attention for few query rows per KV head (single tokens, drafted tokens), and the merge of the
// partial results of every instance. See paged_attention.h.
//
// Bound by HBM: a key and value row is read once and used by at most 48 query rows. Each wave takes its own
// rows of the workgroup's key tile (no barrier in the loop): keys go from memory into registers in the MFMA's A
// layout, values straight into LDS that only this wave uses (two buffers), for the transposing read. The next
// step's loads start as soon as the step's keys are used up, so that all but the logits of a step runs beside
// them: 8 waves of a compute unit have 128 KB under way. 32 tokens over 4 x 32K rows each (28 / 4 heads of 128, bf16)
// take 335 us, 6.4 TB/s; 1 to 6 tokens of 16 sequences over 8 x 20K rows (64 / 8 heads, fp32 out) 226 to 236, 5.6 to
// 5.8 TB/s; fp32, one token of 8 sequences over 4 x 20K rows 117, 5.7 TB/s.
#include <algorithm>

#include "paged_attention.h"

namespace sgdkv {

namespace {

// Rows of values in LDS have no padding (a load writes its lanes' 16 bytes one after the other); piece c of row r
// lies at place c ^ swizzle(r), which spreads the pieces that a read takes from several rows over the banks.
template <typename T, int D>
struct FewShape {
  static constexpr int EB = sizeof(T), RB = D * EB, NC = D / 32, ND = D / 16;
  static constexpr int U = EB == 2 ? 2 : 1;              // 16-row groups per wave and step
  static constexpr int STEP = 16 * U, KT = STEP * kAttnWaves;
  static constexpr int VPR = RB / 16, RPL = 64 / VPR, NV = 16 / RPL;  // rows per load, loads per group
  static constexpr int STAGE = STEP * RB;
  static __device__ __forceinline__ int swizzle(int r) {
    return EB == 4 ? ((r >> 2) & 3) << 2 : (RB == 128 ? ((r >> 1) & 3) << 1 : (r & 7) << 1);
  }
};

// QB: 16-row query blocks. The probabilities of bf16 inputs go into the product as three bf16 terms, all their 24
// bits, whatever the output's type: the products run beside the loads that bound the call (1 token of 32 sequences over
// 32K rows 337 us with one term, 335 with three; 48 rows, 16 x 6 tokens over 4 x 20K rows, 127 and 131), and one term
// adds an error of its own (64 x 1 tokens over 5K rows 1.72e-3 of the output, rms, where the output's own rounding is
// 1.67e-3).
template <typename T, int D, int QB>
__global__ __launch_bounds__(kAttnBlock, 2) void paged_few_kernel(PagedAttnArgs a) {
  using S = FewShape<T, D>;
  constexpr int EB = S::EB, RB = S::RB, NC = S::NC, ND = S::ND, U = S::U, STEP = S::STEP, KT = S::KT, NV = S::NV;
  constexpr int M = 16 * QB;
  constexpr bool QLDS = QB > 2;    // query operands read from LDS at each use: no registers for them
  constexpr int QP = RB + 16;      // their pitch
  constexpr int OP = D + 4;        // pitch of a row of o in LDS, in floats: the rows' writes spread over the banks
  constexpr int kMerge = 16 * OP * 4;
  constexpr int kWaveLds = 2 * S::STAGE > kMerge ? 2 * S::STAGE : kMerge;
  __shared__ __attribute__((aligned(16))) char lds[kAttnWaves][kWaveLds];
  __shared__ __attribute__((aligned(16))) char qlds[QLDS ? M * QP : 16];
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
  if (!find_piece<true>(a, sc, w, share, end, padded, at)) return;
  int64_t pos = share * w;
  char* stage = lds[wid];
  const uint32_t stage0 = lds_address(stage);
  uint32_t voff[NV];  // where this lane's 16 bytes of each load of a group come from
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int r = i * S::RPL + lane / S::VPR;
    voff[i] = r * RB + ((lane % S::VPR) ^ S::swizzle(r)) * 16;
  }

  while (pos < end) {
    if (at.tile >= at.g.tiles) {  // the next segment
      if (++at.seg >= a.S) return;
      at.tile = 0;
      at.g = paged_seg(a, at.seg);
      continue;
    }
    const PagedSeg& g = at.g;
    const int limit = uniform(tile_rows(a, g, at.tile));
    const int nkt = max((limit + KT - 1) / KT, 1);
    const int j0 = (int)((pos - at.start + KT - 1) / KT);
    const int j1 = (int)min((int64_t)nkt, (end - at.start + KT - 1) / KT);
    if (j0 < j1) {
      const int h = at.seg % a.Hkv;
      const int tok0 = at.tile * a.tokens, ntok = min(a.tokens, g.n - tok0);
      const int nrow = ntok * a.G;
      const int32_t* table = a.tables + (int64_t)at.seg * a.max_pages;
      const int first_seen = seen_by(a, g, tok0);
      if (tid < D) first_odd[tid] = 0x7FFFFFFF;
      __syncthreads();  // and the tile before is done with LDS
      auto first_row = [&](int j) { return j * KT + wid * STEP; };
      int page[U];
#pragma unroll
      for (int u = 0; u < U; ++u) page[u] = group_page(a, table, first_row(j0) + 16 * u, limit);

      // query rows as B operands: row lr of block qb is head row % G of token row / G
      Frag<T> q[QLDS ? 1 : QB][NC];
      int seen[QB];
      const rsrc_t qr = make_rsrc(static_cast<const char*>(a.q) + ((int64_t)(g.t0 + tok0) * a.Hq + h * a.G) * RB,
                                  ((uint64_t)(ntok - 1) * a.Hq + a.G) * RB);
      auto query_off = [&](int r) -> uint32_t {
        const int tok = r / a.G, hd = r - tok * a.G;
        return r < nrow ? (uint32_t)((tok * a.Hq + hd) * RB) : 0xFFFF0000u;
      };
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const int r = 16 * qb + lr;
        seen[qb] = r < nrow ? seen_by(a, g, tok0 + r / a.G) : 0;
        if constexpr (!QLDS) {
          const uint32_t off = query_off(r);
#pragma unroll
          for (int c = 0; c < NC; ++c) q[qb][c] = gload_frag<T>(qr, off + (32 * c + 8 * lg) * EB);
        }
      }
      if constexpr (QLDS) {
        for (int i = tid; i < M * S::VPR; i += kAttnBlock) {
          const int r = i / S::VPR, c = i % S::VPR;
          *reinterpret_cast<u32x4*>(qlds + r * QP + c * 16) = ld128(qr, query_off(r) + c * 16);
        }
        __syncthreads();
      }
      auto query = [&](int qb, int c) {
        if constexpr (QLDS) return lds_frag<T>(qlds, (16 * qb + lr) * QP + (32 * c + 8 * lg) * EB);
        else return q[qb][c];
      };
      float m[QB], s[QB];
      f32x4 o[QB][ND];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        m[qb] = -INFINITY;
        s[qb] = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[qb][d] = f32x4{0.f, 0.f, 0.f, 0.f};
      }

      Frag<T> k[U][NC];
      auto load = [&](int j) {
        const int r0 = first_row(j);
        const uint32_t to = uniform((int)(stage0 + (j & 1) * S::STAGE));
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const u32x4 vr = group_words(a, a.v_pages, uniform(page[u]), r0 + 16 * u, limit - r0 - 16 * u, 16, RB);
#pragma unroll
          for (int i = 0; i < NV; ++i) load_to_lds_nt(vr, voff[i], to + u * 16 * RB + i * 1024);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const rsrc_t kr = group_rsrc(a, a.k_pages, uniform(page[u]), r0 + 16 * u, limit - r0 - 16 * u, RB);
#pragma unroll
          for (int c = 0; c < NC; ++c) k[u][c] = gload_frag_nt<T>(kr, (uint32_t)(lr * RB + (32 * c + 8 * lg) * EB));
        }
      };
      load(j0);
      for (int j = j0; j < j1; ++j) {
        const int r0 = first_row(j);
#pragma unroll
        for (int u = 0; u < U; ++u) page[u] = group_page(a, table, first_row(j + 1) + 16 * u, limit);
        wait_loads();  // this step's keys and values, the next one's pages
        f32x4 y[QB][U];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
          for (int u = 0; u < U; ++u) y[qb][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) {
            const Frag<T> qf = query(qb, c);
#pragma unroll
            for (int u = 0; u < U; ++u) y[qb][u] = mma(k[u][c], qf, y[qb][u]);
          }
        if (j + 1 < j1) load(j + 1);
        char* vals = stage + (j & 1) * S::STAGE;
        if (r0 + STEP > first_seen && r0 < limit)
          clean_values<EB, RB>(vals, r0, max(first_seen - r0, 0), min(limit - r0, STEP), first_odd, S::swizzle);
        float p[QB][U][4];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          // lane: query row lr; keys 16u + 4lg + i
          const int left = seen[qb] - r0 - 4 * lg;
          float mx = -INFINITY;
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, 16 * u + i < left ? y[qb][u][i] * a.c2 : -INFINITY);
          mx = max_lane_groups(mx);
          const float mn = fmaxf(m[qb], mx);
          const float ref = mn == -INFINITY ? 0.f : mn;
          const float alpha = m[qb] == -INFINITY ? 1.f : fast_exp2(m[qb] - ref);  // nothing summed yet: any
          m[qb] = mn;
          float sum = 0.f;
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float e = fast_exp2(fmaf(y[qb][u][i], a.c2, -ref));
              p[qb][u][i] = 16 * u + i < left ? e : 0.f;
              sum += p[qb][u][i];
            }
          s[qb] = fmaf(s[qb], alpha, sum);
          if (__any(alpha != 1.f)) {
#pragma unroll
            for (int d = 0; d < ND; ++d) o[qb][d] *= alpha;
          }
        }
        if constexpr (EB == 2) {
          u32x4 piece[QB][3];
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              split_bf16(p[qb][e / 2][2 * (e % 2)], p[qb][e / 2][2 * (e % 2) + 1], piece[qb], e);
          const int row = 4 * lg + lr / 4;  // and 16 further on: the same swizzle
          const char* vp = vals + row * RB + (lr & 1) * 8;
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            const char* vd = vp + (((2 * d + (lr & 3) / 2) ^ S::swizzle(row)) * 16);
            const u32x2 v0 = lds_transposed(vd), v1 = lds_transposed(vd + 16 * RB);
            Frag<__bf16> vt;
            vt.v = u32x4{v0.x, v0.y, v1.x, v1.y};
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
#pragma unroll
              for (int k = 0; k < 3; ++k) o[qb][d] = mma(vt, Frag<__bf16>{piece[qb][k]}, o[qb][d]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const char* vp = vals + (4 * lg + i) * RB + (lr & 3) * 4;
#pragma unroll
            for (int d = 0; d < ND; ++d) {
              const float v = *reinterpret_cast<const float*>(vp + (((4 * d + lr / 4) ^ S::swizzle(4 * lg)) * 16));
#pragma unroll
              for (int qb = 0; qb < QB; ++qb)
                o[qb][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[qb][0][i], o[qb][d], 0, 0, 0);
            }
          }
        }
      }
      // merge the waves' parts in wave order, 16 rows at a time
      const bool whole = j0 == 0 && j1 == nkt;
      const int64_t slot = 2 * (int64_t)w + (at.start > share * w ? 1 : 0);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const float total = sum_lane_groups(s[qb]);
        if (lg == 0) {
          mws[wid][16 * qb + lr] = m[qb];
          sws[wid][16 * qb + lr] = total;
        }
      }
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        if (16 * qb >= nrow) break;
        __syncthreads();
#pragma unroll
        for (int d = 0; d < ND; ++d)
          *reinterpret_cast<f32x4*>(stage + (lr * OP + 16 * d + 4 * lg) * 4) = o[qb][d];
        __syncthreads();
        for (int idx = tid; idx < 16 * (D / 4); idx += kAttnBlock) {
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
            const int64_t row = (int64_t)(g.t0 + tok0 + tok) * a.Hq + h * a.G + hd;
            store_out4(a, row, D, col, acc * (sum == 0.f ? 0.f : 1.0f / sum));
            if (a.lse && col == 0) a.lse[row] = lse_of(mm, sum);
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
    }
    const int64_t next = padded ? end : at.start + max(limit, 1) + (1 << a.min_shift);
    leave_shared(a, w, share, at, nkt, false);
    at.start = pos = next;
    ++at.tile;
  }
}

// Joins the parts of the query tiles that several workers shared: workgroup (x, y) looks at entry x of `shared`.
// Lanes in groups of D / 4 hold a row, four columns each.
//   Few parts: a group takes a row of its own and its parts in batches, each all under way at once.
//   Many (a long segment and few others): a workgroup takes rows y, y + gridDim.y, ...; its groups take a row's
//     parts in turn with a running maximum and are then joined in order.
// Whichever has fewer rounds of reads. (21 tokens over 57K rows of one head, 443 parts: 142 us and 34. 300 tokens
// over 900 rows of four heads, 8 or 9 parts and two rows a workgroup: 32 us and 34.)
template <int D>
__global__ __launch_bounds__(kAttnBlock) void paged_merge_kernel(PagedAttnArgs a) {
  constexpr int LPS = D / 4, NG = kAttnBlock / LPS, kBatch = 8;
  __shared__ float ms[NG], ss[NG];
  __shared__ __attribute__((aligned(16))) float os[NG][D];
  const int tid = threadIdx.x, grp = tid / LPS, col = 4 * (tid % LPS);
  // The reads come from other XCDs' writes, a microsecond each where one waits for the other: the entry and the
  // segment's lengths are asked for together.
  const int4 left = a.shared[blockIdx.x];
  const int seg = a.by_tile ? blockIdx.x / a.max_tiles : (left.w < 0 ? 0 : left.x);
  const PagedSeg g = paged_seg(a, seg);
  if (a.by_tile && (int)blockIdx.x - seg * a.max_tiles >= g.tiles) return;  // no such tile: the entry holds anything
  if (left.w < 0) return;
  const int w = left.z >> 1;
  const int M = a.tile_rows, h = seg % a.Hkv, tok0 = left.y * a.tokens;
  const int nrow = min(a.tokens, g.n - tok0) * a.G, parts = left.w - w + 1;

  float m, s;
  f32x4 o;
  // parts first, first + stride, ... of row r; a part past the last repeats it with weight zero
  auto join = [&](int r, int first, int stride) {
    m = -INFINITY;
    s = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i0 = first; i0 < parts; i0 += kBatch * stride) {
      float pm[kBatch], ps[kBatch];
      f32x4 po[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int i = min(i0 + u * stride, parts - 1);
        const int64_t at = (2 * (int64_t)(w + i) + (i == 0 ? left.z & 1 : 0)) * M + r;
        pm[u] = a.part_ms[at * 2];
        ps[u] = a.part_ms[at * 2 + 1];
        po[u] = *reinterpret_cast<const f32x4*>(a.part + at * D + col);
      }
      float mn = m;
#pragma unroll
      for (int u = 0; u < kBatch; ++u) mn = fmaxf(mn, pm[u]);
      const float ref = mn == -INFINITY ? 0.f : mn, fo = fast_exp2(m - ref);
      m = mn;
      s *= fo;
      o *= fo;
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (i0 + u * stride >= parts) break;
        const float fn = fast_exp2(pm[u] - ref);
        s += ps[u] * fn;
        o += po[u] * fn;
      }
    }
  };
  auto write = [&](int r) {
    const int tok = r / a.G, hd = r - tok * a.G;
    const int64_t row = (int64_t)(g.t0 + tok0 + tok) * a.Hq + h * a.G + hd;
    store_out4(a, row, D, col, o * (s == 0.f ? 0.f : 1.0f / s));
    if (a.lse && col == 0) a.lse[row] = lse_of(m, s);
  };
  const int ny = gridDim.y;
  if ((parts + kBatch - 1) / kBatch <= (nrow + ny - 1) / ny) {
    const int r = blockIdx.y * NG + grp;
    if (r >= nrow) return;
    join(r, 0, 1);
    write(r);
    return;
  }
  for (int r = blockIdx.y; r < nrow; r += ny) {
    join(r, grp, NG);
    __syncthreads();  // the row before is done with LDS
    if (col == 0) {
      ms[grp] = m;
      ss[grp] = s;
    }
    *reinterpret_cast<f32x4*>(&os[grp][col]) = o;
    __syncthreads();
    if (grp != 0) continue;
    m = -INFINITY;
#pragma unroll
    for (int i = 0; i < NG; ++i) m = fmaxf(m, ms[i]);
    const float ref = m == -INFINITY ? 0.f : m;
    s = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const float f = fast_exp2(ms[i] - ref);
      s += ss[i] * f;
      o += *reinterpret_cast<const f32x4*>(&os[i][col]) * f;
    }
    write(r);
  }
}

template <typename T, int D, int QB>
void launch_few(const PagedAttnArgs& a, hipStream_t stream) {
  paged_few_kernel<T, D, QB><<<dim3(kPagedWorkers), dim3(kAttnBlock), 0, stream>>>(a);
}

template <typename T, int D>
void launch_few_rows(const PagedAttnArgs& a, hipStream_t stream) {
  switch (a.tile_rows) {
    case 16: return launch_few<T, D, 1>(a, stream);
    case 32: return launch_few<T, D, 2>(a, stream);
    default:
      if constexpr (sizeof(T) == 2) launch_few<T, D, 3>(a, stream);
  }
}

}  // namespace

PagedAttnShape paged_attn_shape(int dtype, int G, int max_new) {
  const int64_t rows = (int64_t)max_new * G;
  if (rows <= (dtype ? kFewRowsBf16 : kFewRowsF32)) return {16 * (int)((rows + 15) / 16), dtype ? 128 : 64};
  return {128, dtype ? 64 : 32};
}

hipError_t launch_paged_few(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.dtype) a.D == 128 ? launch_few_rows<__bf16, 128>(a, stream) : launch_few_rows<__bf16, 64>(a, stream);
  else a.D == 128 ? launch_few_rows<float, 128>(a, stream) : launch_few_rows<float, 64>(a, stream);
  return hipGetLastError();
}

hipError_t launch_paged_attention(const PagedAttnArgs& a, hipStream_t stream) {
  const bool few = a.tile_rows < 128;
  prof_begin("paged_attention", stream);
  hipError_t e = few ? launch_paged_few(a, stream) : launch_paged_many(a, stream);
  prof_end(stream);
  if (e != hipSuccess) return e;
  prof_begin("paged_merge", stream);
  // A workgroup per row of a tile where that makes at most 4096, at least one per row group.
  const int rows = std::min(a.max_new, a.tokens) * a.G, entries = a.by_tile ? a.S * a.max_tiles : kPagedWorkers;
  const int groups = kAttnBlock / (a.D / 4);
  const dim3 grid(entries, std::max((rows + groups - 1) / groups, std::min(rows, 4096 / entries)));
  if (a.D == 128) paged_merge_kernel<128><<<grid, dim3(kAttnBlock), 0, stream>>>(a);
  else paged_merge_kernel<64><<<grid, dim3(kAttnBlock), 0, stream>>>(a);
  prof_end(stream);
  return hipGetLastError();
}

}  // namespace sgdkv
