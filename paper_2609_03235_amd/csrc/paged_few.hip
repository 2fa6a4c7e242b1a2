// Paged attention for few query rows per KV head (single tokens, drafted tokens), and the merge of the
// partial results of every instance. See paged_attention.h.
//
// Bound by HBM: a key and value row is read once and used by at most 32 query rows. Each wave takes 32 of
// the workgroup's 128 key rows per step on its own (no barrier in the loop): keys go from memory straight
// into the MFMA's A layout, values through 32 rows of LDS that only this wave uses, for the transposing
// read. The next step's rows are in flight while a step is computed.
#include <algorithm>

#include "paged_attention.h"

namespace sgdkv {

namespace {

constexpr int kStep = 32;                    // key rows per wave and step
constexpr int kTile = kStep * kAttnWaves;    // key rows per workgroup and step

// A step's rows of one wave: the keys as two 16-key A operands, the values as they lie in memory.
template <typename T, int D>
struct FewStep {
  static constexpr int EB = sizeof(T), RB = D * EB, NC = D / 32;
  static constexpr int VPR = RB / 16, RPL = 64 / VPR, NV = 16 / RPL;  // value rows per load, loads per 16 rows
  Frag<T> k[2][NC];
  u32x4 v[2][NV];
  __device__ __forceinline__ void load(const PagedAttnArgs& a, const int (&page)[2], int r0, int limit, int lane) {
    const int lr = lane & 15, lg = lane >> 4;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const rsrc_t kr = group_rsrc(a, a.k_pages, page[g], r0 + 16 * g, limit - r0 - 16 * g, RB);
      const rsrc_t vr = group_rsrc(a, a.v_pages, page[g], r0 + 16 * g, limit - r0 - 16 * g, RB);
#pragma unroll
      for (int c = 0; c < NC; ++c) k[g][c] = gload_frag_nt<T>(kr, (uint32_t)(lr * RB + (32 * c + 8 * lg) * EB));
#pragma unroll
      for (int i = 0; i < NV; ++i) v[g][i] = ld128_nt(vr, (uint32_t)(i * 1024 + lane * 16));
    }
  }
};

__device__ __forceinline__ void few_wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// QB: 16-row query blocks. FINE: probabilities as two bf16 terms (fp32 output of bf16 inputs).
template <typename T, int D, int QB, bool FINE>
__global__ __launch_bounds__(kAttnBlock, 2) void paged_few_kernel(PagedAttnArgs a) {
  using S = FewStep<T, D>;
  constexpr int EB = S::EB, RB = S::RB, NC = S::NC, ND = D / 16;
  constexpr int VP = EB == 2 ? RB + 16 : RB + 16;  // pitch of a value row in LDS
  constexpr int kStage = kStep * VP;
  constexpr int OP = D + 4;  // pitch of a row of o in LDS, in floats: the rows' writes spread over the banks
  constexpr int kMerge = 16 * QB * OP * 4;
  constexpr int kWaveLds = kStage > kMerge ? kStage : kMerge;
  __shared__ __attribute__((aligned(16))) char lds[kAttnWaves][kWaveLds];
  __shared__ float mws[kAttnWaves][16 * QB], sws[kAttnWaves][16 * QB];
  __shared__ LineScratch sc;
  constexpr int M = 16 * QB;

  const int tid = threadIdx.x, wid = uniform(tid >> 6), lane = tid & 63;
  const int lr = lane & 15, lg = lane >> 4;
  const int w = worker_of(a);
  int64_t share, end;
  bool padded;
  LineTile at;
  if (tid == 0) a.shared[w] = make_int4(0, 0, -1, 0);
  if (!find_piece<true>(a, sc, w, share, end, padded, at)) return;
  int64_t pos = share * w;
  char* stage = lds[wid];

  while (pos < end) {
    if (at.tile >= at.g.tiles) {  // the next segment
      if (++at.seg >= a.S) return;
      at.tile = 0;
      at.g = paged_seg(a, at.seg);
      continue;
    }
    const PagedSeg& g = at.g;
    const int limit = uniform(tile_rows(a, g, at.tile));
    const int nkt = max((limit + kTile - 1) / kTile, 1);
    const int j0 = (int)((pos - at.start + kTile - 1) / kTile);
    const int j1 = (int)min((int64_t)nkt, (end - at.start + kTile - 1) / kTile);
    const int h = at.seg % a.Hkv;
    if (j0 < j1) {
      const int tok0 = at.tile * a.tokens, ntok = min(a.tokens, g.n - tok0);
      const int nrow = ntok * a.G;
      // query rows as B operands: row lr of block qb is head row % G of token row / G
      Frag<T> q[QB][NC];
      int seen[QB];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const int r = 16 * qb + lr, tok = r / a.G, hd = r - tok * a.G;
        const bool on = r < nrow;
        seen[qb] = on ? seen_by(a, g, tok0 + tok) : 0;
        const rsrc_t qr = make_rsrc(static_cast<const char*>(a.q) + ((int64_t)(g.t0 + tok0) * a.Hq + h * a.G) * RB,
                                    ((uint64_t)(ntok - 1) * a.Hq + a.G) * RB);
#pragma unroll
        for (int c = 0; c < NC; ++c)
          q[qb][c] = gload_frag<T>(qr, on ? (uint32_t)((tok * a.Hq + hd) * RB + (32 * c + 8 * lg) * EB) : 0xFFFFFF00u);
      }
      float m[QB], s[QB];
      f32x4 o[QB][ND];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        m[qb] = -INFINITY;
        s[qb] = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[qb][d] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      const int32_t* table = a.tables + (int64_t)at.seg * a.max_pages;
      auto first_row = [&](int j) { return j * kTile + wid * kStep; };
      S cur, next;
      int page[2];
      auto pages = [&](int j) {
        page[0] = uniform(group_page(a, table, first_row(j), limit));
        page[1] = uniform(group_page(a, table, first_row(j) + 16, limit));
      };
      pages(j0);
      next.load(a, page, first_row(j0), limit, lane);
      if (j0 + 1 < j1) pages(j0 + 1);
      for (int j = j0; j < j1; ++j) {
        cur = next;
        const int r0 = first_row(j);
        if (j + 1 < j1) {
          next.load(a, page, first_row(j + 1), limit, lane);
          pages(j + 2);
        }
        if (r0 >= limit) continue;
        // values to LDS
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < S::NV; ++i) {
            const int row = 16 * u + i * S::RPL + lane / S::VPR;
            *reinterpret_cast<u32x4*>(stage + row * VP + (lane % S::VPR) * 16) = cur.v[u][i];
          }
        few_wave_sync();
        float p[QB][2][4];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          f32x4 y[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            y[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < NC; ++c) y[u] = mma(cur.k[u][c], q[qb][c], y[u]);
          }
          // lane: query row lr; keys 16u + 4lg + i
          float mx = -INFINITY;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (r0 + 16 * u + 4 * lg + i < seen[qb]) mx = fmaxf(mx, y[u][i] * a.c2);
          mx = max_lane_groups(mx);
          const float mn = fmaxf(m[qb], mx);
          const float ref = mn == -INFINITY ? 0.f : mn;
          const float alpha = m[qb] == -INFINITY ? 1.f : fast_exp2(m[qb] - ref);  // nothing summed yet: any
          m[qb] = mn;
          float sum = 0.f;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float e = fast_exp2(fmaf(y[u][i], a.c2, -ref));
              p[qb][u][i] = r0 + 16 * u + 4 * lg + i < seen[qb] ? e : 0.f;
              sum += p[qb][u][i];
            }
          s[qb] = fmaf(s[qb], alpha, sum);
          if (__any(alpha != 1.f)) {
#pragma unroll
            for (int d = 0; d < ND; ++d) o[qb][d] *= alpha;
          }
        }
        if constexpr (EB == 2) {
          u32x4 ph[QB], pl[QB];
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              ph[qb][2 * u] = pack_bf16(p[qb][u][0], p[qb][u][1]);
              ph[qb][2 * u + 1] = pack_bf16(p[qb][u][2], p[qb][u][3]);
              if (FINE) {
                pl[qb][2 * u] = pack_bf16_rest(p[qb][u][0], p[qb][u][1], ph[qb][2 * u]);
                pl[qb][2 * u + 1] = pack_bf16_rest(p[qb][u][2], p[qb][u][3], ph[qb][2 * u + 1]);
              }
            }
          }
          const char* vp = stage + (4 * lg + lr / 4) * VP + (lr % 4) * 8;
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            const u32x2 v0 = lds_transposed(vp + d * 32), v1 = lds_transposed(vp + 16 * VP + d * 32);
            Frag<__bf16> vt;
            vt.v = u32x4{v0.x, v0.y, v1.x, v1.y};
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
              o[qb][d] = mma(vt, Frag<__bf16>{ph[qb]}, o[qb][d]);
              if (FINE) o[qb][d] = mma(vt, Frag<__bf16>{pl[qb]}, o[qb][d]);
            }
          }
        } else {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const char* vp = stage + (16 * u + 4 * lg + i) * VP + lr * 4;
#pragma unroll
              for (int d = 0; d < ND; ++d) {
                const float v = *reinterpret_cast<const float*>(vp + d * 64);
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
                  o[qb][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[qb][u][i], o[qb][d], 0, 0, 0);
              }
            }
        }
        few_wave_sync();
      }
      // merge the waves' parts, in wave order
      __syncthreads();
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        s[qb] = sum_lane_groups(s[qb]);
        if (lg == 0) {
          mws[wid][16 * qb + lr] = m[qb];
          sws[wid][16 * qb + lr] = s[qb];
        }
#pragma unroll
        for (int d = 0; d < ND; ++d)
          *reinterpret_cast<f32x4*>(stage + ((16 * qb + lr) * OP + 16 * d + 4 * lg) * 4) = o[qb][d];
      }
      __syncthreads();
      const bool whole = j0 == 0 && j1 == nkt;
      const int64_t slot = 2 * (int64_t)w + (at.start > share * w ? 1 : 0);
      for (int idx = tid; idx < M * (D / 4); idx += kAttnBlock) {
        const int r = idx / (D / 4), col = 4 * (idx % (D / 4));
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
          acc += f * *reinterpret_cast<const f32x4*>(lds[x] + (r * OP + col) * 4);
        }
        if (whole) {
          const int tok = r / a.G, hd = r - tok * a.G;
          const int64_t row = (int64_t)(g.t0 + tok0 + tok) * a.Hq + h * a.G + hd;
          const float inv = sum == 0.f ? 0.f : 1.0f / sum;
          store_out4(a, row, D, col, acc * inv);
          if (a.lse && col == 0) a.lse[row] = lse_of(mm, sum);
        } else {
          *reinterpret_cast<f32x4*>(a.part + (slot * M + r) * D + col) = acc;
          if (col == 0) {
            a.part_ms[(slot * M + r) * 2] = mm;
            a.part_ms[(slot * M + r) * 2 + 1] = sum;
          }
        }
      }
      __syncthreads();
    }
    const int64_t next = padded ? end : at.start + max(limit, 1);
    if (next >= end) leave_shared(a, w, share, at, nkt);
    at.start = pos = next;
    ++at.tile;
  }
}

// Joins the parts of the query tiles that several workers shared: workgroup (w, y) looks at the tile that
// worker w began and left to the next ones, if any. Lanes in groups of D / 4 hold a row, four columns each.
//   MANY = false: tiles of few rows and up to hundreds of parts. A workgroup takes one row; the groups take its
//     parts in turn with a running maximum and are then joined in order.
//   MANY = true: tiles of many rows and seldom more than three parts. A group takes a row of its own (the rows
//     one after the other with the groups on the parts took 17 us for what takes 5 so).
template <int D, bool MANY>
__global__ __launch_bounds__(kAttnBlock) void paged_merge_kernel(PagedAttnArgs a) {
  constexpr int LPS = D / 4, NG = kAttnBlock / LPS;
  __shared__ float ms[NG], ss[NG];
  __shared__ __attribute__((aligned(16))) float os[NG][D];
  const int tid = threadIdx.x, grp = tid / LPS, col = 4 * (tid % LPS);
  const int w = blockIdx.x;
  const int4 left = a.shared[w];
  if (left.z < 0) return;
  const PagedSeg g = paged_seg(a, left.x);
  const int M = a.tile_rows, h = left.x % a.Hkv, tok0 = left.y * a.tokens;
  const int nrow = min(a.tokens, g.n - tok0) * a.G, parts = left.z - w + 1;
  const int r = MANY ? blockIdx.y * NG + grp : blockIdx.y;
  if (r >= nrow) return;
  float m = -INFINITY, s = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i = MANY ? 0 : grp; i < parts; i += MANY ? 1 : NG) {
    const int64_t at = (2 * (int64_t)(w + i) + (i == 0 ? left.w : 0)) * M + r;
    const float pm = a.part_ms[at * 2], ps = a.part_ms[at * 2 + 1];
    const f32x4 po = *reinterpret_cast<const f32x4*>(a.part + at * D + col);
    const float mn = fmaxf(m, pm), ref = mn == -INFINITY ? 0.f : mn;
    const float fo = fast_exp2(m - ref), fn = fast_exp2(pm - ref);
    m = mn;
    s = s * fo + ps * fn;
    o = o * fo + po * fn;
  }
  if (!MANY) {
    if (col == 0) {
      ms[grp] = m;
      ss[grp] = s;
    }
    *reinterpret_cast<f32x4*>(&os[grp][col]) = o;
    __syncthreads();
    if (grp != 0) return;
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
  }
  const int tok = r / a.G, hd = r - tok * a.G;
  const int64_t row = (int64_t)(g.t0 + tok0 + tok) * a.Hq + h * a.G + hd;
  store_out4(a, row, D, col, o * (s == 0.f ? 0.f : 1.0f / s));
  if (a.lse && col == 0) a.lse[row] = lse_of(m, s);
}

template <typename T, int D, int QB>
void launch_few(const PagedAttnArgs& a, hipStream_t stream) {
  if constexpr (sizeof(T) == 2) {
    if (a.out_dtype == 0) {
      paged_few_kernel<T, D, QB, true><<<dim3(a.workers), dim3(kAttnBlock), 0, stream>>>(a);
      return;
    }
  }
  paged_few_kernel<T, D, QB, false><<<dim3(a.workers), dim3(kAttnBlock), 0, stream>>>(a);
}

}  // namespace

PagedAttnShape paged_attn_shape(int dtype, int G, int max_new) {
  if ((int64_t)max_new * G <= 16) return {16, kTile};
  if ((int64_t)max_new * G <= 32) return {32, kTile};
  return {128, dtype ? 64 : 32};
}

hipError_t launch_paged_few(const PagedAttnArgs& a, int rows, hipStream_t stream) {
  if (a.dtype) {
    if (a.D == 128) rows == 16 ? launch_few<__bf16, 128, 1>(a, stream) : launch_few<__bf16, 128, 2>(a, stream);
    else rows == 16 ? launch_few<__bf16, 64, 1>(a, stream) : launch_few<__bf16, 64, 2>(a, stream);
  } else {
    if (a.D == 128) rows == 16 ? launch_few<float, 128, 1>(a, stream) : launch_few<float, 128, 2>(a, stream);
    else rows == 16 ? launch_few<float, 64, 1>(a, stream) : launch_few<float, 64, 2>(a, stream);
  }
  return hipGetLastError();
}

hipError_t launch_paged_attention(const PagedAttnArgs& a, hipStream_t stream) {
  prof_begin("paged_attention", stream);
  hipError_t e = a.tile_rows <= 32 ? launch_paged_few(a, a.tile_rows, stream) : launch_paged_many(a, stream);
  prof_end(stream);
  if (e != hipSuccess || a.workers == 1) return e;  // one worker shares no tile
  prof_begin("paged_merge", stream);
  if (a.tile_rows <= 32) {
    const dim3 grid(a.workers, std::min(a.max_new, a.tokens) * a.G);
    if (a.D == 128) paged_merge_kernel<128, false><<<grid, dim3(kAttnBlock), 0, stream>>>(a);
    else paged_merge_kernel<64, false><<<grid, dim3(kAttnBlock), 0, stream>>>(a);
  } else {
    const int per = kAttnBlock / (a.D / 4);  // rows of a workgroup
    const dim3 grid(a.workers, (std::min(a.max_new, a.tokens) * a.G + per - 1) / per);
    if (a.D == 128) paged_merge_kernel<128, true><<<grid, dim3(kAttnBlock), 0, stream>>>(a);
    else paged_merge_kernel<64, true><<<grid, dim3(kAttnBlock), 0, stream>>>(a);
  }
  prof_end(stream);
  return hipGetLastError();
}

}  // namespace sgdkv
