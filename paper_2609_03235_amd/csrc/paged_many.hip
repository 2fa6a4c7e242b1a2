// Paged attention for many query rows per KV head (chunks of new tokens). See paged_attention.h.
//
// A workgroup holds 128 query rows, 32 per wave, and walks the keys of its piece of the line in tiles that
// all four waves share through LDS (two buffers, one barrier per tile; the tile after the next is in flight
// in registers). Products are 32x32 MFMAs. Every row keeps a reference for its exponentials that only moves
// when a tile's sum shows that it fell too far behind, so a logit costs one fma, one exp2 and one add.
#include "paged_attention.h"

namespace sgdkv {

namespace {

template <typename T, int D>
struct ManyShape {
  static constexpr int EB = sizeof(T), RB = D * EB;
  static constexpr int KT = EB == 2 ? 64 : 32;    // keys per tile
  static constexpr int RPW = KT / kAttnWaves;     // rows a wave loads
  static constexpr int VPR = RB / 16, RPL = 64 / VPR, NL = RPW / RPL;  // rows per load, loads per wave
  static constexpr int KP = RB + 16;                   // pitch of a key row in LDS
  static constexpr int VP = EB == 2 ? RB + 64 : RB + 16;  // pitch of a value row
  static constexpr int NK = KT / 32, ND = D / 32;
  static constexpr int NC = EB == 2 ? D / 16 : D / 8;  // 16-byte operand pieces of a row per lane half
  static constexpr int LDS = KT * (KP + VP);
};

// Reference kept while a tile's sum of exponentials stays below this.
constexpr float kFar = 1024.f;

template <typename T, int D, bool FINE>
__global__ __launch_bounds__(kAttnBlock, 2) void paged_many_kernel(PagedAttnArgs a) {
  using S = ManyShape<T, D>;
  constexpr int EB = S::EB, RB = S::RB, KT = S::KT, NC = S::NC, NK = S::NK, ND = S::ND, NL = S::NL;
  constexpr int KP = S::KP, VP = S::VP, M = 128;
  __shared__ __attribute__((aligned(16))) char lds[2][S::LDS];
  __shared__ LineScratch sc;

  const int tid = threadIdx.x, wid = uniform(tid >> 6), lane = tid & 63;
  const int lq = lane & 31, half = lane >> 5;
  const int w = worker_of(a);
  int64_t share, end;
  bool padded;
  LineTile at;
  if (tid == 0) a.shared[w] = make_int4(0, 0, -1, 0);
  if (!find_piece<false>(a, sc, w, share, end, padded, at)) return;
  int64_t pos = share * w;

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
    const int h = at.seg % a.Hkv;
    if (j0 < j1) {
      const int tok0 = at.tile * a.tokens, ntok = min(a.tokens, g.n - tok0);
      const int nrow = ntok * a.G;
      const int r = wid * 32 + lq, tok = r / a.G, hd = r - tok * a.G;
      const bool on = r < nrow;
      const int seen = on ? seen_by(a, g, tok0 + tok) : 0;
      // the rows of this wave see between lo and hi keys
      const bool any_row = wid * 32 < nrow;
      const int lo = any_row ? uniform(seen) : 0;
      const int hi = any_row ? seen_by(a, g, tok0 + (min(nrow, wid * 32 + 32) - 1) / a.G) : 0;
      u32x4 q[NC];
      {
        const rsrc_t qr = make_rsrc(static_cast<const char*>(a.q) + ((int64_t)(g.t0 + tok0) * a.Hq + h * a.G) * RB,
                                    ((uint64_t)(ntok - 1) * a.Hq + a.G) * RB);
#pragma unroll
        for (int c = 0; c < NC; ++c)
          q[c] = ld128(qr, on ? (uint32_t)((tok * a.Hq + hd) * RB + 32 * c + 16 * half) : 0xFFFFFF00u);
      }
      float m = on ? -INFINITY : 0.f, s = 0.f;
      f32x16 o[ND];
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

      const int32_t* table = a.tables + (int64_t)at.seg * a.max_pages;
      u32x4 kreg[NL], vreg[NL];
      int page;
      const int my_row = wid * S::RPW;
      auto find_page = [&](int j) { page = uniform(group_page(a, table, j * KT + my_row, limit)); };
      auto load = [&](int j) {
        const int r0 = j * KT + my_row, valid = min(limit - r0, S::RPW);
        const rsrc_t kr = group_rsrc(a, a.k_pages, page, r0, valid, RB);
        const rsrc_t vr = group_rsrc(a, a.v_pages, page, r0, valid, RB);
#pragma unroll
        for (int i = 0; i < NL; ++i) kreg[i] = ld128(kr, (uint32_t)(i * 1024 + lane * 16));
#pragma unroll
        for (int i = 0; i < NL; ++i) vreg[i] = ld128(vr, (uint32_t)(i * 1024 + lane * 16));
      };
      auto stage = [&](char* buf) {
        const int row = my_row + lane / S::VPR, col = (lane % S::VPR) * 16;
#pragma unroll
        for (int i = 0; i < NL; ++i) *reinterpret_cast<u32x4*>(buf + (row + i * S::RPL) * KP + col) = kreg[i];
#pragma unroll
        for (int i = 0; i < NL; ++i)
          *reinterpret_cast<u32x4*>(buf + KT * KP + (row + i * S::RPL) * VP + col) = vreg[i];
      };

      __syncthreads();  // the buffers of the tile before are done with
      find_page(j0);
      load(j0);
      find_page(j0 + 1);
      stage(lds[j0 & 1]);
      load(j0 + 1);
      find_page(j0 + 2);
      __syncthreads();
      for (int j = j0; j < j1; ++j) {
        const char* kb = lds[j & 1];
        const char* vb = kb + KT * KP;
        if (j + 1 < j1) {
          stage(lds[(j + 1) & 1]);
          load(j + 2);
          find_page(j + 3);
        }
        const int key0 = j * KT;
        if (key0 < hi) {
          f32x16 y[NK];
#pragma unroll
          for (int n = 0; n < NK; ++n) {
#pragma unroll
            for (int i = 0; i < 16; ++i) y[n][i] = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              const u32x4 kf = *reinterpret_cast<const u32x4*>(kb + (32 * n + lq) * KP + 32 * c + 16 * half);
              if constexpr (EB == 2) {
                y[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf),
                                                               __builtin_bit_cast(bf16x8, q[c]), y[n], 0, 0, 0);
              } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  y[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), __uint_as_float(q[c][e]), y[n],
                                                              0, 0, 0);
              }
            }
          }
          // lane: query row lq; register i of block n: key 32n + 8(i / 4) + 4 half + i % 4
          const bool edge = key0 + KT > lo;
          const int left = seen - key0 - 4 * half;
          float p[NK][16];
          float sum = 0.f;
          auto exps = [&]() {
            sum = 0.f;
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
              for (int i = 0; i < 16; ++i) p[n][i] = fast_exp2(fmaf(y[n][i], a.c2, -m));
            if (edge) {
#pragma unroll
              for (int n = 0; n < NK; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                  if (32 * n + 8 * (i / 4) + i % 4 >= left) p[n][i] = 0.f;
            }
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
              for (int i = 0; i < 16; ++i) sum += p[n][i];
          };
          exps();
          if (__any(!(sum <= kFar) || m == -INFINITY)) {
            float mx = -INFINITY;
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (32 * n + 8 * (i / 4) + i % 4 < left) mx = fmaxf(mx, y[n][i] * a.c2);
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float mn = fmaxf(m, mx);
            if (mn != m) {
              const float alpha = m == -INFINITY ? 1.f : fast_exp2(m - mn);
              s *= alpha;
#pragma unroll
              for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
              m = mn;
            }
            if (m == -INFINITY) {
              // nothing seen so far
              sum = 0.f;
#pragma unroll
              for (int n = 0; n < NK; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) p[n][i] = 0.f;
            } else {
              exps();
            }
          }
          s += sum;
          if constexpr (EB == 2) {
            const int g16 = lane >> 4, l16 = lane & 15;
            const char* vp = vb + (4 * half + l16 / 4) * VP + (16 * (g16 & 1) + 4 * (l16 & 3)) * 2;
#pragma unroll
            for (int t = 0; t < KT / 16; ++t) {
              const int n = t / 2, i0 = 8 * (t % 2);
              u32x4 ph, pl;
#pragma unroll
              for (int e = 0; e < 4; ++e) ph[e] = pack_bf16(p[n][i0 + 2 * e], p[n][i0 + 2 * e + 1]);
              if (FINE) {
#pragma unroll
                for (int e = 0; e < 4; ++e) pl[e] = pack_bf16_rest(p[n][i0 + 2 * e], p[n][i0 + 2 * e + 1], ph[e]);
              }
#pragma unroll
              for (int d = 0; d < ND; ++d) {
                const u32x2 v0 = lds_transposed(vp + 16 * t * VP + 64 * d);
                const u32x2 v1 = lds_transposed(vp + (16 * t + 8) * VP + 64 * d);
                const u32x4 vt = {v0.x, v0.y, v1.x, v1.y};
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vt),
                                                               __builtin_bit_cast(bf16x8, ph), o[d], 0, 0, 0);
                if (FINE)
                  o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vt),
                                                                 __builtin_bit_cast(bf16x8, pl), o[d], 0, 0, 0);
              }
            }
          } else {
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const char* vp = vb + (32 * n + 8 * (i / 4) + 4 * half + i % 4) * VP + lq * 4;
#pragma unroll
                for (int d = 0; d < ND; ++d)
                  o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(vp + 128 * d), p[n][i],
                                                              o[d], 0, 0, 0);
              }
          }
        }
        __syncthreads();
      }
      s += __shfl_xor(s, 32, 64);
      if (on) {
        const bool whole = j0 == 0 && j1 == nkt;
        if (whole) {
          const int64_t row = (int64_t)(g.t0 + tok0 + tok) * a.Hq + h * a.G + hd;
          const float inv = s == 0.f ? 0.f : 1.0f / s;
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              store_out4(a, row, D, 32 * d + 8 * i + 4 * half,
                         f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]} * inv);
          if (a.lse && half == 0) a.lse[row] = lse_of(m, s);
        } else {
          const int64_t slot = 2 * (int64_t)w + (at.start > share * w ? 1 : 0);
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<f32x4*>(a.part + (slot * M + r) * D + 32 * d + 8 * i + 4 * half) =
                  f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
          if (half == 0) {
            a.part_ms[(slot * M + r) * 2] = m;
            a.part_ms[(slot * M + r) * 2 + 1] = s;
          }
        }
      }
    }
    const int64_t next = at.start + max(limit, 1);
    if (next >= end) leave_shared(a, w, share, at, nkt);
    at.start = pos = next;
    ++at.tile;
  }
}

template <typename T, int D>
void launch_many(const PagedAttnArgs& a, hipStream_t stream) {
  if constexpr (sizeof(T) == 2) {
    if (a.out_dtype == 0) {
      paged_many_kernel<T, D, true><<<dim3(a.workers), dim3(kAttnBlock), 0, stream>>>(a);
      return;
    }
  }
  paged_many_kernel<T, D, false><<<dim3(a.workers), dim3(kAttnBlock), 0, stream>>>(a);
}

}  // namespace

hipError_t launch_paged_many(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.dtype) a.D == 128 ? launch_many<__bf16, 128>(a, stream) : launch_many<__bf16, 64>(a, stream);
  else a.D == 128 ? launch_many<float, 128>(a, stream) : launch_many<float, 64>(a, stream);
  return hipGetLastError();
}

}  // namespace sgdkv
