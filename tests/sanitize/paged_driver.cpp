// Drives the paged cache's host entry points under the sanitizers: sizes at and past their limits, every
// refusal, and well-formed calls, which end at the device check. The launchers are stand-ins.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <initializer_list>

#include "paged_internal.h"
#include "sgdkv.h"

namespace sgdkv {
hipError_t launch_page_update(const PageArgs&, int, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_paged_store(const PagedStoreArgs&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_norm_rope(const NormRopeArgs&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_paged_attention(const PagedAttnArgs&, hipStream_t) { return hipErrorNoDevice; }
PagedAttnShape paged_attn_shape(int dtype, int G, int max_new) {
  return (int64_t)max_new * G <= 48 ? PagedAttnShape{48, 128} : PagedAttnShape{128, dtype ? 64 : 32};
}
}  // namespace sgdkv

namespace {
int failures = 0;
void expect(sgdkv_status got, std::initializer_list<sgdkv_status> want, const char* what, long long value) {
  for (sgdkv_status w : want)
    if (got == w) return;
  std::printf("%s = %lld: status %d (%s)\n", what, value, got, sgdkv_last_error());
  ++failures;
}
int32_t* at(uintptr_t x) { return reinterpret_cast<int32_t*>(x); }
}  // namespace

int main() {
  const int64_t extremes[] = {INT32_MIN, -1, 0, 1, 2, 15, 16, 17, 64, 96, 128, 1024, 4096, 65535, 65536, INT32_MAX};
  int32_t* const p = at(1 << 20);
  const std::initializer_list<sgdkv_status> any = {SGDKV_ERR_INVALID_ARG, SGDKV_ERR_UNSUPPORTED, SGDKV_ERR_WORKSPACE,
                                                   SGDKV_ERR_HIP};
  for (int64_t x : extremes)
    for (int64_t y : extremes) {
      const int32_t a = (int32_t)x, b = (int32_t)y;
      for (int64_t wide : {x, x * y, x * 4294967296}) {
        const sgdkv_page_desc pd[] = {{a, b, 16, 8, 0, 0, 50, 4}, {2, 2, a, b, 1, 0, 50, 4}, {2, 2, 16, 8, a, b, 50, 4},
                                      {2, 2, 16, a, 0, 0, wide, y}, {2, b, 16, 8, 0, 0, y, wide}};
        for (const auto& d : pd)
          expect(sgdkv_page_update(&d, p, p, p, p, p, p, p, p, p, p, nullptr), any, "page_update", wide);
        const sgdkv_page_pool pools[] = {{p, p, wide, 16, 128, 1, 0}, {p, p, 10, a, b, 0, 0},
                                         {p, p, wide, a, 64, b, 0}};
        for (const auto& pool : pools) {
          expect(sgdkv_paged_store(&pool, p, p, p, wide, nullptr), any, "paged_store", wide);
          const sgdkv_norm_rope_desc nd[] = {{wide, a, b, 512, 256, 256, 64, 0, 1e-6f, 0},
                                             {3, 4, 2, wide, y, x, b, 0, 1e-6f, 0},
                                             {3, 4, 2, 512, 256, 256, a, b, 0.f, 0}};
          for (const auto& d : nd)
            expect(sgdkv_norm_rope_store(&pool, &d, p, p, p, p, p, reinterpret_cast<float*>(p), p, p, at(1 << 21),
                                         nullptr),
                   any, "norm_rope_store", wide);
          const sgdkv_paged_desc ad[] = {{a, b, 2, 0, 6, 4, 8, 1, 0.f}, {a, 8, b, 1, 6, 4, 8, 1, 0.f},
                                         {2, 8, 2, 0, wide, a, b, 0, 1.f}, {2, 8, 2, a, 6, b, 8, 1, 0.f}};
          for (const auto& d : ad) {
            size_t n = 0;
            expect(sgdkv_paged_attention_workspace_size(&pool, &d, &n),
                   {SGDKV_OK, SGDKV_ERR_INVALID_ARG, SGDKV_ERR_UNSUPPORTED}, "workspace", wide);
            expect(sgdkv_paged_attention(&pool, &d, p, p, p, p, p, reinterpret_cast<float*>(p), p, n, nullptr), any,
                   "paged_attention", wide);
          }
        }
      }
    }
  expect(sgdkv_page_update(nullptr, p, p, p, p, p, p, p, p, p, p, nullptr), {SGDKV_ERR_INVALID_ARG}, "NULL", 0);
  if (std::strlen(sgdkv_last_error()) == 0) ++failures;
  std::printf(failures ? "%d failures\n" : "SANITIZE PASS\n", failures);
  return failures != 0;
}
