// Calls the launcher of many rows over an 8-bit pool, below the entry points' checks, with what no instance of it
// takes: queries in fp32 of 128 columns. It has to refuse them before any launch.
#include <cstdio>

#include "paged_internal.h"

namespace sgdkv {
hipError_t launch_paged_many_fp8(const PagedAttnArgs& a, hipStream_t stream);
}

int main() {
  int bad = 0;
  // such queries are given other tiles
  for (int group = 1; group <= sgdkv::kMaxPagedGroup; ++group)
    for (int max_new : {1, 3, 48, 49, 1000, 1 << 27})
      bad += sgdkv::paged_attn_fp8_shape_128(0, group, max_new).rows >= 128;
  sgdkv::PagedAttnArgs a{};
  a.D = 128;
  a.dtype = 0;
  a.tile_rows = 128;
  const hipError_t e = sgdkv::launch_paged_many_fp8(a, nullptr);
  if (e != hipErrorInvalidValue) ++bad;
  std::printf(bad ? "%d failures, status %d\n" : "REFUSED\n", bad, (int)e);
  return bad != 0;
}
