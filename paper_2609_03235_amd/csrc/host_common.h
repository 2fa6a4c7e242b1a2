// Error reporting and the device check of the C-ABI layer, shared by its source files.
#pragma once

#include "sgdkv.h"

namespace sgdkv {
// Sets sgdkv_last_error and returns code; clears it and returns SGDKV_OK.
sgdkv_status host_fail(sgdkv_status code, const char* message);
sgdkv_status host_ok();
// The current device is a gfx950 one; cus_out (optional) receives its compute units.
sgdkv_status host_check_device(int* cus_out);
}  // namespace sgdkv
