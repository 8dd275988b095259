// What the units that hold entry points of the C ABI share: the calling thread's
// last error (kept in saki.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/saki_kv.h"

namespace saki {

saki_status abi_fail(saki_status st, const char* msg);
saki_status abi_ok();
saki_status abi_launched(hipError_t e, const char* kernel);
saki_status abi_cus(int* cus);
size_t kv_workspace_bytes(int op, int64_t n, int64_t m);  // kv_cache.hip

}  // namespace saki
