// The kernels of the paged caches in 8 bits (tdk_kv_pages.h has their bodies; tdk_rope.hip the append).
#include "tdk_kv_pages.h"

namespace tdk {

template <bool ONCE>
__global__ __launch_bounds__(64) void tdk_kv8_read_kernel(const KvDev kv, const KvRowsDev rows) {
  read_rows<kMx8, ONCE>(kv, rows);
}

template <int NR>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void tdk_kv8_attend_rows_kernel(const KvDev kv, const KvAttendDev at) {
  attend_rows<kMx8, NR>(kv, at);
}

__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void tdk_kv8_attend_tile_kernel(const KvDev kv, const KvAttendDev at,
                                                                                                             const int last_id) {
  attend_steps<kMx8>(kv, at, last_id);
}

hipError_t launch_kv8_read(const KvDev& kv, const KvRowsDev& rows, bool many, hipStream_t st) {
  return launch(many ? tdk_kv8_read_kernel<true> : tdk_kv8_read_kernel<false>, (int64_t)kv.n_tokens * rows.waves, 64, st, kv, rows);
}

hipError_t launch_kv8_attend(const KvDev& kv, const KvAttendDev& at, const KvAttendPlan& p, int64_t blocks, hipStream_t st) {
  if (p.block_rows == 128) return launch(tdk_kv8_attend_tile_kernel, blocks, 256, st, kv, at, p.forward ? -1 : (int)(p.ids - 1));
  return launch(p.block_rows == 32 ? tdk_kv8_attend_rows_kernel<2> : tdk_kv8_attend_rows_kernel<1>, blocks, 256, st, kv, at);
}

}  // namespace tdk
