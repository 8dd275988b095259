// One part of the attention kernels' instantiations: SAKI_PART 0-2 bf16, 3-5 f32, heads of
// up to 64, 128 and 256 elements.
#include "kv_attention.hpp"

namespace saki {

namespace {

template <typename T, int DP, int R>
hipError_t launch(const KvAttnParams& P, int64_t units, bool join, hipStream_t st) {
  const unsigned grid = static_cast<unsigned>(units + P.items);
  hipLaunchKernelGGL((kv_attention_kernel<T, DP, R>), dim3(grid), dim3(KV_ATT_NT), 0, st, P);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !join) return e;
  const unsigned split_units = static_cast<unsigned>(units < P.items ? units : P.items);
  // one row a workgroup where that fills the card but little more, else four
  if (split_units * 16 * R <= 4096)
    hipLaunchKernelGGL((kv_join_kernel<T, DP, R, 1>), dim3(split_units * 16 * R), dim3(KV_ATT_NT), 0, st, P);
  else
    hipLaunchKernelGGL((kv_join_kernel<T, DP, R, 4>), dim3(split_units * 4 * R), dim3(KV_ATT_NT), 0, st, P);
  return hipGetLastError();
}

}  // namespace

using PartT = std::conditional<(SAKI_PART < 3), uint16_t, float>::type;
constexpr int PART_DP = 64 << (SAKI_PART % 3);

template <>
hipError_t launch_kv_attention<PartT, PART_DP>(const KvAttnParams& P, int row_tiles, int64_t units, bool join,
                                               hipStream_t st) {
  constexpr int MOST = kv_row_tiles<PartT>(PART_DP);
  if constexpr (MOST >= 4)
    if (row_tiles == 4) return launch<PartT, PART_DP, 4>(P, units, join, st);
  if constexpr (MOST >= 2)
    if (row_tiles == 2) return launch<PartT, PART_DP, 2>(P, units, join, st);
  return launch<PartT, PART_DP, 1>(P, units, join, st);
}

}  // namespace saki
