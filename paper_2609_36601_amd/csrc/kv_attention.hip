// One part of the attention kernels' instantiations: SAKI_PART 0-2 bf16, 3-5 f32, heads of
// up to 64, 128 and 256 elements.
#include "kv_attention.hpp"

namespace saki {

namespace {

template <typename T, int DP, int ROWS>
hipError_t launch(void (*kernel)(KvAttnParams), const KvAttnParams& P, int64_t units, bool join, hipStream_t st) {
  constexpr int64_t ITEMS = KV_ITEMS<T, DP, ROWS>;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(units + ITEMS)), dim3(KV_ATT_NT), 0, st, P);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !join) return e;
  // one row a workgroup where few units can be split, else four; at most so many
  // workgroups as the card takes at once
  const int64_t rows = (units < ITEMS ? units : ITEMS) * ROWS;
  if (rows <= 4096)
    hipLaunchKernelGGL((kv_join_kernel<T, DP, ROWS, 1>), dim3(static_cast<unsigned>(rows)), dim3(KV_ATT_NT), 0, st, P);
  else
    hipLaunchKernelGGL((kv_join_kernel<T, DP, ROWS, 4>), dim3(8 * KV_CUS), dim3(KV_ATT_NT), 0, st, P);
  return hipGetLastError();
}

}  // namespace

using PartT = std::conditional<(SAKI_PART < 3), uint16_t, float>::type;
constexpr int PART_DP = 64 << (SAKI_PART % 3);

template <>
hipError_t launch_kv_attention<PartT, PART_DP>(const KvAttnParams& P, int row_tiles, int64_t units, bool join,
                                               hipStream_t st) {
  constexpr int MOST = kv_row_tiles<PartT>(PART_DP);
  if constexpr (sizeof(PartT) == 2 && PART_DP <= 128)
    if (row_tiles == 8)
      return launch<PartT, PART_DP, KV_PROMPT_ROWS>(
          P.p.dim == PART_DP ? kv_prompt_kernel<PART_DP, true> : kv_prompt_kernel<PART_DP, false>, P, units, join, st);
  if constexpr (MOST >= 4)
    if (row_tiles == 4) return launch<PartT, PART_DP, 64>(kv_attention_kernel<PartT, PART_DP, 4>, P, units, join, st);
  if constexpr (MOST >= 2)
    if (row_tiles == 2) return launch<PartT, PART_DP, 32>(kv_attention_kernel<PartT, PART_DP, 2>, P, units, join, st);
  return launch<PartT, PART_DP, 16>(kv_attention_kernel<PartT, PART_DP, 1>, P, units, join, st);
}

}  // namespace saki
