// Top logits and the divergence from them: kernels and C ABI.
#include <algorithm>
#include <cmath>

#include "abi.hpp"
#include "distill.hpp"
#include "top_logits.hpp"

namespace {

using saki::abi_fail;

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1u)) == 0; }

saki_status check_logits(const void* x, int32_t dtype, int64_t n_rows, int64_t vocab, int64_t stride, float temperature) {
  if (dtype != SAKI_F32 && dtype != SAKI_BF16) return abi_fail(SAKI_E_DTYPE, "unknown logits dtype");
  if (n_rows < 0) return abi_fail(SAKI_E_SHAPE, "n_rows < 0");
  if (n_rows >= (int64_t{1} << 31)) return abi_fail(SAKI_E_SHAPE, "more than 2^31 - 1 rows in one call");
  if (vocab < 1 || vocab > SAKI_MAX_VOCAB) return abi_fail(SAKI_E_SHAPE, "vocab outside [1, SAKI_MAX_VOCAB]");
  if (stride < vocab) return abi_fail(SAKI_E_SHAPE, "row_stride < vocab");
  if (!(temperature >= 0x1p-64f && temperature <= 0x1p64f))
    return abi_fail(SAKI_E_VALUE, "temperature outside [2^-64, 2^64]");
  if (n_rows == 0) return SAKI_OK;
  if (!x) return abi_fail(SAKI_E_NULLPTR, "the logits pointer is NULL");
  if (!aligned(x, 16) || (stride * (dtype == SAKI_BF16 ? 2 : 4)) % 16 != 0)
    return abi_fail(SAKI_E_ALIGN, "logits base pointer and row pitch must be 16-byte aligned");
  return SAKI_OK;
}

float log2_scale(float temperature) { return static_cast<float>(1.4426950408889634074 / static_cast<double>(temperature)); }

// Parts of a row: several, of at least TOP_PART_CHUNKS chunks, where rows are longer than TOP_LONG and so few that two parts of
// each leave CUs idle: about TOP_ITEMS workgroups.  The second launch, which joins them, costs what shorter rows would gain.
// Microseconds whole / in parts, bf16:
//   rows            1            16           64           128          255
//   65,536          17.0/19.8    18.5/20.0    19.4/21.0    19.6/21.5    19.8/26.7
//   98,304          22.0/22.8    22.4/23.1    22.7/21.7    23.8/22.5    25.4/29.0
//   151,936         27.8/25.0    32.4/27.1    32.7/23.2    37.4/27.4    36.7/34.2
//   262,144         36.1/31.4    42.5/33.5    43.6/26.1    50.0/31.1    49.6/42.4
// and f32, the rule's 8 parts at most:
//   65,536          22.3/22.7    24.2/23.6    24.7/26.1    25.6/29.0    28.7/36.1
//   98,304          24.8/24.7    27.8/25.7    28.3/28.4    32.9/32.5    33.1/42.3
//   151,936         33.1/25.7    34.0/27.1    46.1/30.9    48.0/38.0    48.8/49.2
//   262,144         44.3/27.5    53.7/30.4    64.1/36.1    63.5/46.4    68.0/66.6
// (bf16 up to 64 parts; 8 at most, which the second launch joins sooner: 151,936, 1 / 16 rows 24.5 / 27.1 -> 20.2 / 20.8, 262,144
// 27.3 / 33.4 -> 23.0 / 23.8, 1,000,000 35.7 / 38.7 -> 32.2 / 38.6)
constexpr int64_t TOP_ITEMS = 512, TOP_LONG = 98304, TOP_PART_CHUNKS = 8, TOP_MOST_PARTS = 8;
int64_t top_parts(int64_t n_rows, int64_t vocab) {
  const int64_t chunks = (vocab + SAKI_CHUNK - 1) / SAKI_CHUNK;
  if (n_rows < 1 || n_rows >= TOP_ITEMS / 2 || vocab <= TOP_LONG) return 1;
  const int64_t want = std::min({(TOP_ITEMS + n_rows - 1) / n_rows, chunks / TOP_PART_CHUNKS, TOP_MOST_PARTS});
  return want < 2 ? 1 : want;
}

// Workgroups of distill_kernel: of 512 threads, two a CU, where a row is long (read and written, over
// DISTILL_LONG bytes): then few rows are under way at a time, and the last-level cache holds more of what the second sweep
// reads again; else of 256, four a CU, whose steps between the sweeps take less (a fifth beside them: bf16 of 4,096 111.9 us
// for 110.6, of 9,000 124.5 for 120.8, of 14,000 134.9 for 139.4; f32 alike).  8,192 rows, microseconds of 512 / 256: bf16 of
// 32,000 329 / 259, of 100,000 716 / 726, f32 of 16,384 263 / 250, of 32,000 474 / 491, bf16 of 50,000 with a gradient in f32
// (a third as many rows) 161 / 214.
constexpr int64_t DISTILL_LONG = 224 << 10;

size_t round256(size_t b) { return (b + 255) & ~static_cast<size_t>(255); }

template <typename T, typename G, bool GRAD>
void launch_distill(const saki::DistillParams& P, int threads, dim3 grid, hipStream_t st) {
  if (threads == 256) hipLaunchKernelGGL((saki::distill_kernel<T, G, GRAD, 256>), grid, dim3(256), 0, st, P);
  else hipLaunchKernelGGL((saki::distill_kernel<T, G, GRAD, 512>), grid, dim3(512), 0, st, P);
}

}  // namespace

namespace saki {

size_t distill_workspace_bytes(int op, int64_t n_rows, int64_t vocab) {
  if (op == SAKI_OP_DISTILL_TOP) return 256 + round256(static_cast<size_t>(n_rows) * sizeof(double));
  if (vocab < 1) return 0;
  const int64_t parts = top_parts(n_rows, vocab);
  if (parts < 2) return 0;
  return round256(static_cast<size_t>(n_rows * parts) * (SAKI_MAX_TOP_K * sizeof(uint64_t) + sizeof(TopPart)));
}

__global__ __launch_bounds__(64) void clear_row_counter_kernel(unsigned int* counter) {
  if (threadIdx.x == 0) *counter = 0u;
}

}  // namespace saki

extern "C" {

saki_status saki_top_logits(const void* logits, int32_t dtype, int64_t n_rows, int64_t vocab, int64_t row_stride,
                            int32_t k, float temperature, float* top_logit, int32_t* top_token, int64_t top_stride,
                            float* rest_logit, uint8_t* row_status, void* ws, size_t ws_bytes, saki_stream_t stream) {
  saki_status st = check_logits(logits, dtype, n_rows, vocab, row_stride, temperature);
  if (st != SAKI_OK) return st;
  if (k < 1 || k > SAKI_MAX_TOP_K || k > vocab) return abi_fail(SAKI_E_SHAPE, "k outside [1, min(SAKI_MAX_TOP_K, vocab)]");
  if (top_stride < k) return abi_fail(SAKI_E_SHAPE, "top_stride < k");
  if (n_rows == 0) return saki::abi_ok();
  if (!top_logit || !top_token) return abi_fail(SAKI_E_NULLPTR, "top_logit and top_token are required");
  if (!aligned(top_logit, 4) || !aligned(top_token, 4) || !aligned(rest_logit, 4))
    return abi_fail(SAKI_E_ALIGN, "outputs of 4 bytes must be 4-byte aligned");
  const int64_t parts = top_parts(n_rows, vocab);
  if (parts > 1) {
    if (!ws || ws_bytes < saki_workspace_bytes(SAKI_OP_TOP_LOGITS, n_rows, vocab))
      return abi_fail(SAKI_E_WORKSPACE, "workspace NULL or smaller than saki_workspace_bytes(SAKI_OP_TOP_LOGITS)");
    if (!aligned(ws, 16)) return abi_fail(SAKI_E_ALIGN, "workspace must be 16-byte aligned");
  }
  saki::TopParams P{};
  P.x = logits;
  P.n_rows = n_rows;
  P.stride = row_stride;
  P.V = static_cast<int>(vocab);
  P.k = k;
  P.c = log2_scale(temperature);
  P.top_logit = top_logit;
  P.top_token = top_token;
  P.top_stride = top_stride;
  P.rest_logit = rest_logit;
  P.row_status = row_status;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  const bool bf16 = dtype == SAKI_BF16;
  const dim3 block(saki::TOP_NT);
  if (parts < 2) {
    // (a workgroup a row: several a workgroup that stays leave the last of them to fewer)
    const dim3 grid(static_cast<unsigned>(std::min(n_rows, int64_t{1} << 22)));
    if (bf16) hipLaunchKernelGGL((saki::top_kernel<uint16_t, saki::TOP_WHOLE>), grid, block, 0, hs, P);
    else hipLaunchKernelGGL((saki::top_kernel<float, saki::TOP_WHOLE>), grid, block, 0, hs, P);
    st = saki::abi_launched(hipGetLastError(), "top_kernel");
    return st != SAKI_OK ? st : saki::abi_ok();
  }
  P.parts = static_cast<int>(parts);
  P.info = static_cast<saki::TopPart*>(ws);
  P.keys = reinterpret_cast<uint64_t*>(P.info + n_rows * parts);
  const dim3 grid(static_cast<unsigned>(n_rows * parts)), rows(static_cast<unsigned>(n_rows));
  if (bf16) hipLaunchKernelGGL((saki::top_kernel<uint16_t, saki::TOP_PART>), grid, block, 0, hs, P);
  else hipLaunchKernelGGL((saki::top_kernel<float, saki::TOP_PART>), grid, block, 0, hs, P);
  st = saki::abi_launched(hipGetLastError(), "top_kernel");
  if (st != SAKI_OK) return st;
  if (bf16) hipLaunchKernelGGL((saki::top_kernel<uint16_t, saki::TOP_MERGE>), rows, block, 0, hs, P);
  else hipLaunchKernelGGL((saki::top_kernel<float, saki::TOP_MERGE>), rows, block, 0, hs, P);
  st = saki::abi_launched(hipGetLastError(), "top_kernel");
  return st != SAKI_OK ? st : saki::abi_ok();
}

saki_status saki_distill_top(const void* student, int32_t dtype, int64_t n_rows, int64_t vocab, int64_t row_stride,
                             const saki_top_list* list, float temperature, int32_t direction, const uint8_t* valid_mask,
                             float grad_scale, float* row_loss, double* loss_sum, void* grad, int32_t grad_dtype,
                             int64_t grad_stride, uint8_t* row_status, void* ws, size_t ws_bytes, saki_stream_t stream) {
  saki_status st = check_logits(student, dtype, n_rows, vocab, row_stride, temperature);
  if (st != SAKI_OK) return st;
  if (!list) return abi_fail(SAKI_E_NULLPTR, "list is NULL");
  if (list->reserved != 0) return abi_fail(SAKI_E_VALUE, "saki_top_list.reserved must be 0");
  if (list->k < 1 || list->k > SAKI_MAX_TOP_K) return abi_fail(SAKI_E_SHAPE, "k outside [1, SAKI_MAX_TOP_K]");
  if (list->stride < list->k) return abi_fail(SAKI_E_SHAPE, "the list's stride < k");
  if (direction != SAKI_KL_FORWARD && direction != SAKI_KL_REVERSE) return abi_fail(SAKI_E_VALUE, "unknown direction");
  if (!std::isfinite(grad_scale)) return abi_fail(SAKI_E_VALUE, "grad_scale is not finite");
  if (grad) {
    if (grad_dtype != SAKI_F32 && grad_dtype != SAKI_BF16) return abi_fail(SAKI_E_DTYPE, "unknown grad dtype");
    if (grad_stride < vocab) return abi_fail(SAKI_E_SHAPE, "grad_stride < vocab");
    if (!aligned(grad, 16) || (grad_stride * (grad_dtype == SAKI_BF16 ? 2 : 4)) % 16 != 0)
      return abi_fail(SAKI_E_ALIGN, "grad base pointer and row pitch must be 16-byte aligned");
    if (grad == student && (grad_dtype != dtype || grad_stride != row_stride))
      return abi_fail(SAKI_E_VALUE, "a gradient in the student's buffer has its dtype and stride");
  }
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (!aligned(loss_sum, 8)) return abi_fail(SAKI_E_ALIGN, "loss_sum must be 8-byte aligned");
  if (n_rows == 0) {  // the sum over no rows
    if (!loss_sum) return saki::abi_ok();
    st = saki::abi_loss_sum(nullptr, 0, loss_sum, hs);
    return st != SAKI_OK ? st : saki::abi_ok();
  }
  if (!list->token || !list->logit) return abi_fail(SAKI_E_NULLPTR, "the list's token and logit are required");
  if (direction == SAKI_KL_REVERSE && !list->rest_logit)
    return abi_fail(SAKI_E_NULLPTR, "the reverse divergence needs rest_logit");
  if (!aligned(list->token, 4) || !aligned(list->logit, 4) || !aligned(list->rest_logit, 4) || !aligned(row_loss, 4))
    return abi_fail(SAKI_E_ALIGN, "an array of 4 bytes an entry is not 4-byte aligned");
  if (!ws || ws_bytes < saki_workspace_bytes(SAKI_OP_DISTILL_TOP, n_rows, vocab))
    return abi_fail(SAKI_E_WORKSPACE, "workspace NULL or smaller than saki_workspace_bytes(SAKI_OP_DISTILL_TOP)");
  if (!aligned(ws, 8)) return abi_fail(SAKI_E_ALIGN, "workspace must be 8-byte aligned");
  int cus = 0;
  st = saki::abi_cus(&cus);
  if (st != SAKI_OK) return st;
  saki::DistillParams P{};
  P.s = student;
  P.n_rows = n_rows;
  P.stride = row_stride;
  P.V = static_cast<int>(vocab);
  P.k = list->k;
  P.token = list->token;
  P.logit = list->logit;
  P.rest = list->rest_logit;
  P.list_stride = list->stride;
  P.c = log2_scale(temperature);
  P.inv_tau = 1.0f / temperature;
  P.reverse = direction == SAKI_KL_REVERSE;
  P.valid = valid_mask;
  P.grad_scale = grad_scale;
  P.row_loss = row_loss;
  double* const scaled = reinterpret_cast<double*>(static_cast<char*>(ws) + 256);
  P.scaled_loss = loss_sum ? scaled : nullptr;
  P.grad = grad;
  P.grad_stride = grad_stride;
  P.row_status = row_status;
  const bool bf16 = dtype == SAKI_BF16;
  const int64_t row_bytes = vocab * ((bf16 ? 2 : 4) + (!grad ? 0 : grad_dtype == SAKI_BF16 ? 2 : 4));
  const int threads = row_bytes <= DISTILL_LONG && list->k < 256 ? 256 : 512;  // (a thread for each token, and one for the others)
  const int64_t slots = static_cast<int64_t>(cus) * (threads == 512 ? 2 : 4);
  const dim3 grid(static_cast<unsigned>(std::min(n_rows, slots)));
  if (n_rows > slots) {
    P.next_row = static_cast<unsigned int*>(ws);
    hipLaunchKernelGGL(saki::clear_row_counter_kernel, dim3(1), dim3(64), 0, hs, P.next_row);
    st = saki::abi_launched(hipGetLastError(), "clear_row_counter_kernel");
    if (st != SAKI_OK) return st;
  }
  const bool gbf = grad_dtype == SAKI_BF16;
  if (bf16)
    !grad ? launch_distill<uint16_t, float, false>(P, threads, grid, hs)
    : gbf ? launch_distill<uint16_t, uint16_t, true>(P, threads, grid, hs)
          : launch_distill<uint16_t, float, true>(P, threads, grid, hs);
  else
    !grad ? launch_distill<float, float, false>(P, threads, grid, hs)
    : gbf ? launch_distill<float, uint16_t, true>(P, threads, grid, hs)
          : launch_distill<float, float, true>(P, threads, grid, hs);
  st = saki::abi_launched(hipGetLastError(), "distill_kernel");
  if (st != SAKI_OK) return st;
  if (loss_sum) {
    st = saki::abi_loss_sum(scaled, n_rows, loss_sum, hs);
    if (st != SAKI_OK) return st;
  }
  return saki::abi_ok();
}

}  // extern "C"
