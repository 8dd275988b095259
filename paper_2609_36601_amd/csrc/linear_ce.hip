// Cross entropy from hidden states.  SAKI_PART 0 .. 3: the product of that CeKind; 4: the other kernels
// and the C ABI.
#include "linear_ce.hpp"

#if SAKI_PART < 4

namespace saki {

template <int KIND, typename TILE>
static hipError_t launch_tile(CeGemm A, bool three, int splits, hipStream_t st) {
  A.p_tiles = (A.n_p + TILE::PT - 1) / TILE::PT;
  A.q_tiles = (A.n_q + TILE::QT - 1) / TILE::QT;
  // (a launch of more threads is cut off without an error; see Plan::s_step)
  if (static_cast<int64_t>(A.p_tiles) * A.q_tiles * splits * TILE::NT > CE_MOST_THREADS) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<unsigned>(A.p_tiles * A.q_tiles * splits)), block(TILE::NT);
  if constexpr (std::is_same_v<TILE, CeFew> && (KIND == CE_LSE || KIND == CE_DL)) {  // (f32: ce_direct_kernel)
    if (three) return hipErrorInvalidValue;
  } else if (three) {
    hipLaunchKernelGGL((ce_gemm_kernel<KIND, TILE, true>), grid, block, 0, st, A);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((ce_gemm_kernel<KIND, TILE, false>), grid, block, 0, st, A);
  return hipGetLastError();
}

template <>
hipError_t launch_ce_part<SAKI_PART>(const CeGemm& A, int tile, bool three, int splits, hipStream_t st) {
  if constexpr (SAKI_PART != CE_DW) {
    if (tile == CE_DIRECT) {
      CeGemm B = A;
      B.p_tiles = (A.n_p + CeDirect::PT - 1) / CeDirect::PT;
      B.q_tiles = (A.n_q + CeDirect::QT - 1) / CeDirect::QT;
      hipLaunchKernelGGL((ce_direct_kernel<SAKI_PART>), dim3(static_cast<unsigned>(B.p_tiles * B.q_tiles * splits)),
                         dim3(CeDirect::NT), 0, st, B);
      return hipGetLastError();
    }
  }
  if (tile == CE_LARGE) return launch_tile<SAKI_PART, CeLarge>(A, three, splits, st);
  if (tile == CE_MIDDLE) return launch_tile<SAKI_PART, CeMiddle>(A, three, splits, st);
  return launch_tile<SAKI_PART, CeFew>(A, three, splits, st);
}

}  // namespace saki

#else

#include <algorithm>
#include <cmath>

#include "abi.hpp"

namespace saki {

template <>
hipError_t launch_ce_part<CE_LSE>(const CeGemm&, int, bool, int, hipStream_t);
template <>
hipError_t launch_ce_part<CE_DL>(const CeGemm&, int, bool, int, hipStream_t);
template <>
hipError_t launch_ce_part<CE_DX>(const CeGemm&, int, bool, int, hipStream_t);
template <>
hipError_t launch_ce_part<CE_DW>(const CeGemm&, int, bool, int, hipStream_t);

// The rows that take part, in order, and the outputs of those that do not.  One workgroup: a scan
// over 1,024 rows at a time.
__global__ __launch_bounds__(1024) void ce_rows_kernel(CeRows P) {
  __shared__ int before[1024 / WAVE];
  const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE;
  int base = 0;
  for (int64_t r0 = 0; r0 < P.n_rows; r0 += 1024) {
    const int64_t r = r0 + threadIdx.x;
    const bool in = r < P.n_rows && P.valid[r] != 0;
    const uint64_t who = __ballot(in);
    if (lane == 0) before[wave] = __popcll(who);
    __syncthreads();
    int at = base, all = base;
    for (int w = 0; w < 1024 / WAVE; ++w) {
      at += w < wave ? before[w] : 0;
      all += before[w];
    }
    at += __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(who >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(who), 0));
    if (in) P.source[at] = static_cast<int>(r);
    if (r < P.n_rows) {
      P.place[r] = in ? at : -1;
      if (!in) {
        if (P.row_loss) P.row_loss[r] = 0.0f;
        if (P.logp_token) P.logp_token[r] = 0.0f;
        if (P.scaled_loss) P.scaled_loss[r] = 0.0;
        if (P.row_status) P.row_status[r] = SAKI_ROW_OK;
      }
    }
    base = all;
    __syncthreads();
  }
  if (threadIdx.x == 0) *P.count = base;
}

// A workgroup a row that takes part: its log-sum-exp from the tiles' maxima and sums, and the row's outputs.  With u the other
// tokens' sum relative to the token's exponential, log p = -log(1 + u) and 1 - p = u / (1 + u): both relatively exact where u is
// small.  What bounds it: latency; every thread has four of its row's loads under way.
__global__ __launch_bounds__(256) void ce_loss_kernel(CeRows P) {
  constexpr int DEEP = 4;
  __shared__ float part_m[4];
  __shared__ double part_s[4];
  const int tid = threadIdx.x, lane = tid & (WAVE - 1), wave = tid / WAVE;
  const int64_t i = blockIdx.x;
  if (P.count && i >= *P.count) return;
  const int64_t r = P.count ? P.source[i] : i;
  const int token = P.token[r];
  const float weight = P.row_weight ? P.row_weight[r] : 1.0f;
  const bool good = token >= 0 && token < P.vocab && isfinite(weight);
  const float target = good ? P.target[i] : 0.0f;
  const float2* stats = P.stats + i * P.slots;
  float m = -finf();
  double sum = 0.0;
  for (int s0 = tid; s0 < P.slots; s0 += 256 * DEEP) {
    float2 f[DEEP];
#pragma unroll
    for (int e = 0; e < DEEP; ++e) f[e] = stats[min(s0 + e * 256, P.slots - 1)];
    float to = m;
#pragma unroll
    for (int e = 0; e < DEEP; ++e) to = fmaxf(to, f[e].x);
    // (-infinity and 0: no token, or logits of -infinity or NaN alone, whose sum is NaN)
    sum = m == -finf() ? sum : sum * static_cast<double>(fexp2(m - to));
    m = to;
    const float ref = m == -finf() ? 0.0f : m;
#pragma unroll
    for (int e = 0; e < DEEP; ++e)
      if (s0 + e * 256 < P.slots) sum += static_cast<double>(f[e].y) * static_cast<double>(fexp2(f[e].x - ref));
  }
  const float wm = wave_max(m);
  sum = m == -finf() ? sum : sum * static_cast<double>(fexp2(m - wm));
#pragma unroll
  for (int k = 1; k < WAVE; k *= 2) sum += __shfl_xor(sum, k);
  if (lane == 0) {
    part_m[wave] = wm;
    part_s[wave] = sum;
  }
  __syncthreads();
  if (tid != 0) return;
  m = fmaxf(fmaxf(part_m[0], part_m[1]), fmaxf(part_m[2], part_m[3]));
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < 4; ++w) sum += part_m[w] == -finf() ? part_s[w] : part_s[w] * static_cast<double>(fexp2(part_m[w] - m));
  // (a row of -infinity alone: m and so the result; a token's logit that is not finite: NaN, or log p)
  const double own = good ? exp2(static_cast<double>(target) - static_cast<double>(m)) : 0.0, all = own + sum;
  const double lse2 = static_cast<double>(m) + log2(all);
  const double logp = own >= 0.25 ? -log1p(sum / own) / (LN2_D * static_cast<double>(LOG2E))
                                  : (static_cast<double>(target) - lse2) / static_cast<double>(LOG2E);
  const bool finite = isfinite(lse2) && (!good || isfinite(logp));
  CeRow R;
  R.lse_hi = finite ? static_cast<float>(lse2) : nanf_();
  R.lse_lo = finite ? static_cast<float>(lse2 - static_cast<double>(R.lse_hi)) : nanf_();
  R.weight = good ? weight : 0.0f;
  R.token = good ? token : -1;
  R.rest = finite ? static_cast<float>(sum / all) : nanf_();
  P.rows[i] = R;
  const bool ok = good && finite;
  const double loss = ok ? -static_cast<double>(weight) * logp : __builtin_nan("");
  if (P.row_loss) P.row_loss[r] = static_cast<float>(loss);
  if (P.logp_token) P.logp_token[r] = ok ? static_cast<float>(logp) : nanf_();
  if (P.scaled_loss) P.scaled_loss[r] = static_cast<double>(P.grad_scale) * loss;
  if (P.row_status) P.row_status[r] = !good ? SAKI_ROW_BAD_TARGET : finite ? SAKI_ROW_OK : SAKI_ROW_NONFINITE;
}

// The gradient of a weight to which no row adds anything.
template <typename T>
__global__ __launch_bounds__(256) void ce_zero_kernel(T* grad, int64_t stride, int64_t vocab, int D) {
  const int pieces = D / 8;
  float g[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) g[e] = 0.0f;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < vocab * pieces; i += gridDim.x * 256ll)
    Storer<T>::store8(grad + i / pieces * stride + i % pieces * 8, g);
}

}  // namespace saki

namespace {

using namespace saki;

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1u)) == 0; }
int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int64_t MOST_STRIDE = int64_t{1} << 22;
constexpr int64_t MOST_ROWS = (int64_t{1} << 31) / 256;
// Bytes of the gradient of a piece's logits, and of a piece of the weight in three parts: what the
// last-level cache holds, at most (its pieces cost each product a start and an end).
constexpr int64_t PIECE_BYTES = int64_t{256} << 20;
// Bytes of logits that a training call keeps, at most; above it, it computes them a second time, in pieces.  Loss and gradients
// in microseconds, kept / again (bf16 but for the one in f32):
//   rows             16         64         200          400          1,024
//   32,000 x 512     49/53      54/57      77/79        111/115      169/177
//   50,000 x 2,048   189/222    204/234    293/329      408/474      719/848
//   151,936 x 4,096  1.05k/1.25k 1.13k/1.34k 1.39k/1.69k  1.98k/2.43k  f32: 50,000 x 2,048 3.79k/5.01k
constexpr int64_t KEEP_BYTES = int64_t{1} << 30;
constexpr int64_t CUS = 256;
constexpr int64_t MOST_SPLITS = 64;
// f32: up to so many rows the weight is read as it is, above them it is written as three parts first.  Loss and gradients in
// microseconds, as it is / in parts:
//   rows             16          128          512          768         1,024        2,048
//   4,000 x 1,024                          145/217      204/247      243/274      439/411
//   32,000 x 1,024   139/301     234/391   825/833    1,227/1,172  1,621/1,387  3,336/2,834
//   50,000 x 2,048   468/1,279   748/1,865 2,597/3,173  3,827/4,076  5,072/5,202 10,002/9,009
//   151,936 x 4,096  2.4k/7.7k   4.2k/14k   15k/20k     23k/23k      30k/34k      59k/58k
constexpr int64_t DIRECT_ROWS = 768;

saki_status check_head(const saki_head* h) {
  if (!h) return abi_fail(SAKI_E_NULLPTR, "head is NULL");
  if (h->dtype != SAKI_F32 && h->dtype != SAKI_BF16) return abi_fail(SAKI_E_DTYPE, "unknown dtype of the head");
  if (h->reserved != 0) return abi_fail(SAKI_E_VALUE, "saki_head.reserved must be 0");
  if (h->n_rows < 0 || h->n_rows >= MOST_ROWS) return abi_fail(SAKI_E_SHAPE, "n_rows outside [0, 2^31 / 256)");
  if (h->vocab < 1 || h->vocab > SAKI_MAX_VOCAB) return abi_fail(SAKI_E_SHAPE, "vocab outside [1, SAKI_MAX_VOCAB]");
  if (h->hidden_size < 8 || h->hidden_size > SAKI_MAX_HIDDEN || h->hidden_size % 8 != 0)
    return abi_fail(SAKI_E_SHAPE, "hidden_size is not a multiple of 8 in [8, SAKI_MAX_HIDDEN]");
  if (h->hidden_stride < h->hidden_size || h->weight_stride < h->hidden_size || h->hidden_stride >= MOST_STRIDE ||
      h->weight_stride >= MOST_STRIDE)
    return abi_fail(SAKI_E_SHAPE, "a row stride outside [hidden_size, 2^22)");
  return SAKI_OK;
}

// Tiles of a product of n_p x n_q entries: the large ones where there is one for each CU, the middle ones below that, and
// where there are few rows (their side is q) those that read the weight with the least beside it.  Loss and dW in
// microseconds, dW in large / middle / small tiles: 32,000 x 1,024, 200 rows 64/66/103, 3,200 rows 573/613/818;
// 151,936 x 4,096, 64 rows 734/723/1,204, 800 rows 2,257/2,352/3,542.
int tile_of(int64_t n_p, int64_t n_q, bool rows_q) {
  if (rows_q && n_q <= CeFew::QT) return CE_FEW;
  return ceil_div(n_p, CeLarge::PT) * ceil_div(n_q, CeLarge::QT) >= CUS ? CE_LARGE : CE_MIDDLE;
}

// A product whose k may be split between workgroups, whose sums are added up afterwards: the tile, from `first` on, and the
// splits that cost least, in microseconds.  A CU takes STEP for a tile of k (of two workgroups, where two fit), rounds
// that leave CUs idle cost like others, starting and ending a tile takes 3, and a split's sums are written and read.
void split_product(int64_t n_q, int64_t n_p, int64_t kt, bool three, int first, int* tile, int64_t* k_split, int64_t* splits) {
  double least = -1.0;
  for (int t = first; t <= std::max<int>(first, CE_FEW); ++t) {
    const int64_t side = t == CE_LARGE ? CeLarge::QT : t == CE_MIDDLE ? CeMiddle::QT : CeFew::QT, per_cu = t == CE_LARGE ? 1 : 2;
    const double step = (t == CE_LARGE ? 1.7 : t == CE_MIDDLE ? 1.1 : t == CE_FEW ? 0.6 : 1.5) * (three ? 6.0 : 1.0);
    const int64_t tiles = ceil_div(n_q, side) * ceil_div(n_p, side);
    for (int64_t s = 1; s <= std::min<int64_t>(MOST_SPLITS, std::max<int64_t>(kt / 4, 1)); ++s) {
      const double rounds = static_cast<double>(ceil_div(tiles * s, per_cu * CUS));
      const double cost = rounds * (3.0 + static_cast<double>(ceil_div(kt, s)) * step) + static_cast<double>(s) * n_q * n_p * 8 / 4.5e6;
      if (least < 0.0 || cost < least) {
        least = cost;
        *tile = t;
        *splits = s;
      }
    }
  }
  *k_split = ceil_div(kt, *splits);
  *splits = std::max<int64_t>(ceil_div(kt, *k_split), 1);
}

// The workspace of a call, and its pieces.
struct Plan {
  int64_t n, V, D, ld;       // ld: elements of a packed row, whole tiles of k
  int64_t rows;              // n, padded to tiles
  int planes;
  int64_t slots, wave_p, piece, pieces;     // wave_p: tokens of a slot
  int64_t s_step;            // tokens of a launch of the loss's product, at most: its threads are fewer than 2^32
  int64_t splits, k_split, w_splits, w_split;  // of dX's and dW's k, and tiles of k of each
  bool direct;               // f32 weights as they are (ce_direct_kernel)
  int tile_s, tile_l, tile_x, tile_w;  // tiles of the products for the loss, for dL, dX and dW
  bool keep;                 // the logits, between the loss and dL
  size_t count, source, place, row, scaled, target, stats, x, w, dl, logits, sums, w_sums, bytes;
};

Plan plan_of(const saki_head* h, bool dx, bool dw) {
  Plan p{};
  p.n = h->n_rows;
  p.V = h->vocab;
  p.D = h->hidden_size;
  p.ld = round_up(p.D, CE_BK);
  p.rows = round_up(p.n, CE_PAD);
  const bool three = h->dtype == SAKI_F32;
  p.planes = three ? 3 : 1;
  p.direct = three && p.n <= DIRECT_ROWS;
  // pieces of the vocabulary, of equal size
  const int64_t padded = round_up(p.V, CE_PAD);
  int64_t most = padded;
  if (dx || dw) most = std::min(most, PIECE_BYTES / (p.rows * 2 * p.planes));
  if (three && !p.direct) most = std::min(most, PIECE_BYTES / (p.ld * 2 * p.planes));
  most = std::max<int64_t>(most / CE_PAD * CE_PAD, CE_PAD);
  p.pieces = ceil_div(padded, most);
  p.piece = round_up(ceil_div(padded, p.pieces), CE_PAD);
  p.pieces = ceil_div(padded, p.piece);
  p.tile_l = p.direct ? CE_DIRECT : tile_of(p.piece, p.n, true);
  p.tile_s = three ? p.tile_l : tile_of(p.V, p.n, true);
  const int64_t tile_p = p.tile_s == CE_LARGE ? CeLarge::PT : p.tile_s == CE_MIDDLE ? CeMiddle::PT : CeFew::PT;
  p.wave_p = tile_p / (p.tile_s == CE_LARGE ? CeLarge::WP : p.tile_s == CE_MIDDLE ? CeMiddle::WP : CeFew::WP);
  static_assert(CeDirect::PT == CeFew::PT && CeDirect::WP == CeFew::WP, "slots alike");
  p.slots = ceil_div(p.V, tile_p) * (tile_p / p.wave_p);
  // The other products stay below it: dL's tiles by its piece's size, the gradients' by what memory holds of their sums.
  const int64_t side_q = p.tile_s == CE_LARGE ? CeLarge::QT : p.tile_s == CE_MIDDLE ? CeMiddle::QT : CeFew::QT;
  const int64_t column = ceil_div(p.n, side_q) * (p.tile_s == CE_LARGE ? CeLarge::NT : CeFew::NT);
  static_assert(CeMiddle::NT == CeFew::NT && CeDirect::NT == CeFew::NT && CeDirect::QT == CeFew::QT, "threads alike");
  static_assert(MOST_ROWS / CeLarge::QT * CeLarge::NT * (CE_PAD / CeLarge::PT) < CE_MOST_THREADS, "a launch takes CE_PAD tokens");
  p.s_step = CE_MOST_THREADS / column * tile_p / CE_PAD * CE_PAD;
  // dX's k are the piece's tokens; dW's, where the piece is the whole vocabulary (which may be small), the rows
  const int64_t kt = p.piece / CE_BK;
  p.tile_x = p.direct ? CE_DIRECT : p.n <= CeFew::QT ? CE_FEW : CE_LARGE;
  split_product(p.n, p.D, kt, three && !p.direct, p.tile_x, &p.tile_x, &p.k_split, &p.splits);
  p.tile_w = tile_of(p.D, p.piece, false);
  p.w_split = ceil_div(p.n, CE_BK);
  p.w_splits = 1;
  if (p.pieces == 1) split_product(p.V, p.D, p.w_split, three, CE_LARGE, &p.tile_w, &p.w_split, &p.w_splits);
  // Logits kept: written, read, 8 bytes each.  Computed again: their products, or where there are few rows the weight's reading.
  const double again = std::max((three ? 6.0 : 1.0) * 2.0 * p.n * p.D / 1.0e9, (three ? 4.0 : 2.0) * p.D / 4.5e6);
  p.keep = (dx || dw) && p.n * padded * 4 <= KEEP_BYTES && p.n * 8 / 5.0e6 < again;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) & ~static_cast<size_t>(255);
    return here;
  };
  const size_t n = static_cast<size_t>(p.n), rows = static_cast<size_t>(p.rows);
  p.count = take(4);
  p.source = take(n * 4);
  p.place = take(n * 4);
  p.row = take(n * sizeof(CeRow));
  p.scaled = take(n * 8);
  p.target = take(n * 4);
  p.stats = take(n * p.slots * sizeof(float2));
  p.x = take(n * p.ld * 2 * p.planes);
  p.w = three && !p.direct ? take(static_cast<size_t>(p.piece) * p.ld * 2 * p.planes) : at;
  p.dl = dx || dw ? take(rows * p.piece * 2 * p.planes) : at;
  p.logits = p.keep ? take(static_cast<size_t>(padded) * n * 4) : at;
  p.sums = dx ? take(static_cast<size_t>(p.splits) * n * p.D * 4) : at;
  p.w_sums = dw && p.w_splits > 1 ? take(static_cast<size_t>(p.w_splits) * p.V * p.D * 4) : at;
  p.bytes = at;
  return p;
}

template <typename T>
saki_status run(const saki_head* h, const saki_ce_args* a, const Plan& p, char* ws, hipStream_t hs) {
  constexpr bool three = sizeof(T) == 4;
  const bool dx = a->grad_hidden != nullptr, dw = a->grad_weight != nullptr;
  CeRows R{};
  R.n_rows = p.n;
  R.vocab = static_cast<int>(p.V);
  R.token = a->token;
  R.row_weight = a->row_weight;
  R.valid = a->valid_mask;
  R.grad_scale = a->grad_scale;
  R.row_loss = a->row_loss;
  R.logp_token = a->logp_token;
  R.scaled_loss = a->loss_sum ? reinterpret_cast<double*>(ws + p.scaled) : nullptr;
  R.row_status = a->row_status;
  R.source = reinterpret_cast<int*>(ws + p.source);
  R.place = reinterpret_cast<int*>(ws + p.place);
  R.rows = reinterpret_cast<CeRow*>(ws + p.row);
  R.stats = reinterpret_cast<float2*>(ws + p.stats);
  R.target = reinterpret_cast<float*>(ws + p.target);
  R.slots = static_cast<int>(p.slots);
  saki_status st;
#define SAKI_LAUNCHED(what)                     \
  st = abi_launched(hipGetLastError(), what);   \
  if (st != SAKI_OK) return st
  if (a->valid_mask) {
    R.count = reinterpret_cast<int*>(ws + p.count);
    hipLaunchKernelGGL(ce_rows_kernel, dim3(1), dim3(1024), 0, hs, R);
    SAKI_LAUNCHED("ce_rows_kernel");
  }
  CeGemm G{};
  G.count = R.count;
  G.planes = p.planes;
  // rows of X as the products take them: as they are, or packed
  const bool pack = three || a->valid_mask || p.D != p.ld;
  const uint16_t* x = static_cast<const uint16_t*>(h->hidden);
  int64_t ldx = h->hidden_stride;
  const int64_t x_plane = p.n * p.ld;
  if (pack) {
    uint16_t* const to = reinterpret_cast<uint16_t*>(ws + p.x);
    const int64_t blocks = std::min<int64_t>(ceil_div(p.n * p.ld / 8, 256), 8192);
    hipLaunchKernelGGL((ce_pack_kernel<T>), dim3(static_cast<unsigned>(blocks)), dim3(256), 0, hs,
                       static_cast<const T*>(h->hidden), h->hidden_stride, p.n, static_cast<int>(p.D),
                       R.count ? R.source : nullptr, R.count, to, p.ld, x_plane);
    SAKI_LAUNCHED("ce_pack_kernel");
    x = to;
    ldx = p.ld;
  }
  uint16_t* const w_parts = reinterpret_cast<uint16_t*>(ws + p.w);
  const int64_t w_plane = p.piece * p.ld;
  // tokens v0 .. v0 + nv of the weight as the products take them
  bool parts_there = false;
  auto weight = [&](int64_t v0, int64_t nv) {
    if constexpr (three) {
      if (p.direct) {
        G.p = static_cast<const T*>(h->weight) + v0 * h->weight_stride;
        G.ldp = h->weight_stride;
        return hipSuccess;
      }
      if (parts_there && p.pieces == 1) return hipSuccess;
      parts_there = true;
      const int64_t blocks = std::min<int64_t>(ceil_div(nv * p.ld / 8, 256), 8192);
      hipLaunchKernelGGL((ce_pack_kernel<T>), dim3(static_cast<unsigned>(blocks)), dim3(256), 0, hs,
                         static_cast<const T*>(h->weight) + v0 * h->weight_stride, h->weight_stride, nv,
                         static_cast<int>(p.D), nullptr, nullptr, w_parts, p.ld, w_plane);
      G.p = w_parts;
      G.ldp = p.ld;
      G.p_plane = w_plane;
    } else {
      G.p = static_cast<const uint16_t*>(h->weight) + v0 * h->weight_stride;
      G.ldp = h->weight_stride;
    }
    return hipGetLastError();
  };
  auto rows_q = [&]() {
    G.q = x;
    G.ldq = ldx;
    G.q_plane = x_plane;
    G.n_q = static_cast<int>(p.n);
    G.n_k = static_cast<int>(three && !p.direct ? p.ld : p.D);
  };
  // the log-sum-exp (bf16: of the whole vocabulary at once)
  G.stats = reinterpret_cast<float2*>(ws + p.stats);
  G.token = a->token;
  G.source = R.source;
  G.target = reinterpret_cast<float*>(ws + p.target);
  G.slots = static_cast<int>(p.slots);
  float* const logits = p.keep ? reinterpret_cast<float*>(ws + p.logits) : nullptr;
  G.ld_logits = round_up(p.V, CE_PAD);
  const int64_t step = three && !p.direct ? p.piece : p.V;
  for (int64_t v0 = 0; v0 < p.V; v0 += step) {
    const int64_t nv = std::min(step, p.V - v0);
    st = abi_launched(weight(v0, nv), "ce_pack_kernel");
    if (st != SAKI_OK) return st;
    rows_q();
    for (int64_t u0 = v0; u0 < v0 + nv; u0 += p.s_step) {
      CeGemm L = G;
      L.p = static_cast<const char*>(G.p) + (u0 - v0) * G.ldp * (p.direct ? 4 : 2);
      L.n_p = static_cast<int>(std::min(p.s_step, v0 + nv - u0));
      L.slot0 = static_cast<int>(u0 / p.wave_p);
      L.v0 = static_cast<int>(u0);
      L.logits = logits ? logits + u0 : nullptr;
      st = abi_launched(launch_ce_part<CE_LSE>(L, p.tile_s, three, 1, hs), "ce_gemm_kernel");
      if (st != SAKI_OK) return st;
    }
  }
  hipLaunchKernelGGL(ce_loss_kernel, dim3(static_cast<unsigned>(p.n)), dim3(256), 0, hs, R);
  SAKI_LAUNCHED("ce_loss_kernel");
  if (a->loss_sum) {
    st = abi_loss_sum(R.scaled_loss, p.n, a->loss_sum, hs);
    if (st != SAKI_OK) return st;
  }
  if (!dx && !dw) return SAKI_OK;
  uint16_t* const dl = reinterpret_cast<uint16_t*>(ws + p.dl);
  const int64_t dl_plane = p.rows * p.piece;
  for (int64_t v0 = 0; v0 < p.V; v0 += p.piece) {
    const int64_t nv = std::min(p.piece, p.V - v0);
    if (dx || !logits) {
      st = abi_launched(weight(v0, nv), "ce_pack_kernel");
      if (st != SAKI_OK) return st;
    }
    rows_q();
    G.n_p = static_cast<int>(nv);
    G.rows = R.rows;
    G.dl = dl;
    G.ld_dl = p.piece;
    G.dl_plane = dl_plane;
    G.v0 = static_cast<int>(v0);
    if (logits) {
      G.logits = logits + v0;
      const dim3 grid(static_cast<unsigned>(ceil_div(nv, 2048)), static_cast<unsigned>(std::min<int64_t>(round_up(p.n, CE_BK), 4096)));
      hipLaunchKernelGGL((ce_share_kernel<three>), grid, dim3(256), 0, hs, G);
      SAKI_LAUNCHED("ce_share_kernel");
    } else {
      st = abi_launched(launch_ce_part<CE_DL>(G, p.tile_l, three, 1, hs), "ce_gemm_kernel");
      if (st != SAKI_OK) return st;
    }
    if (dx) {
      CeGemm X = G;
      X.q = dl;
      X.ldq = p.piece;
      X.q_plane = dl_plane;
      X.n_p = static_cast<int>(p.D);
      X.n_k = static_cast<int>(nv);
      X.k_split = static_cast<int>(p.k_split);
      X.sums = reinterpret_cast<float*>(ws + p.sums);
      X.ld_sums = p.D;
      X.split_stride = p.n * p.D;
      X.add = v0 > 0;
      st = abi_launched(launch_ce_part<CE_DX>(X, p.tile_x, three, static_cast<int>(p.splits), hs), "ce_gemm_kernel");
      if (st != SAKI_OK) return st;
    }
    if (dw) {
      CeGemm W = G;
      W.p = x;
      W.ldp = ldx;
      W.p_plane = x_plane;
      W.q = dl;
      W.ldq = p.piece;
      W.q_plane = dl_plane;
      W.n_p = static_cast<int>(p.D);
      W.n_q = static_cast<int>(nv);
      W.n_k = static_cast<int>(p.n);
      W.grad = static_cast<T*>(a->grad_weight) + v0 * a->grad_weight_stride;
      W.ld_grad = a->grad_weight_stride;
      W.scale = a->grad_scale;
      W.k_split = static_cast<int>(p.w_split);
      if (p.w_splits > 1) {
        W.sums = reinterpret_cast<float*>(ws + p.w_sums);
        W.ld_sums = p.D;
        W.split_stride = p.V * p.D;
      }
      st = abi_launched(launch_ce_part<CE_DW>(W, p.tile_w, three, static_cast<int>(p.w_splits), hs), "ce_gemm_kernel");
      if (st != SAKI_OK) return st;
    }
  }
  using S = std::conditional_t<three, float, uint16_t>;
  auto add_up = [&](const CeSums& C) {
    const int64_t blocks = std::min<int64_t>(ceil_div(C.n_rows * p.D / 4, 256), 16384);
    hipLaunchKernelGGL((ce_sums_kernel<S>), dim3(static_cast<unsigned>(blocks)), dim3(256), 0, hs, C);
  };
  if (dx) {
    add_up(CeSums{reinterpret_cast<float*>(ws + p.sums), p.D, p.n * p.D, static_cast<int>(p.splits), p.n, static_cast<int>(p.D),
                  R.count ? R.place : nullptr, R.rows, a->grad_scale, a->grad_hidden, a->grad_hidden_stride});
    SAKI_LAUNCHED("ce_sums_kernel");
  }
  if (dw && p.w_splits > 1) {
    add_up(CeSums{reinterpret_cast<float*>(ws + p.w_sums), p.D, p.V * p.D, static_cast<int>(p.w_splits), p.V, static_cast<int>(p.D),
                  nullptr, nullptr, a->grad_scale, a->grad_weight, a->grad_weight_stride});
    SAKI_LAUNCHED("ce_sums_kernel");
  }
#undef SAKI_LAUNCHED
  return SAKI_OK;
}

}  // namespace

extern "C" {

size_t saki_linear_ce_workspace_bytes(const saki_head* head, int32_t grads) {
  if (check_head(head) != SAKI_OK || grads < 0 || grads > 3 || head->n_rows == 0) return 0;
  return plan_of(head, grads & 1, grads & 2).bytes;
}

saki_status saki_linear_ce(const saki_head* head, const saki_ce_args* args, void* ws, size_t ws_bytes, saki_stream_t stream) {
  saki_status st = check_head(head);
  if (st != SAKI_OK) return st;
  if (!args) return abi_fail(SAKI_E_NULLPTR, "args is NULL");
  if (args->reserved != 0) return abi_fail(SAKI_E_VALUE, "saki_ce_args.reserved must be 0");
  if (!std::isfinite(args->grad_scale)) return abi_fail(SAKI_E_VALUE, "grad_scale is not finite");
  const int size = head->dtype == SAKI_BF16 ? 2 : 4;
  if ((args->grad_hidden && (args->grad_hidden_stride < head->hidden_size || args->grad_hidden_stride >= MOST_STRIDE)) ||
      (args->grad_weight && (args->grad_weight_stride < head->hidden_size || args->grad_weight_stride >= MOST_STRIDE)))
    return abi_fail(SAKI_E_SHAPE, "a gradient's row stride outside [hidden_size, 2^22)");
  if (head->n_rows > 0 && (!head->hidden || !head->weight || !args->token))
    return abi_fail(SAKI_E_NULLPTR, "hidden, weight and token are required");
  if (!aligned(head->hidden, 16) || !aligned(head->weight, 16) || !aligned(args->grad_hidden, 16) ||
      !aligned(args->grad_weight, 16) || head->hidden_stride * size % 16 != 0 || head->weight_stride * size % 16 != 0 ||
      (args->grad_hidden && args->grad_hidden_stride * size % 16 != 0) ||
      (args->grad_weight && args->grad_weight_stride * size % 16 != 0))
    return abi_fail(SAKI_E_ALIGN, "rows of hidden, weight and their gradients must be 16-byte aligned");
  if (!aligned(args->token, 4) || !aligned(args->row_weight, 4) || !aligned(args->row_loss, 4) ||
      !aligned(args->logp_token, 4) || !aligned(args->loss_sum, 8))
    return abi_fail(SAKI_E_ALIGN, "an array of 4 or 8 bytes an entry is not aligned to them");
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (head->n_rows == 0) {  // the sums over no rows
    if (args->grad_weight) {
      const int D = static_cast<int>(head->hidden_size);
      const dim3 grid(static_cast<unsigned>(std::min<int64_t>(ceil_div(head->vocab * D / 8, 256), 8192))), block(256);
      if (size == 2) hipLaunchKernelGGL((ce_zero_kernel<uint16_t>), grid, block, 0, hs, static_cast<uint16_t*>(args->grad_weight), args->grad_weight_stride, head->vocab, D);
      else hipLaunchKernelGGL((ce_zero_kernel<float>), grid, block, 0, hs, static_cast<float*>(args->grad_weight), args->grad_weight_stride, head->vocab, D);
      st = abi_launched(hipGetLastError(), "ce_zero_kernel");
      if (st != SAKI_OK) return st;
    }
    if (args->loss_sum) {
      st = abi_loss_sum(nullptr, 0, args->loss_sum, hs);
      if (st != SAKI_OK) return st;
    }
    return abi_ok();
  }
  const Plan p = plan_of(head, args->grad_hidden != nullptr, args->grad_weight != nullptr);
  if (!ws || ws_bytes < p.bytes)
    return abi_fail(SAKI_E_WORKSPACE, "workspace NULL or smaller than saki_linear_ce_workspace_bytes()");
  if (!aligned(ws, 256)) return abi_fail(SAKI_E_ALIGN, "workspace must be 256-byte aligned");
  st = head->dtype == SAKI_BF16 ? run<uint16_t>(head, args, p, static_cast<char*>(ws), hs)
                                : run<float>(head, args, p, static_cast<char*>(ws), hs);
  return st != SAKI_OK ? st : abi_ok();
}

}  // extern "C"

#endif
