// Divergence between a student's row and a teacher's list of top logits, and its gradient.
//
// With z = s / tau, U the tokens that are not listed, S_U = sum over U of e^{z - m_U}, m_U their
// largest z, the student's share of the bucket R is p_R = S_U e^{m_U - lse}, and every gradient
// entry of U is one number times e^{z_j - m_U}:
//   forward  (p_R - t_R) / S_U,   reverse  p_R (log(p_R / t_R) - l) / S_U     (times grad_scale / tau).
// So the row needs two sweeps: S_U, then the gradient; the listed tokens, left out of S_U by a bit
// mask in LDS, are a thread each and are written over the second sweep's values, by the lanes that stored those.  S_U has its own
// reference, hence neither p_R nor a gradient entry is a difference of the row's whole
// sum and the listed part of it, and a bucket of 1e-30 of the row has full precision.
//
// What bounds it: memory.  8,192 rows of 151,936 bf16 with a bf16 gradient: 1,167 us, 4.3 TB/s of reads and writes (a large copy
// reaches 4.8); the second sweep runs backwards over what the caches still hold.
#pragma once

#include "common.hpp"
#include "../../include/saki_distill.h"

namespace saki {

struct DistillParams {
  const void* s;
  int64_t n_rows;
  int64_t stride;
  int V;
  int k;
  const int32_t* token;
  const float* logit;
  const float* rest;
  int64_t list_stride;
  float c;      // log2(e) / tau
  int reverse;
  const uint8_t* valid;
  float grad_scale;
  float inv_tau;
  float* row_loss;
  double* scaled_loss;
  void* grad;
  int64_t grad_stride;
  uint8_t* row_status;
  unsigned int* next_row;
};

constexpr int DT_SEG = 1 << 17;  // entries whose mask LDS holds at a time

template <int NT>
struct DistillShared {
  static constexpr int NW = NT / WAVE;
  uint32_t mask[DT_SEG / 32];
  int2 patch[SAKI_MAX_TOP_K];  // listed tokens and their gradients
  double red_d[NW][RED_MAX];
  float red_f[NW][4];
  int red_i[NW][4];
  unsigned int next;
};

// What a row comes to: what its gradient is made of.
struct DistillRow {
  float coef;  // the gradient at tokens that are not listed is coef 2^((x - mU) c)
  float mU;    // the largest of their logits
  bool take;   // the row has a loss (else its gradient is coef: 0, or NaN)
};

// From the block's sums: `slot`, this thread's place in the list (held: it has an entry, `token`, whose logits are s_tok with
// the student and `logit` with the teacher), this wave's largest unlisted logit m, this thread's part S of
// sum 2^((x - m) c) and smallest logit lo; wrong: the entry, or rest, cannot be used.  The bucket of the other tokens is
// the entry behind the list's last.  Writes the row's outputs but the gradient; that of the listed tokens goes to sh.patch.
// Logarithms in natural units, in 64 bits: a divergence near 0 is a difference of large ones.  Only the waves that hold
// entries compute with them; which ones these are differs from workgroup to workgroup, so sums over the list are added in the
// list's order: a row's bits do not depend on the workgroup that takes it.
template <typename BLOCK>
__device__ __forceinline__ DistillRow distill_solve(BLOCK& B, const DistillParams& P, int64_t r, int slot, bool part, bool held,
                                                    bool wrong, int token, float s_tok, float logit, float rest, float m, double S,
                                                    float lo) {
  const double c64 = static_cast<double>(P.c) * LN2_D;
  const int place = __builtin_amdgcn_readfirstlane(slot / WAVE);  // this wave's in the list
  const bool lists = place * WAVE <= P.k, bucket = slot == P.k;
  float mm[3] = {m, held ? s_tok : -finf(), held && !wrong ? logit : -finf()};
  B.max(mm);
  const float mU = mm[0], mP = fmaxf(mm[1], mU), mT = fmaxf(mm[2], rest);
  const float teach = bucket ? rest : logit;
  const bool has_t = (held || bucket) && teach > -finf() && mT > -finf();
  double v[6] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0}, z = 0.0, y = 0.0, own_p = 0.0, own_t = 0.0;
  v[0] = S > 0.0 ? S * static_cast<double>(fexp2((m - mU) * P.c)) : S;
  v[1] = wrong ? 1.0 : 0.0;
  v[2] = (lo > -finf() && mU < finf() ? 0.0 : 1024.0) + (held ? 1.0 : 0.0);  // (fewer than 1,024 threads)
  if (lists) {
    z = (static_cast<double>(bucket ? mU : s_tok) - mP) * c64;
    y = (static_cast<double>(teach) - mT) * c64;
    own_p = held || bucket ? exp(z) : 0.0;
    own_t = has_t ? exp(y) : 0.0;
    v[3] = bucket ? own_p : 0.0;
    v[4] = bucket ? 0.0 : own_p;
    v[5] = own_t;
  }
  B.template sum_placed<4>(v, place);
  const double SU = v[0];
  const int n_held = static_cast<int>(v[2]) & 1023;
  const bool some = mT > -finf(), others = n_held < P.V;
  double lt = 0.0, lp = 0.0, log_p = 0.0, p = 0.0, t = 0.0;
  // infinite divergences: forward, a share of the teacher's where the student has no token; reverse, the
  // other way round
  double l[2] = {0.0, 0.0};
  if (lists) {
    if (bucket) own_p = others ? own_p * SU : 0.0;
    const double all_p = v[4] + (others ? v[3] * SU : 0.0), all_t = v[5];
    const double log_t = log(all_t);
    log_p = log(all_p);
    lt = y - log_t;
    lp = z - log_p + (bucket ? log(SU) : 0.0);
    p = own_p / all_p;
    t = own_t / all_t;
    if (some && (held || (bucket && others))) {
      if (P.reverse) {
        l[0] = p > 0.0 ? p * (lp - lt) : 0.0;
        l[1] = teach > -finf() ? 0.0 : 1.0;
      } else {
        l[0] = t > 0.0 ? t * (lt - lp) : 0.0;
      }
    }
    if (some && bucket && !others && !P.reverse) l[1] = rest > -finf() ? 1.0 : 0.0;
  }
  B.template sum_placed<0>(l, place);
  if (lists) {
    double loss = l[0];
    const bool bad = v[1] != 0.0 || l[1] != 0.0;
    const bool finite = v[2] < 1024.0 && SU == SU && isfinite(log_p);
    const bool take = part && some && !bad && finite, nan = part && (bad || !finite);
    if (!take) loss = nan ? __builtin_nan("") : 0.0;
    const double scale = static_cast<double>(P.grad_scale) * P.inv_tau;
    const double g = (P.reverse ? p * (lp - lt - loss) : p - t) * scale;
    if (slot < P.k) B.sh.patch[slot] = make_int2(take && held ? token : -1, __float_as_int(static_cast<float>(g)));
    if (bucket) {
      B.sh.red_f[0][0] = take ? (others ? static_cast<float>(g / SU) : 0.0f) : nan ? nanf_() : 0.0f;
      B.sh.red_i[0][0] = take ? 1 : 0;
      if (P.row_loss) P.row_loss[r] = static_cast<float>(loss);
      if (P.scaled_loss) P.scaled_loss[r] = static_cast<double>(P.grad_scale) * loss;
      if (P.row_status)
        P.row_status[r] = !part ? SAKI_ROW_OK : !finite ? SAKI_ROW_NONFINITE : bad ? SAKI_ROW_BAD_TARGET : SAKI_ROW_OK;
    }
  }
  __syncthreads();
  DistillRow R;
  R.mU = mU;
  R.coef = B.sh.red_f[0][0];
  R.take = uniform(B.sh.red_i[0][0] != 0);
  return R;
}

typedef __bf16 dt_bf16x2 __attribute__((ext_vector_type(2)));
typedef float dt_f32x2 __attribute__((ext_vector_type(2)));
// Two floats rounded to bf16 (to nearest, ties to even) by one instruction.
__device__ __forceinline__ uint32_t distill_pack(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(dt_f32x2{a, b}, dt_bf16x2));
}
template <typename G>
__device__ __forceinline__ void distill_store8(G* p, const float* x) {
  if constexpr (sizeof(G) == 2) {
    const u32x4 v = {distill_pack(x[0], x[1]), distill_pack(x[2], x[3]), distill_pack(x[4], x[5]), distill_pack(x[6], x[7])};
    __builtin_nontemporal_store(v, (g_u32x4*)(p));
  } else {
    Storer<G>::store8(p, x);
  }
}

template <typename T, typename G, bool GRAD, int NT>
__global__ __launch_bounds__(NT, 4) void distill_kernel(DistillParams P) {
  constexpr int NW = NT / WAVE;
  __shared__ DistillShared<NT> sh;
  Block<NT, DistillShared<NT>> B(sh);
  const int V = P.V, k = P.k, lane = B.lane;
  const int wave = __builtin_amdgcn_readfirstlane(B.wave);
  const float c = P.c;
  const unsigned int n = static_cast<unsigned int>(P.n_rows);
  // this thread's place in the list; the waves that hold it are others in each of a CU's workgroups, whose first
  // waves share a SIMD
  const int slot = (B.tid + static_cast<int>(blockIdx.x >> 8) * WAVE) % NT;
  // What is read of a row's list while the row before it is written; what it holds is looked at when its turn comes.
  unsigned int r = blockIdx.x;  // (the counter's rows come behind the workgroups' first)
  int token_in = -1;
  float logit_in = 0.0f, rest_in = -finf();
  uint8_t valid_in = 1;
  auto entry = [&](unsigned int row) __attribute__((always_inline)) {
    if (row >= n) return;
    if (slot < k) {
      token_in = P.token[static_cast<int64_t>(row) * P.list_stride + slot];
      logit_in = P.logit[static_cast<int64_t>(row) * P.list_stride + slot];
    }
    if (P.rest) rest_in = P.rest[row];
    if (P.valid) valid_in = P.valid[row];
  };
  entry(r);
  while (r < n) {
    __syncthreads();  // (the row before is done with LDS)
    unsigned int next = ~0u;  // (a call of no more rows than workgroups has no counter: one row each)
    if (B.tid == 0 && P.next_row) next = take_index(P.next_row) + gridDim.x;
    const T* row = static_cast<const T*>(P.s) + static_cast<int64_t>(r) * P.stride;
    G* out = GRAD ? static_cast<G*>(P.grad) + static_cast<int64_t>(r) * P.grad_stride : nullptr;
    const bool part = uniform(valid_in != 0);
    const int token = part ? token_in : -1;  // this thread's entry of the list
    const float logit = token >= 0 ? logit_in : 0.0f, rest = part ? rest_in : -finf();
    bool wrong = token < -1 || token >= V;
    const bool held = !wrong && token >= 0;
    const float s_tok = held ? Loader<T>::load1(row + token) : 0.0f;
    wrong |= (held && !(logit < finf())) || !(rest < finf());
    // the sum over the tokens that are not listed
    float m = -finf(), lo = finf();
    double S = 0.0;
    if (part) {
      for (int s0 = 0; s0 < V; s0 += DT_SEG) {
        const int len = min(V - s0, DT_SEG);
        if (s0 > 0) __syncthreads();  // (the mask of the segment before was read)
        for (int w = B.tid; w < (len + 31) / 32; w += NT) sh.mask[w] = 0u;
        __syncthreads();
        if (held && token >= s0 && token - s0 < len) {
          const uint32_t bit = 1u << ((token - s0) & 31);
          wrong |= (atomicOr(&sh.mask[(token - s0) >> 5], bit) & bit) != 0u;  // listed twice
        }
        __syncthreads();
        const uint8_t* const bits = reinterpret_cast<const uint8_t*>(sh.mask);
        for_chunks1<T, NW>(row + s0, len, wave, lane, [&](auto tail, float* x, uint32_t vm, int ch) {
          constexpr bool TAIL = decltype(tail)::value;
          // 8 entries a byte: those of this lane's two pieces of the chunk
          uint32_t listed;
          if (TAIL) {
            const int b0 = ch * (CHUNK / 8) + lane, last = (len - 1) / 8;
            listed = static_cast<uint32_t>(bits[min(b0, last)]) | static_cast<uint32_t>(bits[min(b0 + 64, last)]) << 8;
          } else {
            listed = static_cast<uint32_t>(bits[ch * (CHUNK / 8) + lane]) | static_cast<uint32_t>(bits[ch * (CHUNK / 8) + 64 + lane]) << 8;
          }
#pragma unroll
          for (int e = 0; e < EPL; e += 2) {
            if (!TAIL) lo = min3_raw(lo, x[e], x[e + 1]);
            if (TAIL && ((vm >> e) & 1u)) lo = fminf(lo, x[e]);
            if (TAIL && ((vm >> (e + 1)) & 1u)) lo = fminf(lo, x[e + 1]);
          }
          if (TAIL || wave_any(listed != 0u)) {
#pragma unroll
            for (int e = 0; e < EPL; ++e)
              if ((TAIL && !((vm >> e) & 1u)) || ((listed >> e) & 1u)) x[e] = -finf();
          }
          float lm = -finf();
#pragma unroll
          for (int e = 0; e < EPL; e += 2) lm = max3_raw(lm, x[e], x[e + 1]);
          if (wave_any(lm > m)) {
            const float to = wave_max(lm);
            S = m == -finf() ? 0.0 : S * static_cast<double>(fexp2((m - to) * c));
            m = to;
          }
          if (m > -finf()) {
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) sum += fexp2((x[e] - m) * c);
            S += static_cast<double>(sum);
          } else {
#pragma unroll
            for (int e = 0; e < EPL; ++e) S = x[e] == x[e] ? S : __builtin_nan("");
          }
        });
      }
    }
    if (B.tid == 0) sh.next = next;
    const DistillRow R = distill_solve(B, P, r, slot, part, held, wrong, token, s_tok, logit, rest, m, S, lo);
    const unsigned int after = static_cast<unsigned int>(__builtin_amdgcn_readfirstlane(static_cast<int>(sh.next)));
    entry(after);
    if (GRAD) {
      const float coef = R.coef;
      if (coef == 0.0f || coef != coef) {
        float x[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) x[e] = coef;
        for (int ch = wave; ch < (V + CHUNK - 1) / CHUNK; ch += NW) store_lane<G, true>(out, ch, lane, V, x);
      } else {
        for_chunks1<T, NW, CACHE_NONE, true>(row, V, wave, lane, [&](auto tail, float* x, uint32_t, int ch) {
          constexpr bool TAIL = decltype(tail)::value;
          float g[EPL];
#pragma unroll
          for (int e = 0; e < EPL; ++e) g[e] = coef * fexp2((x[e] - R.mU) * c);
          if constexpr (TAIL) {
            store_lane<G, true>(out, ch, lane, V, g);
          } else {
            distill_store8(out + ch * CHUNK + 8 * lane, g);
            distill_store8(out + ch * CHUNK + 512 + 8 * lane, g + 8);
          }
        });
      }
      // the listed tokens of this wave's chunks, each by the lane that stored the chunk's entry there
      for (int i0 = 0; R.take && i0 < k; i0 += WAVE) {
        const int2 p = i0 + lane < k ? sh.patch[i0 + lane] : make_int2(-1, 0);
        uint64_t mine = __ballot(p.x >= 0 && (p.x / CHUNK) % NW == wave);
        while (mine != 0ull) {
          const int e = __builtin_ctzll(mine);
          mine &= mine - 1;
          const int v = __builtin_amdgcn_readlane(p.x, e);
          const float g = __int_as_float(__builtin_amdgcn_readlane(p.y, e));
          if (lane == (v >> 3) % WAVE) Storer<G>::store1(out + v, g);
        }
      }
    }
    r = after;
  }
}

}  // namespace saki
