// Divergence between a student's row and a teacher's list of top logits, and its gradient.
//
// With z = s / tau, U the tokens that are not listed, S_U = sum over U of e^{z - m_U}, m_U their
// largest z, the student's share of the bucket R is p_R = S_U e^{m_U - lse}, and every gradient
// entry of U is one number times e^{z_j - m_U}:
//   forward  (p_R - t_R) / S_U,   reverse  p_R (log(p_R / t_R) - l) / S_U     (times grad_scale / tau).
// So the row needs two sweeps: S_U, then the gradient; the listed tokens, left out of S_U by a bit
// mask in LDS, are a thread each and are written over the second sweep's values.  S_U has its own
// reference, hence neither p_R nor a gradient entry is a difference of the row's whole
// sum and the listed part of it, and a bucket of 1e-30 of the row has full precision.
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
  double red_d[NW][RED_MAX];
  float red_f[NW][4];
  int red_i[NW][4];
  unsigned int next;
};

// What a row comes to: its loss, and what its gradient is made of.
struct DistillRow {
  float coef;     // the gradient at tokens that are not listed is coef 2^((x - mU) c)
  float mU;       // the largest of their logits
  float listed;   // the gradient at this thread's token
  bool take;      // the row has a loss (else its gradient is coef: 0, or NaN)
};

// From the block's sums: this thread's entry of the list (held: token, its logit with the student s_tok and the
// teacher), this wave's largest unlisted logit m, this thread's part S of sum 2^((x - m) c) and smallest logit lo;
// wrong: the entry, or rest, cannot be used.  Writes the row's outputs but the gradient.  Logarithms in natural units, in 64 bits:
// a divergence near 0 is a difference of large ones.
// Only the waves that hold entries compute with them, and one posts what comes out.
template <typename BLOCK>
__device__ __forceinline__ DistillRow distill_solve(BLOCK& B, const DistillParams& P, int64_t r, bool part, bool held, bool wrong,
                                                    float s_tok, float logit, float rest, float m, double S, float lo) {
  const double c64 = static_cast<double>(P.c) * LN2_D;
  const bool lists = uniform(B.wave * WAVE < P.k);  // this wave holds entries (the first one always)
  float mm[3] = {m, held ? s_tok : -finf(), held && !wrong ? logit : -finf()};
  B.max(mm);
  const float mU = mm[0], mP = fmaxf(mm[1], mU), mT = fmaxf(mm[2], rest);
  double v[6] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0}, z = 0.0, y = 0.0, zU = 0.0, yR = 0.0, eU = 0.0, eR = 0.0;
  v[0] = S > 0.0 ? S * static_cast<double>(fexp2((m - mU) * P.c)) : S;
  v[4] = lo > -finf() && mU < finf() ? 0.0 : 1.0;
  if (lists) {
    z = (static_cast<double>(s_tok) - mP) * c64;
    y = (static_cast<double>(logit) - mT) * c64;
    zU = (static_cast<double>(mU) - mP) * c64;
    yR = (static_cast<double>(rest) - mT) * c64;
    v[1] = held ? exp(z) : 0.0;
    v[2] = held && mT > -finf() ? exp(y) : 0.0;
    v[3] = wrong ? 1.0 : 0.0;
    v[5] = held ? 1.0 : 0.0;
    eU = exp(zU);
    eR = rest > -finf() ? exp(yR) : 0.0;
  }
  const double own_p = v[1], own_t = v[2];
  B.sum(v);
  const double SU = v[0];
  const bool some = mT > -finf(), others = v[5] < static_cast<double>(P.V);
  double lt = 0.0, lp = 0.0, ltR = 0.0, lpR = 0.0, log_p = 0.0, p = 0.0, t = 0.0, pR = 0.0, tR = 0.0;
  // infinite divergences: forward, a share of the teacher's where the student has no token; reverse, the
  // other way round
  double l[2] = {0.0, 0.0};
  if (lists) {
    const double eP = others ? SU * eU : 0.0, all_p = v[1] + eP, all_t = v[2] + eR;
    const double log_t = log(all_t);
    log_p = log(all_p);
    lt = y - log_t;
    lp = z - log_p;
    ltR = yR - log_t;
    lpR = zU + log(SU) - log_p;
    p = own_p / all_p;
    t = own_t / all_t;
    pR = eP / all_p;
    tR = eR / all_t;
    if (held && some) {
      if (P.reverse) {
        l[0] = p > 0.0 ? p * (lp - lt) : 0.0;
        l[1] = logit > -finf() ? 0.0 : 1.0;
      } else {
        l[0] = t > 0.0 ? t * (lt - lp) : 0.0;
      }
    }
  }
  B.sum(l);
  DistillRow R;
  R.mU = mU;
  R.listed = 0.0f;
  if (lists) {
    double loss = l[0];
    bool bad = v[3] != 0.0 || l[1] != 0.0;
    if (P.reverse) {
      if (others) loss += pR > 0.0 ? pR * (lpR - ltR) : 0.0;
      bad |= some && others && !(rest > -finf());
    } else {
      if (tR > 0.0 && others) loss += tR * (ltR - lpR);
      bad |= rest > -finf() && !others;
    }
    const bool finite = v[4] == 0.0 && SU == SU && isfinite(log_p);
    const bool take = part && some && !bad && finite, nan = part && (bad || !finite);
    if (!take) loss = nan ? __builtin_nan("") : 0.0;
    const double scale = static_cast<double>(P.grad_scale) * P.inv_tau;
    R.listed = static_cast<float>((P.reverse ? p * (lp - lt - loss) : p - t) * scale);
    if (B.tid == 0) {
      const double gR = others ? (P.reverse ? pR * (lpR - ltR - loss) : pR - tR) * scale / SU : 0.0;
      B.sh.red_f[0][0] = take ? static_cast<float>(gR) : nan ? nanf_() : 0.0f;
      B.sh.red_i[0][0] = take ? 1 : 0;
      if (P.row_loss) P.row_loss[r] = static_cast<float>(loss);
      if (P.scaled_loss) P.scaled_loss[r] = static_cast<double>(P.grad_scale) * loss;
      if (P.row_status)
        P.row_status[r] = !part ? SAKI_ROW_OK : !finite ? SAKI_ROW_NONFINITE : bad ? SAKI_ROW_BAD_TARGET : SAKI_ROW_OK;
    }
  }
  __syncthreads();
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
  static_assert(SAKI_MAX_TOP_K <= NT, "a thread for each listed token");
  constexpr int NW = NT / WAVE;
  __shared__ DistillShared<NT> sh;
  Block<NT, DistillShared<NT>> B(sh);
  const int V = P.V, k = P.k, lane = B.lane;
  const int wave = __builtin_amdgcn_readfirstlane(B.wave);
  const float c = P.c;
  const unsigned int n = static_cast<unsigned int>(P.n_rows);
  // What is read of a row's list while the row before it is written; what it holds is looked at when its turn comes.
  unsigned int r = blockIdx.x;  // (the counter's rows come behind the workgroups' first)
  int token_in = -1;
  float logit_in = 0.0f, rest_in = -finf();
  uint8_t valid_in = 1;
  auto entry = [&](unsigned int row) __attribute__((always_inline)) {
    if (row >= n) return;
    if (B.tid < k) {
      token_in = P.token[static_cast<int64_t>(row) * P.list_stride + B.tid];
      logit_in = P.logit[static_cast<int64_t>(row) * P.list_stride + B.tid];
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
    const DistillRow R = distill_solve(B, P, r, part, held, wrong, s_tok, logit, rest, m, S, lo);
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
      // the listed tokens over it, once the row's stores are done
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (R.take && held) Storer<G>::store1(out + token, R.listed);
    }
    r = after;
  }
}

}  // namespace saki
