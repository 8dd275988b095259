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

constexpr int DT_NT = 256;
constexpr int DT_NW = DT_NT / WAVE;
constexpr int DT_SEG = 1 << 17;  // entries whose mask LDS holds at a time
static_assert(SAKI_MAX_TOP_K <= DT_NT, "a thread for each listed token");

struct DistillShared {
  uint32_t mask[DT_SEG / 32];
  double red_d[DT_NW][RED_MAX];
  float red_f[DT_NW][4];
  int red_i[DT_NW][4];
  unsigned int next;
};

template <typename T, typename G, bool GRAD>
__global__ __launch_bounds__(DT_NT, 4) void distill_kernel(DistillParams P) {
  __shared__ DistillShared sh;
  Block<DT_NT, DistillShared> B(sh);
  const int V = P.V, k = P.k, lane = B.lane;
  const int wave = __builtin_amdgcn_readfirstlane(B.wave);
  const float c = P.c;
  for (int64_t i = 0; i <= P.n_rows; ++i) {
    // (a call of no more rows than workgroups has no counter: one row each)
    const unsigned int ru = P.next_row ? take_next(P.next_row, &sh.next) : i == 0 ? blockIdx.x : ~0u;
    if (ru >= static_cast<unsigned int>(P.n_rows)) break;
    const int64_t r = ru;
    const T* row = static_cast<const T*>(P.s) + r * P.stride;
    G* out = GRAD ? static_cast<G*>(P.grad) + r * P.grad_stride : nullptr;
    const bool part = P.valid ? uniform(P.valid[r] != 0) : true;
    // this thread's entry of the list
    int token = -1;
    float logit = 0.0f;
    if (part && B.tid < k) {
      token = P.token[r * P.list_stride + B.tid];
      if (token >= 0) logit = P.logit[r * P.list_stride + B.tid];
    }
    bool wrong = token < -1 || token >= V;
    const bool held = !wrong && token >= 0;
    const float s_tok = held ? Loader<T>::load1(row + token) : 0.0f;
    wrong |= held && !(logit < finf());
    const float rest = part && P.rest ? P.rest[r] : -finf();
    wrong |= !(rest < finf());
    // the sum over the tokens that are not listed
    float m = -finf(), lo = finf(), hi = -finf();
    double S = 0.0;
    if (part) {
      for (int s0 = 0; s0 < V; s0 += DT_SEG) {
        const int len = min(V - s0, DT_SEG);
        __syncthreads();  // (the mask of the segment, or row, before was read)
        for (int w = B.tid; w < (len + 31) / 32; w += DT_NT) sh.mask[w] = 0u;
        __syncthreads();
        if (held && token >= s0 && token - s0 < len) {
          const uint32_t bit = 1u << ((token - s0) & 31);
          wrong |= (atomicOr(&sh.mask[(token - s0) >> 5], bit) & bit) != 0u;  // listed twice
        }
        __syncthreads();
        const uint8_t* const bits = reinterpret_cast<const uint8_t*>(sh.mask);
        for_chunks1<T, DT_NW>(row + s0, len, wave, lane, [&](auto tail, float* x, uint32_t vm, int ch) {
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
          for (int e = 0; e < EPL; ++e)
            if ((!TAIL || ((vm >> e) & 1u))) {
              lo = fminf(lo, x[e]);
              hi = fmaxf(hi, x[e]);
            }
          if (TAIL || wave_any(listed != 0u)) {
#pragma unroll
            for (int e = 0; e < EPL; ++e)
              if ((TAIL && !((vm >> e) & 1u)) || ((listed >> e) & 1u)) x[e] = -finf();
          }
          float lm = x[0];
#pragma unroll
          for (int e = 1; e < EPL; ++e) lm = fmaxf(lm, x[e]);
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
    // what the listed tokens and the bucket add up to; logarithms in natural units, in 64 bits
    const double c64 = static_cast<double>(c) * LN2_D;
    const float mU = B.max(m);
    const float mP = fmaxf(B.max(held ? s_tok : -finf()), mU);
    const float mT = fmaxf(B.max(held && !wrong ? logit : -finf()), rest);
    const double z = (static_cast<double>(s_tok) - mP) * c64, y = (static_cast<double>(logit) - mT) * c64;
    double v[6];
    v[0] = S > 0.0 ? S * exp((static_cast<double>(m) - mU) * c64) : S;
    v[1] = held ? exp(z) : 0.0;
    v[2] = held && mT > -finf() ? exp(y) : 0.0;
    v[3] = wrong ? 1.0 : 0.0;
    v[4] = lo > -finf() && hi < finf() ? 0.0 : 1.0;
    v[5] = held ? 1.0 : 0.0;
    B.sum(v);
    const double SU = v[0];
    const bool some = mT > -finf(), others = v[5] < static_cast<double>(V);
    const double yR = (static_cast<double>(rest) - mT) * c64, zR = (static_cast<double>(mU) - mP) * c64 + log(SU);
    const double log_t = log(v[2] + (rest > -finf() ? exp(yR) : 0.0)), log_p = log(v[1] + (others ? exp(zR) : 0.0));
    const double lt = y - log_t, lp = z - log_p, ltR = yR - log_t, lpR = zR - log_p;
    const double p = held ? exp(lp) : 0.0, t = held && logit > -finf() ? exp(lt) : 0.0;
    const double pR = others ? exp(lpR) : 0.0, tR = rest > -finf() ? exp(ltR) : 0.0;
    // infinite divergences: forward, a share of the teacher's where the student has no token; reverse, the
    // other way round
    double l[2] = {0.0, 0.0};
    if (held && some) {
      if (P.reverse) {
        l[0] = p > 0.0 ? p * (lp - lt) : 0.0;
        l[1] = logit > -finf() ? 0.0 : 1.0;
      } else {
        l[0] = t > 0.0 ? t * (lt - lp) : 0.0;
      }
    }
    B.sum(l);
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
    const bool take = part && some && !bad && finite;
    const bool nan = part && (bad || !finite);
    if (!take) loss = nan ? __builtin_nan("") : 0.0;
    if (GRAD) {
      const double scale = static_cast<double>(P.grad_scale) * P.inv_tau;
      const double gR = others ? (P.reverse ? pR * (lpR - ltR - loss) : pR - tR) * scale / SU : 0.0;
      const float coef = take ? static_cast<float>(gR) : nan ? nanf_() : 0.0f;
      if (coef == 0.0f || coef != coef) {
        float x[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) x[e] = coef;
        for (int ch = wave; ch < (V + CHUNK - 1) / CHUNK; ch += DT_NW) store_lane<G, true>(out, ch, lane, V, x);
      } else {
        for_chunks1<T, DT_NW>(row, V, wave, lane, [&](auto tail, float* x, uint32_t, int ch) {
          constexpr bool TAIL = decltype(tail)::value;
          float g[EPL];
#pragma unroll
          for (int e = 0; e < EPL; ++e) g[e] = coef * fexp2((x[e] - mU) * c);
          store_lane<G, TAIL>(out, ch, lane, V, g);
        });
      }
      // the listed tokens over it, once the row's stores are done
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (take && held) {
        const double g = P.reverse ? p * (lp - lt - loss) : p - t;
        Storer<G>::store1(out + token, static_cast<float>(g * scale));
      }
    }
    if (B.tid == 0) {
      if (P.row_loss) P.row_loss[r] = static_cast<float>(loss);
      if (P.scaled_loss) P.scaled_loss[r] = static_cast<double>(P.grad_scale) * loss;
      if (P.row_status)
        P.row_status[r] = !part ? SAKI_ROW_OK : !finite ? SAKI_ROW_NONFINITE : bad ? SAKI_ROW_BAD_TARGET : SAKI_ROW_OK;
    }
  }
}

}  // namespace saki
