// What the gradient kernels of both attention stages share: the statistics of a softmax row and their joining, and the
// kernels that add up the records of a user's pieces.
#pragma once

#include "common.hpp"

namespace vista {

// v_exp_f32: one unit of the last place, results below 2^-126 are zero
__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// (m, l, e): a row's largest score (base 2), sum of 2^(s - m) and sum of 2^(s - m) dP over some of its keys; joined with
// those over others.
__device__ __forceinline__ void join_stats(float& m, float& l, float& e, float m2, float l2, float e2) {
  const float top = fmaxf(m, m2), f = exp2_fast(m - top), f2 = exp2_fast(m2 - top);
  l = fmaf(l2, f2, l * f);
  e = fmaf(e2, f2, e * f);
  m = top;
}

// nearest even, NaN kept: gradients, unlike the forward paths' outputs, may be called on non-finite values
__device__ __forceinline__ uint32_t pair_to_bf16(float a, float b) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
  typedef __attribute__((ext_vector_type(2))) float f32x2_t;
  const f32x2_t f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
}
__device__ __forceinline__ void store_grad(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_grad(bf16_t* p, float v) { p->bits = uint16_t(pair_to_bf16(v, 0.f)); }

// Shapes of the joining kernels.
struct GradRows {
  const int64_t* offsets;
  int B, S, d, H, seg;
  int64_t N, G;
  float scale, scale_log2;
  int64_t q_user_stride;
  int64_t check;          // N: check the offsets on the device; -1: the host has
  int* status;
};

// Records of row statistics [slot][H][rows][3] -> lse (base 2) and delta, [B][H][S] each; slot = segment + user.
// Ks, Vs (else null): fp32 keys and values of the seeds' own, whose score joins the row; own_p and own_ds then receive its
// probability and gradient, [B][H][S].
hipError_t grad_join_stats(const GradRows& r, int dtype, const float* stats, int rows, float* lse, float* delta, const void* Q,
                           const void* dO, const float* Ks, const float* Vs, float* own_p, float* own_ds, hipStream_t s);

// Records [slot][H][rows][dh] of sum dS K -> dQ = factor sum, and with Ks the own key's part and the gradients of
// own keys and values.
hipError_t grad_join_queries(const GradRows& r, int dtype, const float* records, int rows, float factor, const void* Q,
                             const void* dO, const float* Ks, const float* own_p, const float* own_ds, void* d_queries,
                             void* d_self_keys, void* d_self_values, hipStream_t s);

// Records [share][B][H][S][dh] -> d_summaries [B][S][d]
hipError_t grad_join_shares(int dtype, const float* records, int shares, int64_t B, int S, int d, int H, void* d_summ,
                            hipStream_t s);

}  // namespace vista
