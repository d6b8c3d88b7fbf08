// Generated by paper_2609_09020_gb300/gen_gelu_grad.py -- do not edit.
// Phi(-a) - a phi(a) ~= 2^(kGeluGradPower a^2) p(a) on 0 <= a <= 6; max error of GELU' in
// fp32 ~ 3.6e-07.
#pragma once

namespace pic {

constexpr float kGeluGradA = 6.0f;
constexpr float kGeluGradPower = -0.7213475108146667f;
constexpr int kGeluGradDeg = 9;

// Coefficients of p, highest degree first (Horner order).
__host__ __device__ constexpr float gelu_grad_c(int i) {
  constexpr float c[] = {
      -8.06307161838049e-06f,
      0.00015194190200418234f,
      -0.0012711621820926666f,
      0.006382806226611137f,
      -0.022230878472328186f,
      0.05949679762125015f,
      -0.13177289068698883f,
      0.24975229799747467f,
      -0.7978649139404297f,
      0.4999997317790985f,
  };
  return c[i];
}

}  // namespace pic
