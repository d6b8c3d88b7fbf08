// Generated by paper_2609_09020_gb300/gen_gelu_grad.py -- do not edit.
// Phi(-a) - a phi(a) ~= 2^(kGeluGradPower a^2) p(a) on 0 <= a <= 6; max error of GELU' in
// fp32 ~ 3.6e-07 (degree 9), 1.2e-07 (degree 11).
// a Phi(-a) ~= 2^(kGeluGradPower a^2) r(a); max error of GELU on |z| < 12, the rounding of the
// result included, ~ 2.5e-07.
#pragma once

namespace pic {

constexpr float kGeluGradA = 6.0f;
constexpr float kGeluGradPower = -0.7213475108146667f;
constexpr int kGeluGradDeg = 9;
constexpr int kGeluGradDeg32 = 11;
constexpr int kGeluDeg32 = 12;

// Coefficients of p and of r, highest degree first (Horner order).
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
__host__ __device__ constexpr float gelu_grad_c32(int i) {
  constexpr float c[] = {
      -3.155438150770351e-07f,
      7.70879523770418e-06f,
      -8.477114170091227e-05f,
      0.0005636534770019352f,
      -0.0025900928303599358f,
      0.009003852494060993f,
      -0.025471823289990425f,
      0.06192393600940704f,
      -0.13280579447746277f,
      0.24997256696224213f,
      -0.7978828549385071f,
      0.4999999701976776f,
  };
  return c[i];
}
__host__ __device__ constexpr float gelu_c32(int i) {
  constexpr float c[] = {
      -1.750784974774433e-07f,
      4.73991076432867e-06f,
      -5.789172791992314e-05f,
      0.00042691887938417494f,
      -0.002159194787964225f,
      0.008129028603434563f,
      -0.024318480864167213f,
      0.06095236539840698f,
      -0.13230448961257935f,
      0.24982641637325287f,
      -0.3989199697971344f,
      0.4999990165233612f,
      0.0f,
  };
  return c[i];
}

}  // namespace pic
