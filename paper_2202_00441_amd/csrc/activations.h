// activations.h -- GELU and SiLU in fp32, for every kernel that forms them: the few-bit
// forwards and the epilogue of the product in 8-bit integers.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/fewbit.h"

namespace {      // each source has its own

// ---------------------------------------------------------------- activations
// f evaluated in fp32 with hardware exp2 / reciprocal.  x*Phi(x) and
// x*sigmoid(x) are formed as relu(x) - |x| * tail(|x|), tail the upper tail
// probability, which keeps full relative accuracy on the negative side down
// to the subnormals.
//
// The hardware exponential returns no subnormals (results below 2^-126 come
// back as 0), so each exponential is taken of an argument raised by S and
// the factor 2^S is taken back out of the partner operand of the final
// product, which costs nothing: for GELU out of the reciprocal (its
// constants carry 2^S), for SiLU and sigmoid out of the denominator.  S is
// the smallest shift that keeps every product representable in the output
// type (fp16 outputs underflow long before 2^-126, so S = 0 there).
//
// In the product |x| * tail, |x| is clamped to the largest finite float:
// for x = +-inf the other factor is exactly 0 and the product is 0 (not
// inf * 0), so f(x) = relu(x) without a separate branch; NaN still reaches
// the result through the exponential's argument, which is not clamped.
__device__ inline float finite_abs(float x) { return fminf(fabsf(x), 3.4028234663852886e38f); }

// max(x, -0) as one integer op: the unsigned minimum with the bits of -0
// keeps every float with the sign bit clear (+inf, NaN included) and maps
// every negative input to -0.
__device__ inline float relu(float x) {
  return __uint_as_float(min(__float_as_uint(x), 0x80000000u));
}

// 2^e for -1022 <= e <= 1023, from the exponent field
constexpr double pow2(int e) {
  return __builtin_bit_cast(double, static_cast<uint64_t>(1023 + e) << 52);
}

template <int N>
struct Coefs {
  float c[N];
};

// GELU: the normal upper tail Q(t) = P(Z > t) = r exp2(c(r) - t^2/(2 ln 2))
// with r = 1/(1 + p t) and c a polynomial in r (the form of the Chebyshev
// fitted erfc of Numerical Recipes, coefficients fitted here for a minimal
// maximum relative error on t in [0, 15]):
//   degree 3: max rel. error 1.9e-4  (bf16 results: within 1 ulp)
//   degree 4: max rel. error 5.5e-5  (fp16 results: within 1 ulp)
//   degree 6: max rel. error 1.3e-6  (fp32 results: within 1e-5 rel / 2e-6 abs)
template <int DEG>
struct QFit;
template <>
struct QFit<3> {
  static constexpr float p = 0.36950944455033363f;
  static constexpr float c[4] = {-2.7541667327185095f, 1.3469623570975156f,
                                 0.9101290363759839f, -0.5032013588354882f};
};
template <>
struct QFit<4> {
  static constexpr float p = 0.5063964087913556f;
  static constexpr float c[5] = {-2.3043683184461905f, 1.3894173139728148f,
                                 0.6817571899264395f, -1.149862878045882f,
                                 0.38313433006936115f};
};
template <>
struct QFit<6> {
  static constexpr float p = 0.2715552190762726f;
  static constexpr float c[7] = {-3.204975453658058f, 1.4179583422514952f,
                                 0.7853715466157367f, -0.343943261631901f,
                                 1.2761535905064931f, -1.3184075229241483f,
                                 0.3878445554240053f};
};

// Per output type: GELU polynomial degree and the exponent shifts S.
template <int DT>
struct Prec {                       // fp32
  static constexpr int kGeluDeg = 6, kGeluS = 20, kSiluS = 32, kSigmoidS = 24;
};
template <>
struct Prec<FEWBIT_BF16> {
  static constexpr int kGeluDeg = 3, kGeluS = 16, kSiluS = 16, kSigmoidS = 16;
};
template <>
struct Prec<FEWBIT_F16> {
  static constexpr int kGeluDeg = 4, kGeluS = 0, kSiluS = 0, kSigmoidS = 0;
};

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kHalfLog2e = 0.7213475204444817f;   // 1/(2 ln 2)

template <int DT, int ACT>
struct Act;

template <int DT>
struct Act<DT, FEWBIT_GELU> {
  static constexpr int D = Prec<DT>::kGeluDeg, S = Prec<DT>::kGeluS;
  using F = QFit<D>;
  // coefficients of c in r' = 2^-S r: c_i 2^(S i), and c_0 + S (evaluated
  // at compile time: constant-initialised)
  static constexpr Coefs<D + 1> kCoef = [] {
    Coefs<D + 1> a{};
    for (int i = 0; i <= D; ++i)
      a.c[i] = i == 0 ? F::c[0] + static_cast<float>(S)
                      : static_cast<float>(static_cast<double>(F::c[i]) * pow2(S * i));
    return a;
  }();
  static constexpr float kP = static_cast<float>(F::p * pow2(S));
  static constexpr float kScale = static_cast<float>(pow2(S));
  __device__ static float f(float x) {
    const float t = finite_abs(x);
    const float rs = __builtin_amdgcn_rcpf(fmaf(t, kP, kScale));   // 2^-S r
    float c = kCoef.c[D];
#pragma unroll
    for (int i = D - 1; i >= 0; --i) c = fmaf(c, rs, kCoef.c[i]);
    const float e = __builtin_amdgcn_exp2f(fmaf(x * x, -kHalfLog2e, c));    // 2^S Q(t) / r
    return fmaf(-(t * rs), e, relu(x));   // relu(x) - t Q(t); NaN via x*x
  }
};

template <int DT>
struct Act<DT, FEWBIT_SILU> {
  static constexpr int S = Prec<DT>::kSiluS;
  __device__ static float f(float x) {
    const float e = __builtin_amdgcn_exp2f(fmaf(fabsf(x), -kLog2e, static_cast<float>(S)));  // 2^S e^-t
    constexpr float kScale = static_cast<float>(pow2(S));
    const float r = __builtin_amdgcn_rcpf(e + kScale);  // 1/(2^S (1 + e^-t))
    return fmaf(-(finite_abs(x) * e), r, relu(x));    // relu(x) - t sigma(-t); NaN via e
  }
};

// SiLU, fp16 outputs: x sigma(x) = x / (1 + e^-x) directly.  fp16 outputs
// below 2^-25 round to 0, long before e^-x overflows (x < -88), so the
// negative tail needs neither the split above nor a shift; x is raised to
// -FLT_MAX so that -inf gives -FLT_MAX * 0 = -0 (the limit), and a NaN still
// reaches the result through the exponential.  Six instructions instead of
// eight; every fp16 pattern within one unit in the last place.
template <>
struct Act<FEWBIT_F16, FEWBIT_SILU> {
  __device__ static float f(float x) {
    const float r = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -kLog2e));
    return fmaxf(x, -3.4028234663852886e38f) * r;
  }
};

}  // namespace
