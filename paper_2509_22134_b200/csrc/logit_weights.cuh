// Weights of a row of logits, for the kernels that draw tokens.
#pragma once

#include "gto_common.cuh"

namespace gto {

// 2^x in fp64 for x <= 4, without branches, so that several run side by side (the library's exp took
// 300 cycles each, one after the other): Cody and Waite's reduction x = n + f, |f| <= 1/2, and the
// polynomial of degree 10 with the least largest relative error there (by Remez's exchange:
// 2.1e-16; 4.2e-16 in fp64).  Below 2^-1000 the result is 0; NaN gives NaN.
__device__ __forceinline__ double exp2_neg(double x) {
  const double t = x + 6755399441055744.0;  // 1.5 * 2^52: n in the low bits
  const double f = x - (t - 6755399441055744.0);
  double y = 7.0372933257405244e-09;
  y = fma(y, f, 1.0208538304121812e-07);
  y = fma(y, f, 1.321566273860974e-06);
  y = fma(y, f, 1.5252658114109489e-05);
  y = fma(y, f, 0.00015403529961352815);
  y = fma(y, f, 0.0013333558228566251);
  y = fma(y, f, 0.0096181291080343918);
  y = fma(y, f, 0.055504108664458804);
  y = fma(y, f, 0.24022650695908768);
  y = fma(y, f, 0.69314718055994973);
  y = fma(y, f, 1.0);
  const double r = __hiloint2double(__double2hiint(y) + (__double2loint(t) << 20), __double2loint(y));
  return x < -1000.0 ? 0.0 : r;
}

// The largest of 16 bytes of logits, of two packed 16-bit ones at a time; NaN if one of them is.
template <typename T>
__device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
  uint32_t d;
  if (T::kBytes == 4) asm("max.NaN.f32 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else if (T::kNegInfElem == 0xff80u) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
template <typename T>
__device__ __forceinline__ uint32_t max_of(const uint4& v) {
  return max_word<T>(max_word<T>(v.x, v.y), max_word<T>(v.z, v.w));
}
template <typename T>
__device__ __forceinline__ float max_half(uint32_t w) {  // of the word's two halves
  if (T::kBytes == 4) return __uint_as_float(w);
  w = max_word<T>(w, __byte_perm(w, w, 0x1032));
  return T::load1(&w, 0);
}

// The least, likewise (NaN does not count).
template <typename T>
__device__ __forceinline__ uint32_t min_word(uint32_t a, uint32_t b) {
  uint32_t d;
  if (T::kBytes == 4) asm("min.f32 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else if (T::kNegInfElem == 0xff80u) asm("min.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else asm("min.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
template <typename T>
__device__ __forceinline__ uint32_t min_of(const uint4& v) {
  return min_word<T>(min_word<T>(v.x, v.y), min_word<T>(v.z, v.w));
}
template <typename T>
__device__ __forceinline__ float min_half(uint32_t w) {  // of the word's two halves
  if (T::kBytes == 4) return __uint_as_float(w);
  w = min_word<T>(w, __byte_perm(w, w, 0x1032));
  return T::load1(&w, 0);
}

// Sum of the weights of 16 bytes of logits, 2^((f - m) c2), in fp32: pairs side by side.
template <typename T>
__device__ __forceinline__ float weights(const uint4& v, float m, float c2) {
  constexpr int E = T::kPerVec;
  float f[E];
  T::unpack(v, f);
  uint64_t neg, scale, sum[E / 2];
  asm("mov.b64 %0, {%1, %1};" : "=l"(neg) : "f"(-m));
  asm("mov.b64 %0, {%1, %1};" : "=l"(scale) : "f"(c2));
#pragma unroll
  for (int e = 0; e < E / 2; ++e) {
    float a, b;
    asm("{\n .reg .b64 x;\n mov.b64 x, {%2, %3};\n add.rn.f32x2 x, x, %4;\n mul.rn.f32x2 x, x, %5;\n mov.b64 {%0, %1}, x;\n}"
        : "=f"(a), "=f"(b)
        : "f"(f[2 * e]), "f"(f[2 * e + 1]), "l"(neg), "l"(scale));
    a = ex2_approx(a);
    b = ex2_approx(b);
    asm("mov.b64 %0, {%1, %2};" : "=l"(sum[e]) : "f"(a), "f"(b));
  }
#pragma unroll
  for (int w = E / 4; w > 0; w /= 2)
#pragma unroll
    for (int e = 0; e < w; ++e) asm("add.rn.f32x2 %0, %1, %2;" : "=l"(sum[e]) : "l"(sum[e]), "l"(sum[e + w]));
  float a, b;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(sum[0]));
  return a + b;
}

// ---- shared memory of the CTAs of a cluster
__device__ __forceinline__ uint32_t smem_of(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, int cta) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(cta));
  return r;
}

}  // namespace gto
