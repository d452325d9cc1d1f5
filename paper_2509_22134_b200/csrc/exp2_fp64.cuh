// 2^x in fp64, for the weights of a distribution.
#pragma once

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

}  // namespace gto
