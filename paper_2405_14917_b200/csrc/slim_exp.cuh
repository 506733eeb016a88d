// The exponential of the distillation kernels, which compiles for the host too: its error bound is tested there.
#pragma once

#include <math.h>
#include <stdint.h>
#include <string.h>

#ifdef __CUDACC__
#define SLIM_EXP_FN __host__ __device__ __forceinline__
#else
#define SLIM_EXP_FN inline
#endif

namespace slim {

// e^x in 64 bits for x up to a few (a log-probability), within 1e-14 of its value: x = n ln 2 + r after Cody and Waite (ln 2 = 355 / 512 and a
// rest, so that n times the first is exact), Taylor's series of e^r to the eleventh power (|r| < 0.35: 0.35^12 / 12! < 1e-14) summed in pairs,
// times 2^n.  Half as many dependent steps as a general exp(), which takes what lies beyond.
SLIM_EXP_FN double exp_log(double x) {
    if (x > 80.0) return exp(x);
    if (x < -700.0) return 0.0;
    const double n = rint(x * 1.44269504088896340736);
    double r = fma(n, -355.0 / 512, x);
    r = fma(n, 2.12194440054690582768e-4, r);
    const double r2 = r * r, r4 = r2 * r2;
    const double a = fma(r, 1.0, 1.0), b = fma(r, 1.0 / 6, 1.0 / 2), c = fma(r, 1.0 / 120, 1.0 / 24), d = fma(r, 1.0 / 5040, 1.0 / 720),
                 e = fma(r, 1.0 / 362880, 1.0 / 40320), f = fma(r, 1.0 / 39916800, 1.0 / 3628800);
    const double ab = fma(b, r2, a), cd = fma(d, r2, c), ef = fma(f, r2, e);
    const double y = fma(fma(ef, r4, cd), r4, ab);
#ifdef __CUDA_ARCH__
    return __hiloint2double(__double2hiint(y) + (static_cast<int>(n) << 20), __double2loint(y));
#else
    int64_t bits;
    memcpy(&bits, &y, sizeof bits);
    bits += static_cast<int64_t>(n) * (1ll << 52);
    double r2n;
    memcpy(&r2n, &bits, sizeof r2n);
    return r2n;
#endif
}

}  // namespace slim
