// Host-side check of exp2.h against 80-bit arithmetic. Built and run by
// tests/test_exp2.py on the CPU.
#include <cmath>
#include <cstdio>
#include <random>

#include "exp2.h"

int main() {
    std::mt19937_64 rng(260708973);
    std::uniform_real_distribution<double> frac(-0.5, 0.5), wide(-1020.0, 1020.0);
    long double worst = 0, worst9 = 0;
    const auto see = [&](double t) {
        const long double want = exp2l(static_cast<long double>(t));
        const long double e = fabsl(static_cast<long double>(sifar::exp2_64(t)) / want - 1);
        if (e > worst) worst = e;
        if (t < -1000 || t > 0) return;
        const long double want3 = exp2l(static_cast<long double>(t / 3.0) * 3);
        const long double q = sifar::exp2_quick<0>(t / 3.0, 3.0) / want3;
        const long double s = ldexpl(sifar::exp2_quick<42>(t, 1.0), -42) / want;
        worst9 = fmaxl(worst9, fmaxl(fabsl(q - 1), fabsl(s - 1)));
    };
    for (int i = 0; i < 2000000; ++i) {
        see(frac(rng));
        see(wide(rng));
    }
    for (int i = -1020; i <= 1020; ++i) {
        if (sifar::exp2_64(i) != std::ldexp(1.0, i)) return std::printf("2^%d\n", i), 1;
        see(i + 0.5);
        see(std::nextafter(i + 0.5, 0.0));
        if (i <= 0 && i >= -1000 && sifar::exp2_quick<42>(i, 1.0) != std::ldexp(1.0, i + 42))
            return std::printf("2^%d quick\n", i), 1;
    }
    for (double y : {0.0, -0.5, -59.3, -999.0}) {
        const double a = sifar::exp2_quick<0>(y, 1.0, false);
        const double b = sifar::exp2_quick<42>(y, 1.0, false);
        if (!(a > 0 && a < 0x1p-900 && b > 0 && b < 0x1p-900))
            return std::printf("left out\n"), 1;
    }
    std::printf("%.3Le %.3Le\n", worst, worst9);
    return worst < 3e-16L && worst9 < 4e-14L ? 0 : 1;
}
