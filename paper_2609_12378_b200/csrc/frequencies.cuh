// Frequencies of position tables: the angle per position of every pair over pi, as an unevaluated sum of two doubles.  A position of up to 2^50
// multiplies a frequency's error, so the power, the scalings and the division by pi are carried to at least 99 bits (the most that was seen is
// 2^-103.7): no angle up to there is off by more than 2^-52 for it.  Host code in integers and doubles: 64 pairs in 1.0 us, as long as 64 calls of
// pow, and in 1.7 to 2.4 us where pairs are blended.
#pragma once
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "../../include/ckks_b200.h"

namespace freq {

typedef unsigned __int128 u128;

// ---- numbers i + f 2^-128 ------------------------------------------------------------------------------------------------
struct Fixed { uint64_t i; u128 f; };
inline u128 mul_hi(u128 a, u128 b) {                     // a b 2^-128, rounded down
    const uint64_t ah = (uint64_t)(a >> 64), al = (uint64_t)a, bh = (uint64_t)(b >> 64), bl = (uint64_t)b;
    const u128 x = (u128)ah * bl, y = (u128)al * bh;
    const u128 mid = (u128)(uint64_t)x + (uint64_t)y + (uint64_t)(((u128)al * bl) >> 64);
    return (u128)ah * bh + (x >> 64) + (y >> 64) + (mid >> 64);
}
inline Fixed over(Fixed a, uint32_t k) {
    Fixed q;
    q.i = a.i / k;
    const u128 h = ((u128)(a.i % k) << 64) | (uint64_t)(a.f >> 64), l = ((u128)(uint64_t)(h % k) << 64) | (uint64_t)a.f;
    q.f = ((u128)(uint64_t)(h / k) << 64) | (uint64_t)(l / k);
    return q;
}
inline Fixed plus(Fixed a, Fixed b) {
    const u128 f = a.f + b.f;
    return Fixed{a.i + b.i + (f < a.f), f};
}
inline Fixed minus(Fixed a, Fixed b) { return Fixed{a.i - b.i - (a.f < b.f), a.f - b.f}; }
inline bool less(Fixed a, Fixed b) { return a.i < b.i || (a.i == b.i && a.f < b.f); }
constexpr u128 LN2 = ((u128)0xb17217f7d1cf79abull << 64) | 0xc9e3b39803f2f6afull;
inline Fixed ln2_times(uint32_t k) {
    const u128 lo = (u128)(uint64_t)LN2 * k, hi = (LN2 >> 64) * k + (lo >> 64);
    return Fixed{(uint64_t)(hi >> 64), ((u128)(uint64_t)hi << 64) | (uint64_t)lo};
}

// e^(-x 2^-128): the series of e^(-x / 256), whose terms alternate and shrink by more than 2^8 each, squared eight times.  Fourteen terms leave
// 2^-149; the squarings turn the series' rounding of a few units into at most 2^-117.
constexpr u128 ONE = ~(u128)0;
constexpr u128 INVERSE[15] = {0, ONE, ONE / 2, ONE / 3, ONE / 4, ONE / 5, ONE / 6, ONE / 7, ONE / 8, ONE / 9, ONE / 10, ONE / 11, ONE / 12, ONE / 13, ONE / 14};
inline u128 exp_minus(u128 x) {
    const u128 r = x >> 8;
    u128 t = ONE;
    for (uint32_t k = 14; k; k--) t = ONE - mul_hi(mul_hi(r, INVERSE[k]), t);
    for (uint32_t k = 0; k < 8; k++) t = mul_hi(t, t);
    return t;
}
// ln x of a finite x >= 1, within 2^-115: x = f 2^e with f in [1/2, 1), and -ln f is its double plus ln(e^(-that) / f), a number of 2^-51
// whose series needs two terms
inline Fixed ln(double x) {
    if (x == 1.0) return Fixed{0, 0};
    int e, ey;
    const double f = frexp(x, &e), y = -log(f), g = frexp(y, &ey);            // 2^-53 < y < 1, so Y is exact
    const u128 F = (u128)(uint64_t)ldexp(f, 53) << 75, Y = (u128)(uint64_t)ldexp(g, 53) << (75 + ey);
    const __int128 d = (__int128)(exp_minus(Y) - F);
    const double q = (double)d / f;
    __int128 c = (__int128)q;
    const __int128 m = c < 0 ? -(__int128)mul_hi((u128)-c, F) : (__int128)mul_hi((u128)c, F);
    c += (__int128)((double)(d - m) / f);
    c -= (__int128)(ldexp(q, -129) * q);
    return minus(ln2_times((uint32_t)e), Fixed{0, Y + (u128)c});
}
inline double approx(Fixed a) { return (double)a.i + ldexp((double)a.f, -128); }

// ---- numbers m 2^-128 2^-e, m in [2^127, 2^128) -------------------------------------------------------------------------------
struct Scaled { u128 m; int64_t e; };
inline Scaled normal(u128 m, int64_t e) {
    const uint32_t k = (uint32_t)__builtin_clzll((uint64_t)(m >> 64));          // products of two such numbers: at most one
    return Scaled{m << k, e + k};
}
inline Scaled exp_minus(Fixed x) {
    uint32_t k = (uint32_t)(approx(x) / 0.6931471805599453);
    while (k && less(x, ln2_times(k))) k--;
    const Fixed r = minus(x, ln2_times(k));           // below ln 2, or above it by the estimate's rounding
    return normal(exp_minus(r.f), k);
}
inline Scaled times(Scaled a, Scaled b) { return normal(mul_hi(a.m, b.m), a.e + b.e); }

// ---- unevaluated sums of two doubles -------------------------------------------------------------------------------------
struct Pair { double h, l; };
inline Pair quick_sum(double a, double b) { const double s = a + b; return Pair{s, b - (s - a)}; }
inline Pair sum(double a, double b) {
    const double s = a + b, t = s - a;
    return Pair{s, (a - (s - t)) + (b - t)};
}
inline Pair add(Pair a, Pair b) {
    const Pair s = sum(a.h, b.h), t = sum(a.l, b.l), u = quick_sum(s.h, s.l + t.h);
    return quick_sum(u.h, u.l + t.l);
}
inline Pair neg(Pair a) { return Pair{-a.h, -a.l}; }
inline Pair mul(Pair a, Pair b) {
    const double p = a.h * b.h;
    return quick_sum(p, fma(a.h, b.h, -p) + (a.h * b.l + a.l * b.h));
}
inline Pair div(Pair a, Pair b) {
    const double q0 = a.h / b.h;
    Pair r = add(a, neg(mul(b, Pair{q0, 0.0})));
    const double q1 = r.h / b.h;
    r = add(r, neg(mul(b, Pair{q1, 0.0})));
    const Pair q = quick_sum(q0, q1);
    return add(q, Pair{r.h / b.h, 0.0});
}
inline Pair number(double x) { return Pair{x, 0.0}; }
inline Pair pair_of(Scaled a) {             // the upper 53 bits and 63 of the others
    const double h = (double)(int64_t)(a.m >> 75), l = (double)(int64_t)((uint64_t)(a.m >> 12) & ~(1ull << 63)) * 0x1p-63;
    const int64_t e = -53 - a.e;
    if (e <= -900) return quick_sum(ldexp(h, (int)e), ldexp(l, (int)e));
    const uint64_t bits = (uint64_t)(1023 + e) << 52;
    double unit;
    memcpy(&unit, &bits, sizeof(unit));
    return quick_sum(h * unit, l * unit);
}

}  // namespace freq

// hi, lo [rot_dim / 2]: angle per position over pi of every pair.  The descriptor has been checked (ckks_rotary_table).
inline void rotary_frequencies(const ckks_rotary_scaling &f, double few, double many, double *hi, double *lo) {
    using namespace freq;
    const Pair inv_pi{0.318309886183790671538, -1.96786766751824869e-17}, one = number(1.0), length = number(f.original_length);
    const uint32_t half = f.rot_dim / 2;
    const double rot = f.rot_dim;
    Fixed log_theta = ln(f.theta);
    if (f.kind == CKKS_ROTARY_BASE) {                // factor^(rot / (rot - 2)) = factor factor^(1 / (half - 1))
        const Fixed g = ln(f.factor);
        log_theta = plus(log_theta, plus(g, over(g, half - 1)));
    }
    double ramp_lo = 0.0, ramp_hi = 0.0;
    if (f.kind == CKKS_ROTARY_RAMP) {          // pair index at which a wavelength turns `many`, `few` times within the trained length
        ramp_lo = fmax(0.0, floor(rot * log(f.original_length / (many * 2.0 * M_PI)) / (2.0 * log(f.theta))));
        ramp_hi = fmin(rot - 1.0, ceil(rot * log(f.original_length / (few * 2.0 * M_PI)) / (2.0 * log(f.theta))));
    }
    const bool divided = f.kind == CKKS_ROTARY_LINEAR || f.kind == CKKS_ROTARY_BANDS || f.kind == CKKS_ROTARY_RAMP;
    const Pair inv_factor = divided ? div(one, number(f.factor)) : one;
    // the part of a pair that is not divided, where it is neither none nor all of it: num / den
    const Pair den = f.kind == CKKS_ROTARY_BANDS ? sum(many, -few) : number(fmax(ramp_hi - ramp_lo, 0.001)), inv_den = div(one, den);
    const Pair turn{0.5 * inv_pi.h, 0.5 * inv_pi.l};
    const Scaled step = exp_minus(over(log_theta, half));
    Scaled w = step;
    for (uint32_t j = 0; j < half; j++) {
        Pair a = one;
        if (j) {
            if (j > 1) w = times(w, step);
            a = pair_of(w);
        }
        if (f.kind == CKKS_ROTARY_LINEAR) {
            a = mul(a, inv_factor);
        } else if (divided) {
            const Pair num = f.kind == CKKS_ROTARY_BANDS ? add(mul(mul(length, a), turn), number(-few)) : add(den, number(ramp_lo - (double)j));
            const Pair rest = add(den, neg(num));
            if (num.h <= 0.0) {
                a = mul(a, inv_factor);
            } else if (rest.h > 0.0) {
                // (one over a bound's distance next to the smallest double is no number)
                const Pair kept = isfinite(inv_den.h) ? mul(num, inv_den) : number(num.h / den.h), gone = isfinite(inv_den.h) ? mul(rest, inv_den) : number(rest.h / den.h);
                a = add(mul(kept, a), mul(gone, mul(a, inv_factor)));
            }
        }
        a = mul(a, inv_pi);
        hi[j] = a.h;
        lo[j] = a.l;
    }
}
