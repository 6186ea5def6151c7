// ops_two.cuh -- numbers of some 45 bits as sums of two 32-bit ones, and exponentials of that
// precision (64-bit arithmetic runs at a sixty-fourth of the 32-bit rate here).
#pragma once

#include "ops_common.cuh"

namespace e2ops {

struct Two {
    float h, l;                          // l: at most half a step of h, some steps where it says so
};

// (a + b exactly; the shorter form where |a| >= |b|, or a is 0)
__device__ __forceinline__ Two sum_of(float a, float b)
{
    const float s = a + b, t = s - a;
    return Two{s, (a - (s - t)) + (b - t)};
}
__device__ __forceinline__ Two sum_of_larger(float a, float b)
{
    const float s = a + b;
    return Two{s, b - (s - a)};
}
__device__ __forceinline__ Two operator+(const Two &a, const Two &b)
{
    const Two s = sum_of(a.h, b.h);
    return sum_of_larger(s.h, s.l + (a.l + b.l));
}
__device__ __forceinline__ Two operator-(const Two &a) { return Two{-a.h, -a.l}; }
__device__ __forceinline__ Two operator-(const Two &a, const Two &b) { return a + -b; }
__device__ __forceinline__ Two operator*(const Two &a, const Two &b)
{
    const float p = a.h * b.h;
    return sum_of_larger(p, __fmaf_rn(a.h, b.h, -p) + __fmaf_rn(a.h, b.l, a.l * b.h));
}
__device__ __forceinline__ Two operator/(const Two &a, const Two &b)
{
    const float q = __fdiv_rn(a.h, b.h);
    const Two r = a - Two{q, 0} * b;
    return sum_of_larger(q, __fdiv_rn(r.h, b.h));
}
// (of numbers whose second part is at most half a step of the first)
__device__ __forceinline__ bool operator<(const Two &a, const Two &b) { return a.h < b.h || (a.h == b.h && a.l < b.l); }

__device__ __forceinline__ Two shuffle_xor(const Two &a, int k)
{
    return Two{__shfl_xor_sync(~0u, a.h, k), __shfl_xor_sync(~0u, a.l, k)};
}
// The sum over a warp, the same in all lanes.
__device__ __forceinline__ Two warp_sum(Two a)
{
#pragma unroll
    for (int k = 1; k < 32; k *= 2) a = a + shuffle_xor(a, k);
    return a;
}
// Lane i: the sum of lanes 0..i.
__device__ __forceinline__ Two warp_prefix(Two a, int lane)
{
#pragma unroll
    for (int k = 1; k < 32; k *= 2) {
        const Two b{__shfl_up_sync(~0u, a.h, k), __shfl_up_sync(~0u, a.l, k)};
        if (lane >= k) a = b + a;
    }
    return a;
}

// A long sum of numbers that are not negative.
struct LongSum {
    float s = 0, c = 0;
    __device__ __forceinline__ void add(const Two &w)
    {
        const Two t = sum_of(s, w.h);
        s = t.h;
        c += t.l + w.l;
    }
    __device__ __forceinline__ Two value() const { return sum_of(s, c); }
};

// 2^(j / 512), j < 512, in two parts, from the exponential's series; made by the host's compiler.
struct PowerTable {
    static constexpr int kBits = 9, kSize = 1 << kBits;
    float2 v[kSize];
    constexpr PowerTable() : v{}
    {
        for (int j = 0; j < kSize; ++j) {
            const double x = 0.693147180559945309417 * j / kSize;
            double term = 1, sum = 1;
            for (int n = 1; n < 24; ++n) {
                term = term * x / n;
                sum += term;
            }
            v[j].x = (float)sum;
            v[j].y = (float)(sum - v[j].x);
        }
    }
};

// exp((x - m) r) / 2^e, x <= m, r > 0, in 1..2, to some 2^-44 of itself (2^-39 near e^-745); false
// where it is at most e^lowest.  With t = (x - m) r in two parts and k = rint(t 512 / ln 2), t - k
// ln2 / 512 is exact in its first part (k times the first part of ln2 / 512 and t are multiples of
// 2^-34, the rest is below 2^-10), and its exponential takes three terms.  (The second part may be
// some steps of the first.)
constexpr float kLowestExp = -64.0f, kLowestWideExp = -745.0f;
__device__ __forceinline__ bool exp_parts(float x, float m, const Two &r, const float2 *table, float lowest, Two &w, int &e)
{
    constexpr double kStep = 0.693147180559945309417 / PowerTable::kSize;
    constexpr float kPer = (float)(1 / kStep), kStep1 = (float)kStep, kStep2 = (float)(kStep - (double)kStep1), kShift = 12582912.0f;
    const Two d = sum_of(x, -m);
    const float t = d.h * r.h;
    const float tl = __fmaf_rn(d.l, r.h, __fmaf_rn(d.h, r.l, __fmaf_rn(d.h, r.h, -t)));
    const float shifted = __fmaf_rn(fmaxf(t, lowest), kPer, kShift), kf = shifted - kShift;
    const int k = __float_as_int(shifted) - __float_as_int(kShift);
    const Two y = sum_of_larger(__fmaf_rn(-kf, kStep1, t), __fmaf_rn(-kf, kStep2, tl));
    const float more = __fmaf_rn(y.h * y.h, __fmaf_rn(y.h, 1.0f / 6, 0.5f), y.l);
    const float2 p = table[k & (PowerTable::kSize - 1)];
    const float a = p.x * y.h;
    const float b = __fmaf_rn(p.x, y.h, -a) + __fmaf_rn(p.x, more, __fmaf_rn(p.y, y.h, p.y));
    w = sum_of_larger(p.x, a);
    w.l += b;
    e = k >> PowerTable::kBits;
    return t > lowest;                   // (of -inf, and of differences that are infinite, the parts are NaN)
}
// The same whole, 0 below e^-64.
__device__ __forceinline__ Two exp_of(float x, float m, const Two &r, const float2 *table)
{
    Two w;
    int e;
    const bool some = exp_parts(x, m, r, table, kLowestExp, w, e);
    const float scale = __int_as_float((e + 127) << 23);
    return some ? Two{w.h * scale, w.l * scale} : Two{0, 0};
}

}  // namespace e2ops
