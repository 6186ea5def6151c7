// ops_two.cuh -- numbers of some 45 bits as sums of two 32-bit ones, and exponentials of that
// precision (64-bit arithmetic runs at a sixty-fourth of the 32-bit rate here).  Sums without
// error are Knuth's, where one is the larger Dekker's, as are products and quotients of pairs.
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

// A sum of numbers that are not negative.  Of n of them c is up to n 2^-24 of s and off by half a step n times: n^2 2^-49 of
// the sum at most (2^-33 at 256, where equal ones, the worst that were tried, gave 2^-36.8).
struct LongSum {
    float s = 0, c = 0;
    __device__ __forceinline__ void add(const Two &w)
    {
        const Two t = sum_of(s, w.h);
        s = t.h;
        c += t.l + w.l;
    }
    __device__ __forceinline__ Two value() const { return sum_of(s, c); }
    __device__ __forceinline__ void close(int) {}
    __device__ __forceinline__ Two total() const { return value(); }
};
// One of as many as 2^30: close() after every 32 of them brings c back to half a step of s (512 are off by 2^-35 at most),
// and after 512 puts what there is by, which is off by 2^-47 each time.
struct LongerSum : LongSum {
    Two by{0, 0};
    __device__ __forceinline__ void close(int times)
    {
        const Two t = value();
        s = t.h, c = t.l;
        if (times % 16 == 15) by = by + t, s = c = 0;
    }
    __device__ __forceinline__ Two total() const { return by + value(); }
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

// exp(t + tl) / 2^e, in 1..2 or so, to some 2^-44 of itself (2^-41 at |t| = 256, 2^-39 at 745): with k =
// rint(t 512 / ln 2), t - k ln2 / 512 is exact in its first part (k times the first part of
// ln2 / 512 and t are multiples of 2^-34, the rest is below 2^-10), and its exponential takes three
// terms.  (The second part may be some steps of the first.)
__device__ __forceinline__ Two exp_parts(float t, float tl, const float2 *table, int &k)
{
    constexpr double kStep = 0.693147180559945309417 / PowerTable::kSize;
    constexpr float kPer = (float)(1 / kStep), kStep1 = (float)kStep, kStep2 = (float)(kStep - (double)kStep1), kShift = 12582912.0f;
    const float shifted = __fmaf_rn(t, kPer, kShift), kf = shifted - kShift;
    k = __float_as_int(shifted) - __float_as_int(kShift);
    const Two y = sum_of_larger(__fmaf_rn(-kf, kStep1, t), __fmaf_rn(-kf, kStep2, tl));
    const float more = __fmaf_rn(y.h * y.h, __fmaf_rn(y.h, 1.0f / 6, 0.5f), y.l);
    const float2 p = table[k & (PowerTable::kSize - 1)];
    const float a = p.x * y.h;
    const float b = __fmaf_rn(p.x, y.h, -a) + __fmaf_rn(p.x, more, __fmaf_rn(p.y, y.h, p.y));
    Two w = sum_of_larger(p.x, a);
    w.l += b;
    return w;
}

// (x - m) r in two parts.
__device__ __forceinline__ void exponent_of(float x, float m, const Two &r, float &t, float &tl)
{
    const Two d = sum_of(x, -m);
    t = d.h * r.h;
    tl = __fmaf_rn(d.l, r.h, __fmaf_rn(d.h, r.l, __fmaf_rn(d.h, r.h, -t)));
}

// exp((x - m) r), times a number that is the same for all x: what a row's elements weigh.  m is one of
// the larger x, and none is above it by e^44.  Below e^-64 of m: 0.  Where |m r| is small the
// exponent is x r itself (m's power of two is left out), otherwise x - m in two parts comes first.
struct Weigher {
    static constexpr float kLowest = -64.0f, kDirect = 192.0f;
    Two r;
    float m, low;
    int bias;
    bool direct;
    __device__ __forceinline__ Weigher(float m, const Two &r) : r(r), m(m)
    {
        low = m + __fdiv_rn(kLowest, r.h);
        direct = fabsf(m * r.h) <= kDirect && low > -3e38f;
        bias = direct ? (int)rintf(m * r.h * 1.44269504f) : 0;
    }
    // N of them (the exponents in one place, for the branch).
    template <int N> __device__ __forceinline__ void of(const float (&x)[N], const float2 *table, Two (&w)[N]) const
    {
        float t[N], tl[N];
        bool some[N];
        if (direct) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float a = fmaxf(x[j], low);
                t[j] = a * r.h;
                tl[j] = __fmaf_rn(a, r.l, __fmaf_rn(a, r.h, -t[j]));
                some[j] = x[j] > low;
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                exponent_of(x[j], m, r, t[j], tl[j]);
                // (of -inf, and of differences that are infinite, the second part is NaN)
                some[j] = t[j] > kLowest;
                t[j] = fmaxf(t[j], kLowest), tl[j] = some[j] ? tl[j] : 0.0f;
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            int k;
            w[j] = exp_parts(t[j], tl[j], table, k);
            const float scale = some[j] ? __int_as_float(((k >> PowerTable::kBits) + (127 - bias)) << 23) : 0.0f;
            w[j] = Two{w[j].h * scale, w[j].l * scale};
        }
    }
    __device__ __forceinline__ Two of(float x, const float2 *table) const
    {
        const float a[1] = {x};
        Two w[1];
        of(a, table, w);
        return w[0];
    }
    // w 2^e is the same, however small; false: it is 0, or below e^-745, which 64 bits do not hold.
    __device__ __forceinline__ bool wide(float x, const float2 *table, Two &w, int &e) const
    {
        float t, tl;
        int k;
        exponent_of(x, m, r, t, tl);
        if (direct) {
            // (not in these few bits more, but as `of` does)
            t = x * r.h;
            tl = __fmaf_rn(x, r.l, __fmaf_rn(x, r.h, -t));
        }
        const bool some = x > -INFINITY && (direct ? t - m * r.h : t) > -745.0f;
        w = exp_parts(some ? t : 0.0f, some ? tl : 0.0f, table, k);
        e = (k >> PowerTable::kBits) - bias;
        return some;
    }
};

}  // namespace e2ops
