// logit_cap.cuh -- scores <q, k> to capped logits in the log2 domain:
//   x = cap_log2 * tanh(u),  u = to_cap * <q, k>,
//   cap_log2 = cap * log2(e), to_cap = sm_scale / cap (times the kv head's K
//   scale with e4m3 KV).
//
// Mathematics.  Where |u| < kCapSeries, tanh(u) = u (1 + t (a1 + a2 t + a3 t^2)),
// t = u^2, with coefficients fitted here for the least maximum relative error
// (1.2e-7 before rounding, 1.8e-7 in fp32): the logit keeps the relative
// accuracy of the plain product, so a cap far above the scores costs nothing.
// Elsewhere tanh(u) = 1 - 2 / (1 + e^(2u)), whose absolute error of about 2e-7
// is at most 5e-7 of tanh(kCapSeries).  With caps above kCapFreeLog2 every score
// takes the form its own size asks for; below, where that error is 1e-5 at most, a
// block with a large score takes the exponential for all of them.
//
// A cap also bounds the logits, so where 2^cap_log2 leaves fp32 and bf16 room
// (kCapFreeLog2) the softmax needs no maximum: P = 2^x, l = sum 2^x, with the
// partials' reference m = 0.  There is then no pass over the scores before the
// exponentials, no rescaling of O, and no order in which P has to wait.  f16 P
// (e4m3 KV) has no such range, and larger caps have none either: they keep the
// running maximum (kCapRef).
//
// What bounds it: the softmax warps' instructions (their issue, and their fetch:
// long unrolled loops run no faster than they are fetched).  The series is 6
// packed instructions per two scores and no MUFU; the exponential form adds an
// exponential per score and a reciprocal per two.  Models keep nearly all logits
// far below their cap, so a warp votes: if no score of the block reaches
// kCapSeries, it runs the series alone.
//
// Measured, one GB300, uncapped -> capped with scores of N(0, 1) -> with scores 8
// times that, at a cap of 50: 16 trials of a request 30.6 -> 31.6 -> 32.6 us; 128
// branches of a 32k prefix 130 -> 144 -> 186; 64 branches in e4m3 97 -> 127 -> 170;
// join prefill 509 -> 626 -> 783, in e4m3 662 -> 894 -> 1142; fork prefill 39 -> 49 ->
// 58.  In 4 bits, uncapped -> capped with scores of N(0, 1): 16 trials 22.1 -> 24.2, 64
// branches of 8192 tokens 113 -> 124, 128 branches of a 32k prefix 99 -> 124, the join 587
// -> 894, the fork 49 -> 64.  The compiler's tanhf for every score took 45 us for the 16 trials and 1687
// for the join.
//
// A NaN score makes its row NaN, as it does without a cap.  The exponential form
// shares a reciprocal between two scores, so they are of one row, or the NaN is cut
// in it and put back (CUT).
#pragma once

#include "device_common.cuh"
#include "tile_common.cuh"

namespace parason {
namespace {

// what an attention kernel does to its logits
enum : int { kCapNone = 0, kCapFree = 1, kCapRef = 2 };
// 2^73 is what a cap of 50 needs; sums of 2^20 tokens stay finite for |v| to 2^34.
// (The join takes 626 us below and 825 above, 128 branches of a 32k prefix 144 and 180.)
constexpr float kCapFreeLog2 = 73.f;

constexpr float kCapSeries = 0.4f;
constexpr float kCapA1 = -0.33331882f, kCapA2 = 0.13277629f, kCapA3 = -0.047794217f;

__device__ __forceinline__ float fast_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The factors of one item's scores, in both halves of packed pairs.
struct CapFactors {
    unsigned long long to_cap;           // u = to_cap <q, k>
    unsigned long long c0, a1, a2, a3;   // cap_log2, and the series' coefficients times it
    unsigned long long two_u;            // two_u <q, k> = 2 u log2(e)
    float to, cap;
    __device__ __forceinline__ CapFactors(float to_, float cap_) : to(to_), cap(cap_) {
        const float w = 2.f * 1.4426950408889634f * to;
        to_cap = dev::f32x2(to, to);
        c0 = dev::f32x2(cap, cap);
        a1 = dev::f32x2(kCapA1 * cap, kCapA1 * cap);
        a2 = dev::f32x2(kCapA2 * cap, kCapA2 * cap);
        a3 = dev::f32x2(kCapA3 * cap, kCapA3 * cap);
        two_u = dev::f32x2(w, w);
    }
};

// cap_log2 tanh - m of K pairs of scores by the series (nm: -m in both halves), in place,
// step by step; u^2 of them in `t`.
template <int K>
__device__ __forceinline__ void cap_series(unsigned long long (&x)[K], unsigned long long nm, const CapFactors &f,
                                           unsigned long long (&t)[K]) {
    unsigned long long q[K];
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = dev::mul_f32x2(x[k], f.to_cap);
#pragma unroll
    for (int k = 0; k < K; ++k) t[k] = dev::mul_f32x2(x[k], x[k]);
#pragma unroll
    for (int k = 0; k < K; ++k) q[k] = dev::fma_f32x2(t[k], f.a3, f.a2);
#pragma unroll
    for (int k = 0; k < K; ++k) q[k] = dev::fma_f32x2(q[k], t[k], f.a1);
#pragma unroll
    for (int k = 0; k < K; ++k) q[k] = dev::fma_f32x2(q[k], t[k], f.c0);
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = dev::fma_f32x2(x[k], q[k], nm);
}

// One pair.
__device__ __forceinline__ unsigned long long cap_series(unsigned long long x, unsigned long long nm,
                                                         const CapFactors &f, unsigned long long &t) {
    unsigned long long y[1] = {x}, t1[1];
    cap_series<1>(y, nm, f, t1);
    t = t1[0];
    return y[0];
}

// 1 + e^(2u) of two scores, whose factors are cut at 2^60 (tanh is 1 there in fp32,
// infinities included).  A NaN stays one, or with CUT is cut like infinity.
template <bool CUT>
__device__ __forceinline__ void cap_divisors(float x0, float x1, const CapFactors &f, float &d0, float &d1) {
    float w0, w1;
    dev::f32x2_split(dev::mul_f32x2(dev::f32x2(x0, x1), f.two_u), w0, w1);
    w0 = CUT ? fminf(w0, 60.f) : dev::min_nan(w0, 60.f);
    w1 = CUT ? fminf(w1, 60.f) : dev::min_nan(w1, 60.f);
    dev::f32x2_split(dev::add_f32x2(dev::f32x2(dev::fast_exp2(w0), dev::fast_exp2(w1)), dev::f32x2(1.f, 1.f)), d0, d1);
}

// cap_log2 tanh - m of two scores by the exponential (base: cap_log2 - m in both
// halves).  They share one reciprocal, 1 / (d0 d1), and so a NaN, which only scores of
// one row may that both count; with CUT the caller makes the row NaN.
template <bool CUT>
__device__ __forceinline__ unsigned long long cap_exp_pair(float x0, float x1, const CapFactors &f,
                                                           unsigned long long base) {
    float d0, d1;
    cap_divisors<CUT>(x0, x1, f, d0, d1);
    const float r = fast_rcp(d0 * d1);
    return dev::fma_f32x2(dev::f32x2(r * d1, r * d0), dev::f32x2(-2.f * f.cap, -2.f * f.cap), base);
}

// The same (with CUT) with every score in the form its own size asks for.
__device__ __forceinline__ void cap_pair(float x0, float x1, unsigned long long nm, const CapFactors &f,
                                         float &y0, float &y1) {
    unsigned long long t;
    float s0, s1, t0, t1, e0, e1;
    dev::f32x2_split(cap_series(dev::f32x2(x0, x1), nm, f, t), s0, s1);
    dev::f32x2_split(t, t0, t1);
    dev::f32x2_split(cap_exp_pair<true>(x0, x1, f, dev::add_f32x2(dev::f32x2(f.cap, f.cap), nm)), e0, e1);
    y0 = t0 < kCapSeries * kCapSeries ? s0 : e0;
    y1 = t1 < kCapSeries * kCapSeries ? s1 : e1;
}

// One score's logit.
__device__ __forceinline__ float cap_one(float x, const CapFactors &f) {
    float y, unused;
    cap_pair(x, x, dev::f32x2(0.f, 0.f), f, y, unused);
    return y;
}

// Four scores of an mma.sync accumulator, in place, by the exponential.  Scores 0 and
// 1, and 2 and 3, are of one row (APART 1), or 0 and 2, and 1 and 3 (APART 2).
template <int APART>
__device__ __forceinline__ void cap_exp_quad(float (&x)[4], const CapFactors &f) {
    const unsigned long long base = dev::f32x2(f.cap, f.cap), twice = dev::f32x2(-2.f * f.cap, -2.f * f.cap);
    float d[4];
    cap_divisors<false>(x[0], x[1], f, d[0], d[1]);
    cap_divisors<false>(x[2], x[3], f, d[2], d[3]);
    const float ra = fast_rcp(d[0] * d[APART]), rb = fast_rcp(d[3] * d[3 - APART]);
    const float n0 = ra * d[APART], n1 = APART == 1 ? ra * d[0] : rb * d[3];
    const float n2 = APART == 1 ? rb * d[3] : ra * d[0], n3 = rb * d[3 - APART];
    dev::f32x2_split(dev::fma_f32x2(dev::f32x2(n0, n1), twice, base), x[0], x[1]);
    dev::f32x2_split(dev::fma_f32x2(dev::f32x2(n2, n3), twice, base), x[2], x[3]);
}

// ---------------------------------------------------------------- mma.sync steps
// A lane's M accumulators of scores to logits in place; the whole warp calls.
// Scores that do not count are finite.  large: whether the warp's last scores of the same
// item had one at kCapSeries or past it.  The series runs on trust, and the scores are done again
// if one turns up.
template <int APART, int M>
__device__ __forceinline__ void cap_scores(float (&x)[M][4], bool &large, const CapFactors &f) {
    if (!large) {
        float most = 0.f, y[M][4];
#pragma unroll
        for (int i = 0; i < M; ++i)
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                unsigned long long t;
                float t0, t1;
                dev::f32x2_split(cap_series(dev::f32x2(x[i][j], x[i][j + 1]), 0ull, f, t), y[i][j], y[i][j + 1]);
                dev::f32x2_split(t, t0, t1);
                most = dev::max3(most, t0, t1);
            }
        large = __any_sync(0xffffffffu, most >= kCapSeries * kCapSeries);
        if (!large) {
#pragma unroll
            for (int i = 0; i < M; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[i][j] = y[i][j];
            return;
        }
    }
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < M; ++i) {
        most = dev::max3(dev::max3(most, fabsf(x[i][0]), fabsf(x[i][1])), fabsf(x[i][2]), fabsf(x[i][3]));
        float e[4] = {x[i][0], x[i][1], x[i][2], x[i][3]};
        cap_exp_quad<APART>(e, f);
        if (f.cap > kCapFreeLog2) {
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                unsigned long long t;
                float s0, s1, t0, t1;
                dev::f32x2_split(cap_series(dev::f32x2(x[i][j], x[i][j + 1]), 0ull, f, t), s0, s1);
                dev::f32x2_split(t, t0, t1);
                if (t0 < kCapSeries * kCapSeries) e[j] = s0;
                if (t1 < kCapSeries * kCapSeries) e[j + 1] = s1;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = e[j];
    }
    large = __any_sync(0xffffffffu, most * f.to >= kCapSeries);
}

// The same to P = 2^x (caps up to kCapFreeLog2).
template <int APART, int M>
__device__ __forceinline__ void cap_free_scores(float (&x)[M][4], bool &large, const CapFactors &f) {
    cap_scores<APART>(x, large, f);
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = dev::fast_exp2(x[i][j]);
}

// ---------------------------------------------------------------- tiles
// A tile's softmax keeps a row's scores as they come from TMEM and caps them
// inside the loop that takes their exponentials, where the series (FMA pipe)
// runs beside the exponentials (MUFU); tanh is monotone, so the row's largest
// logit is that of its largest score, and no pass over the logits is needed
// before.  Keys a row does not see (from `seen` on) are left out of the range
// and get P = 0, whatever their score.

__device__ __forceinline__ float score_of(float x) { return x; }
__device__ __forceinline__ float score_of(uint32_t x) { return __uint_as_float(x); }

// Where a tile's P goes: packed 16-bit pairs and the row's sum.
template <bool F16>
struct PackedRow {
    uint32_t *pw;
    unsigned long long sum;
    __device__ __forceinline__ void start() { sum = 0ull; }
    __device__ __forceinline__ void operator()(int c, float p0, float p1) {
        sum = dev::add_f32x2(sum, dev::f32x2(p0, p1));
        pw[c] = F16 ? dev::pack_f16(p0, p1) : dev::pack_bf16(p0, p1);
    }
};

// P = 2^x (caps up to kCapFreeLog2) of N scores, the first `seen` of which count
// (hidden: for some lane of the warp not all), handed pair by pair to `put` (again from
// `start()` on where a block is done twice); the whole warp calls.  large: whether the
// warp's last block of the same item had a score at kCapSeries or past it.  The series runs on trust,
// and the block is done again if one turns up; the exponential form then serves all of
// its scores: its absolute error, 2e-7 cap, is 1e-5 at most there.  K pairs go
// through the series side by side: 8 in the prefill, whose registers hold them (calls
// back to back, in turn on one GPU: the join 635 us with 1, 649 with 4, 625 with 8 and
// 16; the fork 50.3, 49.5, 49.4, 50.0), 1 in the decode tiles (128 branches of a 32k
// prefix 144 with 1, 149 with 8).
template <int K, int N, class X, class Put>
__device__ __forceinline__ void cap_free(const X (&x)[N], int seen, bool hidden, bool &large, const CapFactors &f,
                                         Put &put) {
    const unsigned long long base = dev::f32x2(f.cap, f.cap);
    put.start();
    if (hidden) {
#pragma unroll
        for (int c = 0; c < N / 2; ++c) {
            const float x0 = score_of(x[2 * c]), x1 = score_of(x[2 * c + 1]);
            float e0, e1;
            dev::f32x2_split(cap_exp_pair<true>(x0, x1, f, base), e0, e1);
            const float p0 = x0 == x0 ? dev::fast_exp2(e0) : x0, p1 = x1 == x1 ? dev::fast_exp2(e1) : x1;
            put(c, 2 * c < seen ? p0 : 0.f, 2 * c + 1 < seen ? p1 : 0.f);
        }
        return;
    }
    if (!large) {
        float most = 0.f;
#pragma unroll
        for (int c = 0; c < N / 2; c += K) {
            unsigned long long y[K], t[K];
#pragma unroll
            for (int k = 0; k < K; ++k) y[k] = dev::f32x2(score_of(x[2 * (c + k)]), score_of(x[2 * (c + k) + 1]));
            cap_series<K>(y, 0ull, f, t);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float e0, e1, t0, t1;
                dev::f32x2_split(y[k], e0, e1);
                dev::f32x2_split(t[k], t0, t1);
                most = dev::max3(most, t0, t1);
                put(c + k, dev::fast_exp2(e0), dev::fast_exp2(e1));
            }
        }
        large = __any_sync(0xffffffffu, most >= kCapSeries * kCapSeries);
        if (!large) return;
        put.start();
    }
    float most = 0.f;
#pragma unroll
    for (int c = 0; c < N / 2; ++c) {
        const float x0 = score_of(x[2 * c]), x1 = score_of(x[2 * c + 1]);
        float e0, e1;
        dev::f32x2_split(cap_exp_pair<false>(x0, x1, f, base), e0, e1);
        most = dev::max3(most, fabsf(x0), fabsf(x1));
        put(c, dev::fast_exp2(e0), dev::fast_exp2(e1));
    }
    large = __any_sync(0xffffffffu, most * f.to >= kCapSeries);
}

// Widen [lo, hi] by N scores of which the first `seen` count; hi is NaN from the
// first NaN on, and cap_reference then too.
template <int N, class X>
__device__ __forceinline__ void cap_range(const X (&x)[N], int seen, float &lo, float &hi) {
    if (seen >= N) {
#pragma unroll
        for (int j = 0; j < N; j += 2) {
            hi = dev::max3_nan(hi, score_of(x[j]), score_of(x[j + 1]));
            lo = dev::min3(lo, score_of(x[j]), score_of(x[j + 1]));
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float s = score_of(x[j]);
            hide_from(s, j, seen);                     // -inf from `seen` on
            hi = dev::max3_nan(hi, s, s);
            lo = j < seen ? fminf(lo, score_of(x[j])) : lo;
        }
    }
}

// What a row's P is taken against: 0 if it has seen no key, NaN if one is.
__device__ __forceinline__ float cap_reference(float m_use, float hi) {
    return hi != hi ? hi : m_use == -INFINITY ? 0.f : m_use;
}

// P of N scores, the first `seen` of which count (hidden: for some lane of the warp
// not all), against the reference (nm: its negative in both halves), handed to
// `put`.  large: some score of the warp's block reaches kCapSeries; caps up to
// kCapFreeLog2 then take the exponential form for all of it.
template <int N, class X, class Put>
__device__ __forceinline__ void cap_exponentials(const X (&x)[N], int seen, bool hidden, bool large,
                                                 unsigned long long nm, const CapFactors &f, Put &put) {
    put.start();
    if (!hidden && !large) {
#pragma unroll
        for (int c = 0; c < N / 2; ++c) {
            unsigned long long t;
            float e0, e1;
            dev::f32x2_split(cap_series(dev::f32x2(score_of(x[2 * c]), score_of(x[2 * c + 1])), nm, f, t), e0, e1);
            put(c, dev::fast_exp2(e0), dev::fast_exp2(e1));
        }
    } else if (!hidden && f.cap <= kCapFreeLog2) {
        const unsigned long long base = dev::add_f32x2(dev::f32x2(f.cap, f.cap), nm);
#pragma unroll
        for (int c = 0; c < N / 2; ++c) {
            float e0, e1;
            dev::f32x2_split(cap_exp_pair<true>(score_of(x[2 * c]), score_of(x[2 * c + 1]), f, base), e0, e1);
            put(c, dev::fast_exp2(e0), dev::fast_exp2(e1));
        }
    } else {
#pragma unroll
        for (int c = 0; c < N / 2; ++c) {
            float e0, e1;
            cap_pair(score_of(x[2 * c]), score_of(x[2 * c + 1]), nm, f, e0, e1);
            const float p0 = dev::fast_exp2(e0), p1 = dev::fast_exp2(e1);
            put(c, 2 * c < seen ? p0 : 0.f, 2 * c + 1 < seen ? p1 : 0.f);
        }
    }
}

}  // namespace
}  // namespace parason
