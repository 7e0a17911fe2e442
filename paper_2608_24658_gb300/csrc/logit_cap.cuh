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
// is at most 5e-7 of tanh(kCapSeries).  Which form a score takes depends on that
// score alone.
//
// What bounds it: the softmax warps' issue slots and the MUFU.  The series is 7
// packed instructions per two scores and no MUFU; the exponential form adds an
// exponential and a reciprocal per score to the softmax's own exponential.  Models
// keep nearly all logits far below their cap, so a warp votes: if no score of
// the block reaches kCapSeries, it runs the series alone.
#pragma once

#include "device_common.cuh"

namespace parason {
namespace {

constexpr float kCapSeries = 0.4f;
constexpr float kCapA1 = -0.33331882f, kCapA2 = 0.13277629f, kCapA3 = -0.047794217f;

__device__ __forceinline__ float fast_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The factors of one item's scores, in both halves of packed pairs.
struct CapFactors {
    unsigned long long to_cap, scale;    // u = to_cap <q, k>, scale = cap_log2 to_cap
    float two_u, cap_log2;               // two_u <q, k> = 2 u log2(e)
    __device__ __forceinline__ CapFactors(float to, float cap) {
        const float s = cap * to;
        to_cap = dev::f32x2(to, to);
        scale = dev::f32x2(s, s);
        two_u = 2.f * 1.4426950408889634f * to;
        cap_log2 = cap;
    }
};

// cap_log2 tanh of two scores by the series; u of both in `u`.
__device__ __forceinline__ unsigned long long cap_series(unsigned long long x, const CapFactors &f,
                                                         unsigned long long &u) {
    u = dev::mul_f32x2(x, f.to_cap);
    const unsigned long long t = dev::mul_f32x2(u, u);
    const unsigned long long s = dev::mul_f32x2(x, f.scale);
    unsigned long long q = dev::fma_f32x2(t, dev::f32x2(kCapA3, kCapA3), dev::f32x2(kCapA2, kCapA2));
    q = dev::fma_f32x2(q, t, dev::f32x2(kCapA1, kCapA1));
    return dev::fma_f32x2(dev::mul_f32x2(s, t), q, s);
}

// ... of one score by the exponential (x = +-inf gives +-cap_log2).
__device__ __forceinline__ float cap_exp(float x, const CapFactors &f) {
    return fmaf(-2.f * f.cap_log2, fast_rcp(1.f + dev::fast_exp2(x * f.two_u)), f.cap_log2);
}

// ... of one score, either way.
__device__ __forceinline__ float cap_one(float x, const CapFactors &f) {
    unsigned long long u;
    float s, unused, u0;
    dev::f32x2_split(cap_series(dev::f32x2(x, x), f, u), s, unused);
    dev::f32x2_split(u, u0, unused);
    return fabsf(u0) < kCapSeries ? s : cap_exp(x, f);
}

__device__ __forceinline__ float score_of(float x) { return x; }
__device__ __forceinline__ float score_of(uint32_t x) { return __uint_as_float(x); }
__device__ __forceinline__ void set_score(float &x, float v) { x = v; }
__device__ __forceinline__ void set_score(uint32_t &x, float v) { x = __float_as_uint(v); }

// M x N scores of a lane (floats or their bits) in place; the whole warp calls.
template <int M, int N, class X>
__device__ __forceinline__ void cap_scores(X (&x)[M][N], float to_cap, float cap_log2) {
    static_assert(N % 2 == 0, "scores come in pairs");
    const CapFactors f(to_cap, cap_log2);
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int j = 0; j < N; j += 2)
            most = dev::max3(most, fabsf(score_of(x[i][j])), fabsf(score_of(x[i][j + 1])));
    if (!__any_sync(0xffffffffu, most * fabsf(to_cap) >= kCapSeries)) {
#pragma unroll
        for (int i = 0; i < M; ++i)
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                unsigned long long u;
                float a, b;
                dev::f32x2_split(cap_series(dev::f32x2(score_of(x[i][j]), score_of(x[i][j + 1])), f, u), a, b);
                set_score(x[i][j], a);
                set_score(x[i][j + 1], b);
            }
        return;
    }
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int j = 0; j < N; j += 2) {
            const float p = score_of(x[i][j]), q = score_of(x[i][j + 1]);
            unsigned long long u;
            float a, b, u0, u1;
            dev::f32x2_split(cap_series(dev::f32x2(p, q), f, u), a, b);
            dev::f32x2_split(u, u0, u1);
            set_score(x[i][j], fabsf(u0) < kCapSeries ? a : cap_exp(p, f));
            set_score(x[i][j + 1], fabsf(u1) < kCapSeries ? b : cap_exp(q, f));
        }
}

template <int N, class X>
__device__ __forceinline__ void cap_scores(X (&x)[N], float to_cap, float cap_log2) {
    cap_scores<1, N, X>(*reinterpret_cast<X(*)[1][N]>(&x), to_cap, cap_log2);
}

}  // namespace
}  // namespace parason
