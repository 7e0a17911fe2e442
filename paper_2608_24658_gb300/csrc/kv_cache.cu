// kv_cache.cu -- filling and reading the paged KV cache: rows of tokens rotated
// to their positions, rounded to the cache's type and written into their slots
// (parason_kv_write), taken out again (parason_kv_read), and the e4m3 scales
// that hold them (parason_kv_scales).
//
// All three move bytes: HBM bounds them on long inputs, launches and one chain
// of dependent loads (slot or position, then rows) on short ones.
#include <cuda_fp8.h>

#include <cmath>

#include "device_common.cuh"
#include "internal.h"

namespace parason {
namespace {

constexpr int kMaxFreqs = 64;            // rotary_dim / 2 at head_dim 128
constexpr int kMaxAxes = 4;
constexpr float kE4m3Max = 448.f;

struct Rows {
    const void *data;
    int64_t token_stride, head_stride;
};

// A rotary description by value: the axis of each frequency travels in the
// kernel's parameters.
struct RotaryArgs {
    const float *inv_freq;
    const int32_t *positions;
    int64_t position_stride;
    int32_t half;                        // pairs of a head; 0: nothing turns
    int32_t interleaved;
    uint8_t axis[kMaxFreqs];
};

struct WriteArgs {
    Rows q, k, v;
    RotaryArgs rot;
    const int32_t *slots;
    const float *k_scale, *v_scale;
    void *q_out, *k_pages, *v_pages;
    int64_t num_tokens;
    int64_t num_slots;                   // of the pool
    int32_t num_q_heads, num_kv_heads;   // num_q_heads 0: no queries
};

struct ReadArgs {
    const int32_t *slots;
    const void *k_pages, *v_pages;
    const float *k_scale, *v_scale;
    Rows k, v;
    int64_t num_tokens, num_slots;
    int32_t num_kv_heads;
};

struct ScalesArgs {
    Rows k, v;
    const int32_t *slots;
    float *k_scale, *v_scale;
    int64_t num_tokens;
    int32_t num_kv_heads, half, interleaved;
};

// Eight consecutive elements, the unit every kernel here moves: 16 bytes of
// bf16, 32 of fp32, 8 of e4m3.
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float (&x)[8]) {
    const uint4 u = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float4 u = reinterpret_cast<const float4 *>(p)[i];
        x[4 * i] = u.x;
        x[4 * i + 1] = u.y;
        x[4 * i + 2] = u.z;
        x[4 * i + 3] = u.w;
    }
}

__device__ __forceinline__ void load8(const __nv_fp8_e4m3 *p, float (&x)[8]) {
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    const uint32_t w[2] = {u.x, u.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(w[i >> 1] >> (16 * (i & 1)))));
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}

__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&x)[8]) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(dev::pack_bf16(x[0], x[1]), dev::pack_bf16(x[2], x[3]),
                                               dev::pack_bf16(x[4], x[5]), dev::pack_bf16(x[6], x[7]));
}

__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// Round to nearest even, saturating at +-448 (infinities too); NaN stays NaN.
__device__ __forceinline__ void store8(__nv_fp8_e4m3 *p, const float (&x)[8]) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i], x[4 * i + 1]), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i + 2], x[4 * i + 3]), __NV_SATFINITE, __NV_E4M3);
        w[i] = lo | (hi << 16);
    }
    *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
}

template <class KV>
constexpr bool kScaled = sizeof(KV) == 1;

// cos and sin of positions[axis] * inv_freq[i].  A turn's fraction is what
// counts, so the angle is taken in turns: the product (exact: 31 and 24 bits)
// times 1 / 2 pi in 64 bits is off by less than 2^-52 of its size, a
// millionth of a turn at position 2^31 and below fp32's own rounding of the
// fraction up to position 2^24.
__device__ __forceinline__ float2 turn(const RotaryArgs &r, int64_t t, int i) {
    constexpr double kTurnsPerRadian = 0.15915494309189533577;
    const double f = static_cast<double>(r.inv_freq[i]) * kTurnsPerRadian;
    const double turns = static_cast<double>(r.positions[r.axis[i] * r.position_stride + t]) * f;
    float s, c;
    sincospif(2.f * static_cast<float>(turns - rint(turns)), &s, &c);
    return make_float2(c, s);
}

constexpr int kThreads = 128;

// One CTA per token: the token's angles into shared memory, then its heads in
// units of two 8-element chunks that hold whole pairs.
template <class T, class KV, int D>
__global__ void __launch_bounds__(kThreads) kv_write_kernel(const WriteArgs a) {
    __shared__ float2 cs[kMaxFreqs];
    constexpr int kUnits = D / 16;
    const int64_t t = blockIdx.x;
    dev::grid_wait();
    if (static_cast<int>(threadIdx.x) < a.rot.half) cs[threadIdx.x] = turn(a.rot, t, threadIdx.x);
    const int64_t slot = a.slots[t];
    const bool live = slot >= 0 && slot < a.num_slots;
    __syncthreads();
    const int heads = a.num_q_heads + 2 * a.num_kv_heads;
    for (int w = threadIdx.x; w < heads * kUnits; w += kThreads) {
        const int u = w % kUnits;
        int h = w / kUnits;
        const Rows *src;
        void *pool = nullptr;
        const float *scale = nullptr;
        bool turned = true;
        if (h < a.num_q_heads) {
            src = &a.q;
        } else if ((h -= a.num_q_heads) < a.num_kv_heads) {
            src = &a.k;
            pool = a.k_pages;
            scale = a.k_scale;
        } else {
            h -= a.num_kv_heads;
            src = &a.v;
            pool = a.v_pages;
            scale = a.v_scale;
            turned = false;
        }
        if (pool && !live) continue;
        // chunks c0 and c1: where pairs are halves of the rotated part, chunk u
        // and its partner; else neighbours
        const bool rotates = turned && 8 * u < a.rot.half;
        int e0 = 16 * u, e1 = e0 + 8, f0 = 8 * u;
        if (turned && !a.rot.interleaved && rotates) {
            e0 = 8 * u;
            e1 = e0 + a.rot.half;
        }
        const T *x = static_cast<const T *>(src->data) + t * src->token_stride + h * src->head_stride;
        float x0[8], x1[8];
        load8(x + e0, x0);
        load8(x + e1, x1);
        if (rotates) {
            if (a.rot.interleaved) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float(&y)[8] = i < 4 ? x0 : x1;
                    const float2 c = cs[f0 + i];
                    const float p = y[2 * (i & 3)], q = y[2 * (i & 3) + 1];
                    y[2 * (i & 3)] = p * c.x - q * c.y;
                    y[2 * (i & 3) + 1] = p * c.y + q * c.x;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 c = cs[f0 + i];
                    const float p = x0[i], q = x1[i];
                    x0[i] = p * c.x - q * c.y;
                    x1[i] = p * c.y + q * c.x;
                }
            }
        }
        if (!pool) {
            T *dst = static_cast<T *>(a.q_out) + (t * a.num_q_heads + h) * D;
            store8(dst + e0, x0);
            store8(dst + e1, x1);
        } else {
            if constexpr (kScaled<KV>) {
                const float s = scale[h];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x0[i] /= s;
                    x1[i] /= s;
                }
            }
            KV *dst = static_cast<KV *>(pool) +
                      ((slot / kPageSize * a.num_kv_heads + h) * kPageSize + slot % kPageSize) * D;
            store8(dst + e0, x0);
            store8(dst + e1, x1);
        }
    }
}

// One CTA per token.
template <class T, class KV, int D>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(const ReadArgs a) {
    constexpr int kUnits = D / 8;
    const int64_t t = blockIdx.x;
    dev::grid_wait();
    const int64_t slot = a.slots[t];
    const bool live = slot >= 0 && slot < a.num_slots;
    for (int w = threadIdx.x; w < 2 * a.num_kv_heads * kUnits; w += kThreads) {
        const int u = w % kUnits;
        int h = w / kUnits;
        const bool is_k = h < a.num_kv_heads;
        if (!is_k) h -= a.num_kv_heads;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (live) {
            load8(static_cast<const KV *>(is_k ? a.k_pages : a.v_pages) +
                      ((slot / kPageSize * a.num_kv_heads + h) * kPageSize + slot % kPageSize) * D + 8 * u,
                  x);
            if constexpr (kScaled<KV>) {
                const float s = (is_k ? a.k_scale : a.v_scale)[h];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] *= s;
            }
        }
        const Rows &dst = is_k ? a.k : a.v;
        store8(static_cast<T *>(const_cast<void *>(dst.data)) + t * dst.token_stride + h * dst.head_stride + 8 * u, x);
    }
}

// Scales at their least, 2^-126, before the tokens raise them.
__global__ void reset_scales_kernel(float *k_scale, float *v_scale, int n) {
    dev::grid_wait();
    for (int i = threadIdx.x; i < n; i += blockDim.x) k_scale[i] = v_scale[i] = 1.17549435e-38f;
}

// min(|x|, 2^63), 0 for NaN: squares of these add up within fp32.
__device__ __forceinline__ float magnitude(float x) {
    return fmaxf(fminf(fabsf(x), 9.2233720369e18f), 0.f) * (x == x ? 1.f : 0.f);
}

// One CTA per (256 tokens, head, K or V).  Positive floats order as their
// bits do, so the maxima meet in integer atomics, whose order does not matter;
// max / 448 is the max of the quotients, since rounding is monotone.
template <int D>
__global__ void __launch_bounds__(kThreads) kv_scales_kernel(const ScalesArgs a) {
    constexpr int kUnits = D / 16, kTokens = 256;
    __shared__ float part[kThreads / 32];
    const int h = blockIdx.y;
    const bool is_k = blockIdx.z == 0;
    const Rows &src = is_k ? a.k : a.v;
    const int half = is_k ? a.half : 0;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTokens;
    dev::grid_wait();
    float one = 0.f, pair = 0.f;         // max |x|, max of x0^2 + x1^2
    for (int w = threadIdx.x; w < kTokens * kUnits; w += kThreads) {
        const int64_t t = t0 + w / kUnits;
        const int u = w % kUnits;
        if (t >= a.num_tokens || (a.slots && a.slots[t] < 0)) continue;
        const bool rotates = 8 * u < half;
        int e0 = 16 * u, e1 = e0 + 8;
        if (rotates && !a.interleaved) {
            e0 = 8 * u;
            e1 = e0 + half;
        }
        const __nv_bfloat16 *x = static_cast<const __nv_bfloat16 *>(src.data) + t * src.token_stride +
                                 h * src.head_stride;
        float x0[8], x1[8];
        load8(x + e0, x0);
        load8(x + e1, x1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x0[i] = magnitude(x0[i]);
            x1[i] = magnitude(x1[i]);
            one = fmaxf(one, fmaxf(x0[i], x1[i]));
        }
        if (rotates) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = a.interleaved ? (i < 4 ? x0 : x1)[2 * (i & 3)] : x0[i];
                const float q = a.interleaved ? (i < 4 ? x0 : x1)[2 * (i & 3) + 1] : x1[i];
                pair = fmaxf(pair, p * p + q * q);
            }
        }
    }
    float m = fmaxf(one, sqrtf(pair));
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kThreads / 32; ++i) m = fmaxf(m, part[i]);
        atomicMax(reinterpret_cast<int *>((is_k ? a.k_scale : a.v_scale) + h), __float_as_int(m / kE4m3Max));
    }
}

template <class T, class KV, int D>
cudaError_t launch_write(const WriteArgs &a, cudaStream_t s) {
    return launch_dependent(true, kv_write_kernel<T, KV, D>, dim3(static_cast<unsigned>(a.num_tokens)),
                            dim3(kThreads), 0, s, a);
}

template <class T, class KV, int D>
cudaError_t launch_read(const ReadArgs &a, cudaStream_t s) {
    return launch_dependent(true, kv_read_kernel<T, KV, D>, dim3(static_cast<unsigned>(a.num_tokens)),
                            dim3(kThreads), 0, s, a);
}

// ---------------------------------------------------------------- arguments

bool misaligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

parason_status check_rows(const parason_rows *r, int64_t tokens, int32_t heads, int32_t d, int elem, bool out) {
    if (!r || !r->data || misaligned(r->data, 16)) return PARASON_EINVAL;
    const int64_t strides[2] = {tokens > 1 ? r->token_stride : d, heads > 1 ? r->head_stride : d};
    for (int64_t st : strides) {
        if (st < 0 || st * elem % 16 != 0) return PARASON_EINVAL;
        if (out && st < d) return PARASON_EINVAL;
    }
    return PARASON_OK;
}

Rows to_rows(const parason_rows *r) { return Rows{r->data, r->token_stride, r->head_stride}; }

// the checks every call shares
parason_status check_call(const parason_attn_config *cfg, int64_t tokens, int64_t pages) {
    const parason_status st = check_config(cfg);
    if (st != PARASON_OK) return st;
    if (tokens < 0 || tokens > INT32_MAX || pages < 0) return PARASON_EINVAL;
    if (pages > INT32_MAX / kPageSize / cfg->num_kv_heads) return PARASON_EUNSUPPORTED;
    return PARASON_OK;
}

// the part of a rotary description that kv_scales uses too
parason_status check_pairs(const parason_rotary *r, int32_t d) {
    if (r->rotary_dim <= 0 || r->rotary_dim > d || r->rotary_dim % 16 != 0) return PARASON_EINVAL;
    if (r->pairs != PARASON_ROTARY_HALVES && r->pairs != PARASON_ROTARY_INTERLEAVED) return PARASON_EINVAL;
    return PARASON_OK;
}

parason_status to_rotary(const parason_rotary *r, int32_t d, RotaryArgs *out) {
    *out = RotaryArgs{};
    if (!r) return PARASON_OK;
    const parason_status st = check_pairs(r, d);
    if (st != PARASON_OK) return st;
    if (r->num_axes < 1 || r->num_axes > kMaxAxes || !r->inv_freq || !r->positions ||
        misaligned(r->inv_freq, 4) || misaligned(r->positions, 4) || (r->num_axes > 1 && r->position_stride < 0))
        return PARASON_EINVAL;
    out->inv_freq = r->inv_freq;
    out->positions = r->positions;
    out->position_stride = r->num_axes > 1 ? r->position_stride : 0;
    out->half = r->rotary_dim / 2;
    out->interleaved = r->pairs == PARASON_ROTARY_INTERLEAVED;
    for (int i = 0; r->freq_axis && i < out->half; ++i) {
        if (r->freq_axis[i] >= r->num_axes) return PARASON_EINVAL;
        out->axis[i] = r->freq_axis[i];
    }
    return PARASON_OK;
}

parason_status launched(cudaError_t e) { return e == cudaSuccess ? PARASON_OK : PARASON_ECUDA; }

}  // namespace
}  // namespace parason

using namespace parason;

extern "C" parason_status parason_kv_write(const parason_attn_config *cfg, int64_t num_tokens,
                                           const parason_rows *q, const parason_rows *k,
                                           const parason_rows *v, const parason_rotary *rotary,
                                           const int32_t *slots, const float *k_scale,
                                           const float *v_scale, void *q_out, void *k_pages,
                                           void *v_pages, int64_t num_physical_pages,
                                           parason_stream_t stream) {
    parason_status st = check_call(cfg, num_tokens, num_physical_pages);
    if (st != PARASON_OK) return st;
    const int32_t d = cfg->head_dim;
    const int elem = cfg->mode == PARASON_FP32 ? 4 : 2;
    WriteArgs a{};
    if ((st = to_rotary(rotary, d, &a.rot)) != PARASON_OK) return st;
    if (num_tokens == 0) return PARASON_OK;
    if ((st = check_rows(k, num_tokens, cfg->num_kv_heads, d, elem, false)) != PARASON_OK) return st;
    if ((st = check_rows(v, num_tokens, cfg->num_kv_heads, d, elem, false)) != PARASON_OK) return st;
    if (q && (st = check_rows(q, num_tokens, cfg->num_q_heads, d, elem, false)) != PARASON_OK) return st;
    if (q && (!q_out || misaligned(q_out, 16))) return PARASON_EINVAL;
    if (!slots || misaligned(slots, 4)) return PARASON_EINVAL;
    if (num_physical_pages > 0 && (!k_pages || !v_pages || misaligned(k_pages, 16) || misaligned(v_pages, 16)))
        return PARASON_EINVAL;
    if (cfg->mode == PARASON_FP8_E4M3_KV &&
        (!k_scale || !v_scale || misaligned(k_scale, 4) || misaligned(v_scale, 4)))
        return PARASON_EINVAL;
    if (q) a.q = to_rows(q);
    a.k = to_rows(k);
    a.v = to_rows(v);
    a.slots = slots;
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.q_out = q_out;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.num_tokens = num_tokens;
    a.num_slots = num_physical_pages * kPageSize;
    a.num_q_heads = q ? cfg->num_q_heads : 0;
    a.num_kv_heads = cfg->num_kv_heads;
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (cfg->mode == PARASON_FP8_E4M3_KV) return launched(launch_write<__nv_bfloat16, __nv_fp8_e4m3, 128>(a, s));
    if (cfg->mode == PARASON_FP32)
        return launched(d == 128 ? launch_write<float, float, 128>(a, s) : launch_write<float, float, 64>(a, s));
    return launched(d == 128 ? launch_write<__nv_bfloat16, __nv_bfloat16, 128>(a, s)
                             : launch_write<__nv_bfloat16, __nv_bfloat16, 64>(a, s));
}

extern "C" parason_status parason_kv_read(const parason_attn_config *cfg, int64_t num_tokens,
                                          const int32_t *slots, const void *k_pages,
                                          const void *v_pages, int64_t num_physical_pages,
                                          const float *k_scale, const float *v_scale,
                                          const parason_rows *k_out, const parason_rows *v_out,
                                          parason_stream_t stream) {
    parason_status st = check_call(cfg, num_tokens, num_physical_pages);
    if (st != PARASON_OK) return st;
    if (num_tokens == 0) return PARASON_OK;
    const int32_t d = cfg->head_dim;
    const int elem = cfg->mode == PARASON_FP32 ? 4 : 2;
    if ((st = check_rows(k_out, num_tokens, cfg->num_kv_heads, d, elem, true)) != PARASON_OK) return st;
    if ((st = check_rows(v_out, num_tokens, cfg->num_kv_heads, d, elem, true)) != PARASON_OK) return st;
    if (!slots || misaligned(slots, 4)) return PARASON_EINVAL;
    if (num_physical_pages > 0 && (!k_pages || !v_pages || misaligned(k_pages, 16) || misaligned(v_pages, 16)))
        return PARASON_EINVAL;
    if (cfg->mode == PARASON_FP8_E4M3_KV &&
        (!k_scale || !v_scale || misaligned(k_scale, 4) || misaligned(v_scale, 4)))
        return PARASON_EINVAL;
    ReadArgs a{};
    a.slots = slots;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.k = to_rows(k_out);
    a.v = to_rows(v_out);
    a.num_tokens = num_tokens;
    a.num_slots = num_physical_pages * kPageSize;
    a.num_kv_heads = cfg->num_kv_heads;
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (cfg->mode == PARASON_FP8_E4M3_KV) return launched(launch_read<__nv_bfloat16, __nv_fp8_e4m3, 128>(a, s));
    if (cfg->mode == PARASON_FP32)
        return launched(d == 128 ? launch_read<float, float, 128>(a, s) : launch_read<float, float, 64>(a, s));
    return launched(d == 128 ? launch_read<__nv_bfloat16, __nv_bfloat16, 128>(a, s)
                             : launch_read<__nv_bfloat16, __nv_bfloat16, 64>(a, s));
}

extern "C" parason_status parason_kv_scales(const parason_attn_config *cfg, int64_t num_tokens,
                                            const parason_rows *k, const parason_rows *v,
                                            const parason_rotary *rotary, const int32_t *slots,
                                            int32_t accumulate, float *k_scale, float *v_scale,
                                            parason_stream_t stream) {
    parason_status st = check_call(cfg, num_tokens, 0);
    if (st != PARASON_OK) return st;
    if (cfg->mode != PARASON_FP8_E4M3_KV) return PARASON_EINVAL;
    if (rotary && (st = check_pairs(rotary, cfg->head_dim)) != PARASON_OK) return st;
    if (accumulate != 0 && accumulate != 1) return PARASON_EINVAL;
    if (!k_scale || !v_scale || misaligned(k_scale, 4) || misaligned(v_scale, 4) || misaligned(slots, 4))
        return PARASON_EINVAL;
    ScalesArgs a{};
    if (num_tokens > 0) {
        if ((st = check_rows(k, num_tokens, cfg->num_kv_heads, cfg->head_dim, 2, false)) != PARASON_OK) return st;
        if ((st = check_rows(v, num_tokens, cfg->num_kv_heads, cfg->head_dim, 2, false)) != PARASON_OK) return st;
        a.k = to_rows(k);
        a.v = to_rows(v);
    }
    a.slots = slots;
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.num_tokens = num_tokens;
    a.num_kv_heads = cfg->num_kv_heads;
    a.half = rotary ? rotary->rotary_dim / 2 : 0;
    a.interleaved = rotary && rotary->pairs == PARASON_ROTARY_INTERLEAVED;
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (!accumulate) {
        const cudaError_t e = launch_dependent(true, reset_scales_kernel, dim3(1), dim3(kThreads), 0, s, k_scale,
                                               v_scale, static_cast<int>(cfg->num_kv_heads));
        if (e != cudaSuccess) return PARASON_ECUDA;
    }
    if (num_tokens == 0) return PARASON_OK;
    return launched(launch_dependent(true, kv_scales_kernel<128>,
                                     dim3(static_cast<unsigned>((num_tokens + 255) / 256),
                                          static_cast<unsigned>(cfg->num_kv_heads), 2),
                                     dim3(kThreads), 0, s, a));
}
