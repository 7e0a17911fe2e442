// kv_cache.cu -- filling and reading the paged KV cache: rows of tokens rotated
// to their positions, rounded to the cache's type and written into their slots
// (parason_kv_write), taken out again (parason_kv_read), and the e4m3 scales
// that hold them (parason_kv_scales).
//
// All three move bytes: HBM bounds them on long inputs, launches and one chain
// of dependent loads (slot or position, then rows) on short ones.
#include <cuda_fp8.h>

#include <atomic>
#include <cmath>

#include "device_common.cuh"
#include "internal.h"

namespace parason {
namespace {

constexpr int kMaxAxes = 4;
constexpr float kE4m3Max = 448.f;
constexpr int kMaxHeads = 16384;         // of q, and of k: what the kernels' counters hold
constexpr int kMaxDevices = 64;
constexpr int64_t kMaxRows = 1ll << 34;  // tokens times kv heads: what a grid holds (16 and more a CTA)

struct Rows {
    const void *data;
    int64_t token_stride, head_stride;
};

// A rotary description by value: the axis of each frequency travels in the
// kernel's parameters, as 2 bits (an array there would be read lane by lane); 64
// frequencies at most, at head_dim 128.
struct RotaryArgs {
    const uint64_t *turns;
    const int32_t *positions;
    int64_t position_stride;
    int32_t half;                        // pairs of a head; 0: nothing turns
    int32_t interleaved;
    uint64_t axes[2];                    // of frequencies 0..31 and 32..63
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
    int32_t parts;                       // warps that share a token
};

struct ReadArgs {
    const int32_t *slots;
    const void *k_pages, *v_pages;
    const float *k_scale, *v_scale;
    Rows k, v;
    int64_t num_tokens, num_slots;
    int32_t num_kv_heads;
    uint32_t heads_magic;                // n / heads is the high word of n times it (below 2^32 / heads;
                                         // 0: one head)
    bool short_rows;                     // rows fit 32 bits
    bool aligned;                        // k's and v's rows to 32 bytes
};

struct ScalesArgs {
    Rows k, v;
    const int32_t *slots;
    float *k_scale, *v_scale;
    int64_t num_tokens;
    int32_t num_kv_heads, half, interleaved;
};

// Eight consecutive elements, the unit every kernel here moves: 16 bytes of
// bf16, 32 of fp32, 8 of e4m3; loaded as they are, unpacked when they are used.
template <class T>
struct Raw8 {
    uint32_t w[2 * sizeof(T)];
};

template <class T>
__device__ __forceinline__ Raw8<T> load8(const T *p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) {
        const uint4 u = __ldcs(reinterpret_cast<const uint4 *>(p) + i);
        r.w[4 * i] = u.x;
        r.w[4 * i + 1] = u.y;
        r.w[4 * i + 2] = u.z;
        r.w[4 * i + 3] = u.w;
    }
    return r;
}

__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16> &r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(r.w[i] << 16);
        x[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ void unpack8(const Raw8<float> &r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r.w[i]);
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

constexpr int kThreads = 128;            // 4 warps, each of them on its own
constexpr int kWarps = kThreads / 32;

// CTAs of kv_write to ask an SM's registers for: bf16 and e4m3 rows fit 5 without
// spills (e4m3 took 105 registers unasked, and 300 tokens of 64 / 8 heads 4.5 us for
// 3.5); fp32 rows do not everywhere, and are left to themselves (96 to 104).
template <class T>
constexpr int kAskedCtas = sizeof(T) == 2 ? 5 : 0;

// cos and sin of positions[axis] * inv_freq[i].  The frequency is held as turns a
// position modulo 1, in 2^-64: the low 64 bits of its product with the position are
// the angle's part of a turn (off by 2^-33 at most, at position 2^31), whose upper 32
// as a signed number are it within half a turn: integers, as 64-bit floating point
// has a pipe of 2 lanes a cycle here.
__device__ __forceinline__ float2 turn(const RotaryArgs &r, int64_t t, int i) {
    const int axis = static_cast<int>((i < 32 ? r.axes[0] : r.axes[1]) >> (2 * (i & 31))) & 3;
    const int64_t pos = r.positions[axis * r.position_stride + t];
    const uint64_t part = static_cast<uint64_t>(pos) * r.turns[i];
    float s, c;
    sincospif(static_cast<float>(static_cast<int32_t>(part >> 32)) * 0x1p-31f, &s, &c);
    return make_float2(c, s);
}

// This lane's two chunks of kBatch steps (of G heads of one kind, q, k or v, of a token)
// from step s on, loaded together: src + e0 and src + e1, a step further `src_step`.
template <class T, int kBatch>
struct Batch {
    Raw8<T> r0[kBatch], r1[kBatch];
    template <int G>
    __device__ __forceinline__ void load(const T *src, int64_t src_step, int s, int s1, int heads, int mine, int e0,
                                         int e1) {
        src += s * src_step;
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (s + b >= s1 || (s + b) * G + mine >= heads) break;
            r0[b] = load8(src + b * src_step + e0);
            r1[b] = load8(src + b * src_step + e1);
        }
    }
};

// x / s in place, rounded to nearest: the product q with the rounded reciprocal y and its
// remainder q s - x, which an FMA gives exactly, make q - (q s - x) y the rounded quotient
// (P. Markstein, Computation of elementary functions on the IBM RISC System/6000,
// 1990); for s outside [2^-92, 2^126], where the remainder or y may be subnormal,
// within a last place.  In this order a zero keeps its sign.
//
// e4m3 needs it to the bit: a scale of amax / 448 puts many quotients on its ties, and
// with the product alone up to one value in fifty of a head came out a step off.  The
// product is cut at +-512, so that infinities leave no NaN (the remainder takes the
// quotient on).  20000 tokens of 64 / 8 heads 121.3 us with the product alone, 122.2 so,
// 129.3 with the compiler's division; of 8 heads without queries, where all is
// quotients, 25.8, 27.6 and 38.8.
__device__ __forceinline__ void quotients8(float (&x)[8], float s) {
    const float y = 1.f / s;
    const unsigned long long y2 = dev::f32x2(y, y), ny2 = dev::f32x2(-y, -y), s2 = dev::f32x2(s, s);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float q0, q1;
        dev::f32x2_split(dev::mul_f32x2(dev::f32x2(x[i], x[i + 1]), y2), q0, q1);
        const unsigned long long q = dev::f32x2(fminf(fmaxf(q0, -512.f), 512.f), fminf(fmaxf(q1, -512.f), 512.f));
        const unsigned long long r = dev::fma_f32x2(q, s2, dev::f32x2(-x[i], -x[i + 1]));
        dev::f32x2_split(dev::fma_f32x2(r, ny2, q), x[i], x[i + 1]);
    }
}

// Heads of one kind, steps [s0, s1): rotated, scaled, rounded, stored at dst + e0 and
// dst + e1, a step further `dst_step`.  `batch` holds the first steps already.
template <class T, class Out, int G, bool ROTATE, int kBatch>
__device__ __forceinline__ void write_heads(Batch<T, kBatch> &batch, const T *src, int64_t src_step, Out *dst,
                                            int64_t dst_step, int s0, int s1, int heads, int mine, int e0, int e1,
                                            bool interleaved, bool rotates, const unsigned long long (&cs)[4],
                                            const unsigned long long (&sn)[4], const float *scale) {
    dst += s0 * dst_step;
    for (int s = s0; s < s1; s += kBatch, dst += kBatch * dst_step) {
        if (s != s0) batch.template load<G>(src, src_step, s, s1, heads, mine, e0, e1);
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int h = (s + b) * G + mine;
            if (s + b >= s1 || h >= heads) break;
            float x0[8], x1[8];
            unpack8(batch.r0[b], x0);
            unpack8(batch.r1[b], x1);
            if (ROTATE && rotates) {
                // (p c - q s, p s + q c), two pairs an instruction
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float &p0 = interleaved ? (i < 2 ? x0 : x1)[4 * (i & 1)] : x0[2 * i];
                    float &p1 = interleaved ? (i < 2 ? x0 : x1)[4 * (i & 1) + 2] : x0[2 * i + 1];
                    float &q0 = interleaved ? (i < 2 ? x0 : x1)[4 * (i & 1) + 1] : x1[2 * i];
                    float &q1 = interleaved ? (i < 2 ? x0 : x1)[4 * (i & 1) + 3] : x1[2 * i + 1];
                    const unsigned long long p = dev::f32x2(p0, p1), q = dev::f32x2(q0, q1);
                    const unsigned long long nq = dev::f32x2(-q0, -q1);
                    dev::f32x2_split(dev::fma_f32x2(p, cs[i], dev::mul_f32x2(nq, sn[i])), p0, p1);
                    dev::f32x2_split(dev::fma_f32x2(p, sn[i], dev::mul_f32x2(q, cs[i])), q0, q1);
                }
            }
            if constexpr (sizeof(Out) == 1) {
                const float div = scale[h];
                quotients8(x0, div);
                quotients8(x1, div);
            }
            store8(dst + b * dst_step + e0, x0);
            store8(dst + b * dst_step + e1, x1);
        }
    }
}

// A warp is 512 / D groups of D / 16 lanes, a group a head: each lane has two 8-element
// chunks of it that hold whole pairs, chunk u of the first half of the rotated part and
// its partner, or two neighbours.  So no element crosses a lane, rotation is in place
// for q, and a warp's loads and stores are whole sectors.  G groups share a token and
// take its heads G at a step, first q's, then k's, then v's: a warp takes as many tokens
// as it has such teams, or one of `parts` equal parts of one token's steps.
//
// Three steps of a head are loaded ahead in bf16: with 1, 2, 3, 4 the prompt of 8192
// tokens takes 40.6, 34.5, 33.5, 33.1 us and the e4m3 batch of 2500 22.2, 19.0, 18.7,
// 19.5.
//
// The angles are made once for all heads of a token: the G lanes of one u share 8
// pairs' angles, make 8 / G each and pass them round (out of shared memory they were
// read four lanes to a bank).
template <class T, class KV, int D, bool INTERLEAVED, int G>
__global__ void __launch_bounds__(kThreads, kAskedCtas<T>) kv_write_kernel(const WriteArgs a) {
    constexpr int kLanes = D / 16, kTeams = 32 / kLanes / G, kMake = 8 / G;
    constexpr int kBatch = sizeof(T) == 4 ? 2 : 3;            // (steps in flight, as above)
    const int lane = threadIdx.x % 32;
    const int64_t job = static_cast<int64_t>(blockIdx.x) * kWarps + threadIdx.x / 32;
    const int64_t t0 = a.parts == 1 ? job : job / a.parts;
    if (t0 * kTeams >= a.num_tokens) return;
    const int part = static_cast<int>(job - t0 * a.parts);
    const int q_steps = (a.num_q_heads + G - 1) / G, kv_steps = (a.num_kv_heads + G - 1) / G;
    const int steps = q_steps + 2 * kv_steps;                 // (3 * 2^14 at most)
    const int first = a.parts == 1 ? 0 : static_cast<int>(static_cast<int64_t>(steps) * part / a.parts);
    const int last = a.parts == 1 ? steps : static_cast<int>(static_cast<int64_t>(steps) * (part + 1) / a.parts);
    const int u = lane % kLanes, team = lane / kLanes / G, mine = lane / kLanes % G;
    const int64_t t = t0 * kTeams + team;
    const bool there = t < a.num_tokens;
    const bool rotates = 8 * u < a.rot.half, halves = rotates && !INTERLEAVED;
    // the elements of this lane's chunks in q and k; in v: 16 u and 16 u + 8
    const int e0 = halves ? 8 * u : 16 * u, e1 = e0 + (halves ? a.rot.half : 8);
    dev::grid_wait();
    const int64_t slot = there ? a.slots[t] : -1;

    // the first loads go out before the angles are made
    const T *q = static_cast<const T *>(a.q.data) + t * a.q.token_stride + mine * a.q.head_stride;
    const T *k = static_cast<const T *>(a.k.data) + t * a.k.token_stride + mine * a.k.head_stride;
    const T *v = static_cast<const T *>(a.v.data) + t * a.v.token_stride + mine * a.v.head_stride;
    const int64_t q_step = G * a.q.head_stride, k_step = G * a.k.head_stride, v_step = G * a.v.head_stride;
    const int k0 = max(first, q_steps) - q_steps, k1 = min(last - q_steps, kv_steps);
    const int v0 = max(first - q_steps - kv_steps, 0), v1 = last - q_steps - kv_steps;
    Batch<T, kBatch> batch;
    if (there) {
        if (first < q_steps)
            batch.template load<G>(q, q_step, first, min(last, q_steps), a.num_q_heads, mine, e0, e1);
        else if (k0 < k1)
            batch.template load<G>(k, k_step, k0, k1, a.num_kv_heads, mine, e0, e1);
    }

    unsigned long long cs[4], sn[4];
    if (a.rot.half && first < q_steps + kv_steps) {
        float2 own[kMake];
#pragma unroll
        for (int i = 0; i < kMake; ++i)
            own[i] = rotates && there ? turn(a.rot, t, 8 * u + kMake * mine + i) : make_float2(1.f, 0.f);
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int from = (team * G + i / kMake) * kLanes + u;
            c[i] = G == 1 ? own[i % kMake].x : __shfl_sync(0xffffffffu, own[i % kMake].x, from);
            s[i] = G == 1 ? own[i % kMake].y : __shfl_sync(0xffffffffu, own[i % kMake].y, from);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            cs[i] = dev::f32x2(c[2 * i], c[2 * i + 1]);
            sn[i] = dev::f32x2(s[2 * i], s[2 * i + 1]);
        }
    }
    if (!there) return;
    if (first < q_steps)
        write_heads<T, T, G, true, kBatch>(batch, q, q_step, static_cast<T *>(a.q_out) + (t * a.num_q_heads + mine) * D,
                                           G * D, first, min(last, q_steps), a.num_q_heads, mine, e0, e1, INTERLEAVED,
                                           rotates, cs, sn, nullptr);
    if (slot < 0 || slot >= a.num_slots || last <= q_steps) return;
    const int64_t row = (slot / kPageSize * a.num_kv_heads + mine) * kPageSize * D + slot % kPageSize * D;
    if (k0 < k1) {
        if (first < q_steps) batch.template load<G>(k, k_step, k0, k1, a.num_kv_heads, mine, e0, e1);
        write_heads<T, KV, G, true, kBatch>(batch, k, k_step, static_cast<KV *>(a.k_pages) + row, G * kPageSize * D, k0,
                                            k1, a.num_kv_heads, mine, e0, e1, INTERLEAVED, rotates, cs, sn, a.k_scale);
    }
    if (v0 < v1) {
        batch.template load<G>(v, v_step, v0, v1, a.num_kv_heads, mine, 16 * u, 16 * u + 8);
        write_heads<T, KV, G, false, kBatch>(batch, v, v_step, static_cast<KV *>(a.v_pages) + row, G * kPageSize * D,
                                             v0, v1, a.num_kv_heads, mine, 16 * u, 16 * u + 8, INTERLEAVED, false, cs,
                                             sn, a.v_scale);
    }
}

// Sixteen consecutive elements, as two of the units above.
template <class T>
struct Raw16 {
    Raw8<T> h[2];
};

template <class T>
__device__ __forceinline__ Raw16<T> load16(const T *p) {
    Raw16<T> r;
    if constexpr (sizeof(T) == 1) {
        const uint4 u = __ldcs(reinterpret_cast<const uint4 *>(p));
        r.h[0].w[0] = u.x;
        r.h[0].w[1] = u.y;
        r.h[1].w[0] = u.z;
        r.h[1].w[1] = u.w;
    } else {
        r.h[0] = load8(p);
        r.h[1] = load8(p + 8);
    }
    return r;
}

// 32 bytes in one store where they are aligned so (whole sectors), else 16 and 16.
__device__ __forceinline__ void store32(void *p, const uint32_t (&w)[8], bool aligned) {
    if (aligned) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]),
                     "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        reinterpret_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// 16 elements of the cache as the caller's: bits where the types are the same.
template <class T, class KV>
__device__ __forceinline__ void store_read16(T *dst, const Raw16<KV> &r, float scale, bool aligned) {
    if constexpr (kScaled<KV>) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t h;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;"
                : "=r"(h)
                : "h"(static_cast<uint16_t>(r.h[i >> 2].w[(i >> 1) & 1] >> (16 * (i & 1)))));
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
            float lo, hi;
            dev::f32x2_split(dev::mul_f32x2(dev::f32x2(f.x, f.y), dev::f32x2(scale, scale)), lo, hi);
            w[i] = dev::pack_bf16(lo, hi);
        }
        store32(dst, w, aligned);
    } else if constexpr (sizeof(T) == 2) {
        const uint32_t w[8] = {r.h[0].w[0], r.h[0].w[1], r.h[0].w[2], r.h[0].w[3],
                               r.h[1].w[0], r.h[1].w[1], r.h[1].w[2], r.h[1].w[3]};
        store32(dst, w, aligned);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) store32(dst + 8 * i, r.h[i].w, aligned);
    }
}

// Rows (token, head) in order: a warp takes kSteps x (32 / kLanes) of them, K and V of
// each, a lane 16 elements, all loads in flight.  38.8k e4m3 tokens of 8 heads: 37.2 us
// (35.2 us of bytes), fp32 95.5 (93.8); 8 elements a lane, whose scales and addresses
// then come twice as often, 39.6 in e4m3; a warp to a token leaves lanes without a head
// where there are few (38.4k bf16 tokens of one head 6.2 us, 13.1 so).
template <class T, class KV, int D>
__global__ void __launch_bounds__(kThreads, 8) kv_read_kernel(const ReadArgs a) {
    constexpr int kLanes = D / 16, kGroups = 32 / kLanes, kSteps = sizeof(T) == 4 ? 1 : 2;
    const int lane = threadIdx.x % 32, u = lane % kLanes, mine = lane / kLanes;
    // the warp's first row: token t0, head h0
    const int64_t row0 = (static_cast<int64_t>(blockIdx.x) * kWarps + threadIdx.x / 32) * (kGroups * kSteps);
    int64_t t0;
    if (a.short_rows)
        t0 = static_cast<uint32_t>(row0) / static_cast<uint32_t>(a.num_kv_heads);
    else
        t0 = row0 / a.num_kv_heads;
    const uint32_t h0 = static_cast<uint32_t>(row0 - t0 * a.num_kv_heads);
    dev::grid_wait();
    Raw16<KV> rk[kSteps], rv[kSteps];
    float ks[kSteps], vs[kSteps];
    int64_t t[kSteps];
    int h[kSteps];
#pragma unroll
    for (int b = 0; b < kSteps; ++b) {
        const uint32_t at = h0 + b * kGroups + mine, over = a.heads_magic ? __umulhi(at, a.heads_magic) : at;
        t[b] = t0 + over;
        h[b] = static_cast<int>(at - over * a.num_kv_heads);
        if (t[b] >= a.num_tokens) continue;
        const int64_t slot = a.slots[t[b]];
        if (slot >= 0 && slot < a.num_slots) {
            const int64_t at_row = ((slot / kPageSize * a.num_kv_heads + h[b]) * kPageSize + slot % kPageSize) * D + 16 * u;
            rk[b] = load16(static_cast<const KV *>(a.k_pages) + at_row);
            rv[b] = load16(static_cast<const KV *>(a.v_pages) + at_row);
            if constexpr (kScaled<KV>) {
                ks[b] = a.k_scale[h[b]];
                vs[b] = a.v_scale[h[b]];
            }
        } else {
            rk[b] = rv[b] = Raw16<KV>{};
            ks[b] = vs[b] = 0.f;
        }
    }
#pragma unroll
    for (int b = 0; b < kSteps; ++b) {
        if (t[b] >= a.num_tokens) continue;
        T *k = static_cast<T *>(const_cast<void *>(a.k.data)) + t[b] * a.k.token_stride + h[b] * a.k.head_stride;
        T *v = static_cast<T *>(const_cast<void *>(a.v.data)) + t[b] * a.v.token_stride + h[b] * a.v.head_stride;
        store_read16<T, KV>(k + 16 * u, rk[b], ks[b], a.aligned);
        store_read16<T, KV>(v + 16 * u, rv[b], vs[b], a.aligned);
    }
}

// Scales at their least, 2^-126, before the tokens raise them.
__global__ void reset_scales_kernel(float *k_scale, float *v_scale, int n) {
    dev::grid_wait();
    for (int i = threadIdx.x; i < n; i += blockDim.x) k_scale[i] = v_scale[i] = 1.17549435e-38f;
}

// min(|x|, 2^63), 0 for NaN: squares of these add up within fp32.
__device__ __forceinline__ float magnitude(float x) { return x == x ? fminf(fabsf(x), 9.2233720369e18f) : 0.f; }

// The larger magnitudes of two bf16 pairs (signs are not kept apart; NaN loses).
__device__ __forceinline__ uint32_t most_bf16x2(uint32_t a, uint32_t b) {
    uint32_t m;
    asm("max.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
}

// A warp takes kScaleRows tokens of one head of K or of V, all their loads in flight, a
// lane 16 elements of a token as kv_write takes them (more tokens a warp: 1024 tokens of
// 2 heads 3.3 us with 32, 5.0 with 64, for 2.6).  max |x| goes in bf16 pairs, two elements an
// instruction; squares of pairs in packed fp32.  Where their largest sum is past 2^126
// (elements from 2^62 on, infinities) or below 2^-100 (squares that lose bits, or are
// 0), the warp goes over its tokens once more, with magnitudes cut at 2^63, or taken
// times 2^100 before they are squared.  A NaN's partner counts in max |x|.
//
// Positive floats order as their bits do, so the maxima meet in integer atomics, whose
// order does not matter; max / 448 is the max of the quotients, since rounding is
// monotone.  A CTA's warps meet first: an atomic a warp took 33 us for the 21.1 of 32768
// tokens of 8 heads (19.8 us of bytes).  CTAs go over the heads of the same tokens
// first, whose rows are neighbours (head by head 22.3 us).
constexpr int kScaleRows = 16;
template <int D>
__global__ void __launch_bounds__(kThreads, 8) kv_scales_kernel(const ScalesArgs a) {
    constexpr int kLanes = D / 16, kRows = 32 / kLanes, kBatch = kScaleRows / kRows;
    __shared__ float part[kWarps];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rest = blockIdx.x / static_cast<uint32_t>(a.num_kv_heads);
    const int h = blockIdx.x - rest * a.num_kv_heads;
    const bool is_k = rest % 2 == 0;
    const Rows &src = is_k ? a.k : a.v;
    const int half = is_k ? a.half : 0;
    const int u = lane % kLanes;
    const bool rotates = 8 * u < half, halves = rotates && !a.interleaved;
    const int e0 = halves ? 8 * u : 16 * u, e1 = e0 + (halves ? half : 8);
    const int64_t t0 = (static_cast<int64_t>(rest / 2) * kWarps + warp) * kScaleRows + lane / kLanes;
    const __nv_bfloat16 *x = static_cast<const __nv_bfloat16 *>(src.data) + h * src.head_stride;
    dev::grid_wait();
    uint32_t one = 0;                    // max |x| of even and of odd elements
    float pair = 0.f;                    // max of x0^2 + x1^2
    Raw8<__nv_bfloat16> r0[kBatch], r1[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
        const int64_t t = t0 + b * kRows;
        if (t < a.num_tokens && (!a.slots || a.slots[t] >= 0)) {
            r0[b] = load8(x + t * src.token_stride + e0);
            r1[b] = load8(x + t * src.token_stride + e1);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) r0[b].w[i] = r1[b].w[i] = 0;
        }
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t p = r0[b].w[i], q = r1[b].w[i];
            one = most_bf16x2(one, most_bf16x2(p, q));
            if (rotates) {
                // halves: elements i of both chunks; neighbours: within a word
                const float p0 = __uint_as_float(p << 16), p1 = __uint_as_float(p & 0xffff0000u);
                const float q0 = __uint_as_float(q << 16), q1 = __uint_as_float(q & 0xffff0000u);
                const unsigned long long v = halves ? dev::f32x2(p0, p1) : dev::f32x2(p0, q0);
                const unsigned long long w = halves ? dev::f32x2(q0, q1) : dev::f32x2(p1, q1);
                float s0, s1;
                dev::f32x2_split(dev::fma_f32x2(v, v, dev::mul_f32x2(w, w)), s0, s1);
                pair = dev::max3(pair, s0, s1);
            }
        }
    }
    float m = fmaxf(magnitude(__uint_as_float(one << 16)), magnitude(__uint_as_float(one & 0xffff0000u)));
    if (half > 0) {
        const float most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(pair)));
        const bool tiny = most < 0x1p-100f && __any_sync(0xffffffffu, m > 0.f);
        if (tiny || most > 0x1p126f) {
            const float up = tiny ? 0x1p100f : 1.f;
            pair = 0.f;
            for (int r = 0; rotates && r < kScaleRows; r += kRows) {
                const int64_t t = t0 + r;
                if (t >= a.num_tokens || (a.slots && a.slots[t] < 0)) continue;
                float x0[8], x1[8];
                unpack8(load8(x + t * src.token_stride + e0), x0);
                unpack8(load8(x + t * src.token_stride + e1), x1);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p = magnitude(up * (halves ? x0[i] : (i < 4 ? x0 : x1)[2 * (i & 3)]));
                    const float q = magnitude(up * (halves ? x1[i] : (i < 4 ? x0 : x1)[2 * (i & 3) + 1]));
                    pair = fmaxf(pair, p * p + q * q);
                }
            }
            pair = sqrtf(pair) * (tiny ? 0x1p-100f : 1.f);
        } else {
            pair = sqrtf(pair);
        }
        m = fmaxf(m, pair);
    }
    m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
    if (lane == 0) part[warp] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kWarps; ++i) m = fmaxf(m, part[i]);
        atomicMax(reinterpret_cast<int *>((is_k ? a.k_scale : a.v_scale) + h), __float_as_int(m / kE4m3Max));
    }
}

// Warps of kv_write (a token to a warp) that run at once on the current device, one
// wave: asked for once a device.
template <class T, class KV, int D, bool INTERLEAVED>
cudaError_t wave_warps(int64_t *warps) {
    static std::atomic<int> known[kMaxDevices];          // 0: not asked yet
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorNotSupported;
    int n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        int sms = 0, ctas = 0;
        e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e == cudaSuccess)
            e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&ctas, kv_write_kernel<T, KV, D, INTERLEAVED, 512 / D>,
                                                              kThreads, 0);
        if (e != cudaSuccess) return e;
        n = sms * ctas * kWarps;
        known[dev].store(n, std::memory_order_relaxed);
    }
    *warps = n;
    return cudaSuccess;
}

// Parts of a token: as many as one wave of warps has room for, of one step at least
// (1200 tokens of 32 / 8 heads: 5.5 us in 2 parts, 7.1 in 3, whose warps wait for a
// place and make the same angles again).
int parts_of(int64_t tokens, int steps, int64_t wave) {
    const int64_t room = wave / tokens;
    return static_cast<int>(room < 1 ? 1 : room < steps ? room : steps);
}

unsigned blocks_of(int64_t tokens, int parts) {
    return static_cast<unsigned>((tokens * parts + kWarps - 1) / kWarps);
}

template <class T, class KV, int D, int G>
cudaError_t launch_write(WriteArgs a, int64_t wave, cudaStream_t s) {
    constexpr int kTeams = 512 / D / G;
    const int steps = (a.num_q_heads + G - 1) / G + 2 * ((a.num_kv_heads + G - 1) / G);
    a.parts = kTeams == 1 ? parts_of(a.num_tokens, steps, wave) : 1;
    return launch_dependent(
        true, a.rot.interleaved ? kv_write_kernel<T, KV, D, true, G> : kv_write_kernel<T, KV, D, false, G>,
        dim3(blocks_of((a.num_tokens + kTeams - 1) / kTeams, a.parts)), dim3(kThreads), 0, s, a);
}

// A token to a warp, or two or four of them where a token is fewer than 10 steps and
// their warps would pass one wave: a short warp spends its life on its slot, its angles and its
// first loads (9728 bf16 tokens of 128 elements, a token, two and four to a warp: 14.1,
// 11.9, 10.0 us at 8 / 2 heads, 4 to 12 steps; 22.0, 19.2, 19.0 at 16 / 4; 34.1, 35.0,
// 34.5 at 24 / 8, 10 to 40 steps).
template <class T, class KV, int D>
cudaError_t launch_write(const WriteArgs &a, cudaStream_t s) {
    constexpr int kGroups = 512 / D;
    int64_t wave = 0;
    const cudaError_t e = a.rot.interleaved ? wave_warps<T, KV, D, true>(&wave) : wave_warps<T, KV, D, false>(&wave);
    if (e != cudaSuccess) return e;
    auto few = [&](int g) {
        return (a.num_q_heads + g - 1) / g + 2 * ((a.num_kv_heads + g - 1) / g) < 10 &&
               a.num_tokens > kGroups / g * wave;
    };
    if (!few(kGroups)) return launch_write<T, KV, D, kGroups>(a, wave, s);
    return few(kGroups / 2) ? launch_write<T, KV, D, kGroups / 4>(a, wave, s)
                            : launch_write<T, KV, D, kGroups / 2>(a, wave, s);
}

template <class T, class KV, int D>
cudaError_t launch_read(ReadArgs a, cudaStream_t s) {
    constexpr int kRowsOfCta = kWarps * (32 / (D / 16)) * (sizeof(T) == 4 ? 1 : 2);
    uintptr_t odd = 0;
    for (const Rows *r : {&a.k, &a.v})
        odd |= reinterpret_cast<uintptr_t>(r->data) | static_cast<uintptr_t>(r->token_stride * sizeof(T)) |
               static_cast<uintptr_t>(r->head_stride * sizeof(T));
    a.aligned = odd % 32 == 0;
    a.heads_magic = static_cast<uint32_t>(((1ull << 32) + a.num_kv_heads - 1) / a.num_kv_heads);
    const int64_t rows = a.num_tokens * a.num_kv_heads, ctas = (rows + kRowsOfCta - 1) / kRowsOfCta;
    a.short_rows = ctas * kRowsOfCta <= UINT32_MAX;
    return launch_dependent(true, kv_read_kernel<T, KV, D>, dim3(static_cast<unsigned>(ctas)), dim3(kThreads), 0, s, a);
}

// ---------------------------------------------------------------- arguments

bool misaligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

parason_status check_rows(const parason_rows *r, int64_t tokens, int32_t heads, int32_t d, int elem, bool out) {
    if (!r || !r->data || misaligned(r->data, 16)) return PARASON_EINVAL;
    const int64_t strides[2] = {tokens > 1 ? r->token_stride : d, heads > 1 ? r->head_stride : d};
    for (int64_t st : strides) {
        if (st < 0 || st * elem % 16 != 0) return PARASON_EINVAL;
    }
    if (out) {
        // rows apart: the nearer dimension's stride is a row at least, the other's its whole reach
        const int64_t counts[2] = {tokens, heads};
        const int near = (tokens > 1 && strides[0] <= strides[1]) || heads <= 1 ? 0 : 1;
        if (strides[near] < d) return PARASON_EINVAL;
        if (counts[1 - near] > 1 && (strides[1 - near] - d) / strides[near] < counts[near] - 1) return PARASON_EINVAL;
    }
    return PARASON_OK;
}

Rows to_rows(const parason_rows *r) { return Rows{r->data, r->token_stride, r->head_stride}; }

// the checks every call shares
parason_status check_call(const parason_attn_config *cfg, int64_t tokens, int64_t pages) {
    const parason_status st = check_config(cfg);
    if (st != PARASON_OK) return st;
    if (tokens < 0 || tokens > INT32_MAX || pages < 0) return PARASON_EINVAL;
    if (cfg->num_q_heads > kMaxHeads || cfg->num_kv_heads > kMaxHeads) return PARASON_EUNSUPPORTED;
    if (pages > INT32_MAX / kPageSize / cfg->num_kv_heads) return PARASON_EUNSUPPORTED;
    return PARASON_OK;
}

// the part of a rotary description that kv_scales uses too
parason_status check_pairs(const parason_rotary *r, int32_t d) {
    if (r->rotary_dim <= 0 || r->rotary_dim > d || r->rotary_dim % 16 != 0) return PARASON_EINVAL;
    if (r->pairs != PARASON_ROTARY_HALVES && r->pairs != PARASON_ROTARY_INTERLEAVED) return PARASON_EINVAL;
    return PARASON_OK;
}

parason_status to_rotary(const parason_rotary *r, int64_t tokens, int32_t d, RotaryArgs *out) {
    *out = RotaryArgs{};
    if (!r) return PARASON_OK;
    const parason_status st = check_pairs(r, d);
    if (st != PARASON_OK) return st;
    if (r->num_axes < 1 || r->num_axes > kMaxAxes || !r->turns || (!r->positions && tokens > 0) ||
        misaligned(r->turns, 8) || misaligned(r->positions, 4) || (r->num_axes > 1 && r->position_stride < 0))
        return PARASON_EINVAL;
    out->turns = r->turns;
    out->positions = r->positions;
    out->position_stride = r->num_axes > 1 ? r->position_stride : 0;
    out->half = r->rotary_dim / 2;
    out->interleaved = r->pairs == PARASON_ROTARY_INTERLEAVED;
    for (int i = 0; r->freq_axis && i < out->half; ++i) {
        if (r->freq_axis[i] >= r->num_axes) return PARASON_EINVAL;
        out->axes[i / 32] |= static_cast<uint64_t>(r->freq_axis[i]) << (2 * (i % 32));
    }
    return PARASON_OK;
}

// 1 / (2 pi) in 2^-192, most significant 64 bits first
constexpr uint64_t kInvTwoPi[3] = {0x28be60db9391054aull, 0x7f09d5f47d4d3770ull, 0x36d8a5664f10e410ull};

// |f| / (2 pi) modulo 1 in 2^-64: f = m 2^e, and m kInvTwoPi 2^(e + 64 - 192) rounded.
// (kInvTwoPi is below 1 / (2 pi) by less than 2^-192, so the product by less than
// 2^24 2^(e - 192): 2^-127 of a turn at e = 41, the largest.)
uint64_t turns_of(float f) {
    int e = 0;
    const uint64_t m = static_cast<uint64_t>(std::ldexp(std::frexp(std::fabs(f), &e), 24));
    e -= 24;
    uint64_t w[5] = {0, 0, 0, 0, 0};                     // m kInvTwoPi, least significant first
    unsigned __int128 carry = 0;
    for (int i = 0; i < 3; ++i) {
        carry += static_cast<unsigned __int128>(m) * kInvTwoPi[2 - i];
        w[i] = static_cast<uint64_t>(carry);
        carry >>= 64;
    }
    w[3] = static_cast<uint64_t>(carry);
    const int shift = 128 - e;                           // 87 and up for |f| <= 2^64
    if (shift > 256) return 0;
    const int half = shift - 1;                          // the bit that rounds
    unsigned __int128 up = static_cast<unsigned __int128>(1) << (half % 64);
    for (int i = half / 64; i < 5; ++i) {
        up += w[i];
        w[i] = static_cast<uint64_t>(up);
        up >>= 64;
    }
    if (shift == 256) return w[4];
    const int at = shift / 64, by = shift % 64;
    return by ? (w[at] >> by) | (w[at + 1] << (64 - by)) : w[at];
}

parason_status launched(cudaError_t e) { return e == cudaSuccess ? PARASON_OK : PARASON_ECUDA; }

}  // namespace
}  // namespace parason

using namespace parason;

extern "C" parason_status parason_rotary_turns(const float *inv_freq, int32_t n, uint64_t *turns) {
    if (n < 0 || (n > 0 && (!inv_freq || !turns))) return PARASON_EINVAL;
    for (int32_t i = 0; i < n; ++i)
        if (!(std::fabs(inv_freq[i]) <= 0x1p64f)) return PARASON_EINVAL;
    for (int32_t i = 0; i < n; ++i) {
        const uint64_t t = turns_of(inv_freq[i]);
        turns[i] = inv_freq[i] < 0.f ? 0 - t : t;
    }
    return PARASON_OK;
}

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
    if ((st = to_rotary(rotary, num_tokens, d, &a.rot)) != PARASON_OK) return st;
    if (num_tokens == 0) return PARASON_OK;
    if ((st = check_rows(k, num_tokens, cfg->num_kv_heads, d, elem, false)) != PARASON_OK) return st;
    if ((st = check_rows(v, num_tokens, cfg->num_kv_heads, d, elem, false)) != PARASON_OK) return st;
    if (q && (st = check_rows(q, num_tokens, cfg->num_q_heads, d, elem, false)) != PARASON_OK) return st;
    if (q && (!q_out || misaligned(q_out, 16))) return PARASON_EINVAL;
    // (in place: the rows as q_out has them, or a row would be written before it is read)
    if (q && q_out == q->data &&
        ((num_tokens > 1 && q->token_stride != static_cast<int64_t>(cfg->num_q_heads) * d) ||
         (cfg->num_q_heads > 1 && q->head_stride != d)))
        return PARASON_EINVAL;
    if (!slots || misaligned(slots, 4)) return PARASON_EINVAL;
    if (num_physical_pages > 0 && (!k_pages || !v_pages || misaligned(k_pages, 16) || misaligned(v_pages, 16)))
        return PARASON_EINVAL;
    if (cfg->mode == PARASON_FP8_E4M3_KV &&
        (!k_scale || !v_scale || misaligned(k_scale, 4) || misaligned(v_scale, 4)))
        return PARASON_EINVAL;
    // (outputs in one place: two warps would write it, or one before another has read it)
    if (num_physical_pages > 0 && k_pages == v_pages) return PARASON_EINVAL;
    if (q && (q_out == k->data || q_out == v->data)) return PARASON_EINVAL;
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
    if (num_tokens * cfg->num_kv_heads > kMaxRows) return PARASON_EUNSUPPORTED;
    if (k_out->data == v_out->data) return PARASON_EINVAL;
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
    if (num_tokens * cfg->num_kv_heads > kMaxRows) return PARASON_EUNSUPPORTED;
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
    const int64_t ctas = (num_tokens + kWarps * kScaleRows - 1) / (kWarps * kScaleRows) * 2 * cfg->num_kv_heads;
    return launched(launch_dependent(true, kv_scales_kernel<128>, dim3(static_cast<unsigned>(ctas)), dim3(kThreads), 0,
                                     s, a));
}
