// logit_cap.cuh -- scores <q, k> to capped logits in the log2 domain:
//   x = cap_log2 * tanh(to_cap * <q, k>),  cap_log2 = cap * log2(e),
//   to_cap = sm_scale / cap (times the kv head's K scale with e4m3 KV).
#pragma once

#include "device_common.cuh"

namespace parason {
namespace {

template <int N>
__device__ __forceinline__ void cap_scores(float (&x)[N], float to_cap, float cap_log2) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = cap_log2 * tanhf(x[i] * to_cap);
}

template <int M, int N>
__device__ __forceinline__ void cap_scores(float (&x)[M][N], float to_cap, float cap_log2) {
#pragma unroll
    for (int i = 0; i < M; ++i) cap_scores<N>(x[i], to_cap, cap_log2);
}

// the same for scores held as bits
template <int N>
__device__ __forceinline__ void cap_scores(uint32_t (&x)[N], float to_cap, float cap_log2) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __float_as_uint(cap_log2 * tanhf(__uint_as_float(x[i]) * to_cap));
}

}  // namespace
}  // namespace parason
