// Shared by the router block's kernels (router_tf.hip, router_fused.hip).
#pragma once

#include "common.hpp"
#include "internal.hpp"

namespace readme {

// The router block's two fused kernels (router_fused.hip): D = 512, a padded
// MLP width of at most kFusedRouterMlp.
constexpr int kFusedRouterWidth = 512;
constexpr int kFusedRouterMlp = 1536;
// Tokens from which the two kernels are the faster form (router_fused.hip).
inline int64_t fused_router_tokens(int64_t F) { return 1800 + F * 7 / 5; }
// `given`: pos holds the positions (else they are found from ro and written).
hipError_t launch_router_head(int64_t T, int32_t R, int64_t V, float eps, const int32_t* tokens,
                              const int32_t* ro, const void* emb, float* x, uint16_t* a,
                              int32_t* pos, bool given, int32_t* offs, const void* wqkv,
                              uint16_t* qkv, hipStream_t s);
hipError_t launch_router_tail(int64_t T, int64_t F, int E, float eps, const uint16_t* o,
                              const void* wo, const void* mlp, const void* gate, const float* bias,
                              float* x, uint16_t* m, uint16_t* h, uint16_t* f, int32_t* ids,
                              float* logits, hipStream_t s);

// Request offsets staged in LDS for the position search when they fit.
constexpr int kRoLds = 4096;

// Position of token t in its request: t - ro[r] for the last r with
// ro[r] <= t (ro = request offsets [R + 1], ro[0] = 0, ro[R] = T).
__device__ __forceinline__ int32_t position_of(int64_t t, int32_t R,
                                               const int32_t* __restrict__ ro) {
    int lo = 0, hi = R;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (ro[mid] <= t) lo = mid;
        else hi = mid;
    }
    int64_t start = ro[lo];
    if (start < 0) start = 0;
    if (start > t) start = t;
    return (int32_t)(t - start);
}

// Sum over the wave to lane 0 in a fixed order, then broadcast, so that every
// lane holds the same fp32 total.
__device__ __forceinline__ float wave_sum_bcast(float v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_down(v, off, 64);
    return __shfl(v, 0, 64);
}

}  // namespace readme
