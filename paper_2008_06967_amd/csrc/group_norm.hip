// Group normalisation with an activation, channels last.
#include <algorithm>
#include <cmath>

#include "common.h"

namespace meso {

namespace {

constexpr int kGnThreads = 256;

template <typename T>
__device__ __forceinline__ float gn_load(const T* p) {
    if constexpr (sizeof(T) == 4)
        return *p;
    else
        return bf16_to_f32(*p);
}

template <typename T>
__device__ __forceinline__ void gn_store(T* p, float v) {
    if constexpr (sizeof(T) == 4)
        *p = v;
    else
        *p = f32_to_bf16_any(v);
}

__device__ __forceinline__ float gn_act(float v, int act) {
    switch (act) {
        case MESORASI_ACT_RELU: return v < 0.0f ? 0.0f : v;
        case MESORASI_ACT_SILU: return v / (1.0f + expf(-v));
        case MESORASI_ACT_GELU: return 0.5f * v * (1.0f + erff(v * 0.70710678f));
        default: return v;
    }
}

__device__ __forceinline__ float gn_block_sum(float v, float* sh) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = 0.0f;
    for (int i = 0; i < kGnThreads / 64; ++i) t += sh[i];
    return t;
}

// One workgroup per cloud and group: mean, variance, output, a pass each.
template <typename TX, typename TY>
__global__ __launch_bounds__(kGnThreads) void group_norm_kernel(const TX* __restrict__ x, int64_t ldx, int64_t N, int C,
                                                                int G, const int32_t* __restrict__ lens,
                                                                const float* __restrict__ gamma,
                                                                const float* __restrict__ beta, float eps, int act,
                                                                TY* __restrict__ y, int64_t ldy) {
    __shared__ float sh[kGnThreads / 64];
    const int64_t b = blockIdx.x / G;
    const int g = (int)(blockIdx.x % G), c = C / G;
    const int64_t n = lens ? min(max((int64_t)lens[b], (int64_t)0), N) : N;
    const TX* xb = x + b * N * ldx + (int64_t)g * c;
    TY* yb = y + b * N * ldy + (int64_t)g * c;
    const int64_t total = n * c;
    // differences to a value of the group keep the spread's precision
    const float pv = n > 0 ? gn_load(xb) : 0.0f;
    float s = 0.0f;
    for (int64_t i = threadIdx.x; i < total; i += kGnThreads) s += gn_load(xb + (i / c) * ldx + i % c) - pv;
    const float mu = gn_block_sum(s, sh) / (float)total;
    s = 0.0f;
    for (int64_t i = threadIdx.x; i < total; i += kGnThreads) {
        const float d = gn_load(xb + (i / c) * ldx + i % c) - pv - mu;
        s += d * d;
    }
    const float rs = 1.0f / sqrtf(gn_block_sum(s, sh) / (float)total + eps);
    for (int64_t i = threadIdx.x; i < N * c; i += kGnThreads) {
        const int64_t r = i / c;
        const int ch = (int)(i % c), cc = g * c + ch;
        float v = 0.0f;
        if (r < n) {
            v = (gn_load(xb + r * ldx + ch) - pv - mu) * rs;
            v = gn_act(v * (gamma ? gamma[cc] : 1.0f) + (beta ? beta[cc] : 0.0f), act);
        }
        gn_store(yb + r * ldy + ch, v);
    }
}

}  // namespace

}  // namespace meso

using namespace meso;

extern "C" size_t mesorasi_group_norm_workspace(int64_t B, int64_t N, int32_t C, int32_t G, int32_t x_dtype) {
    return 0;
}

extern "C" int mesorasi_group_norm(const void* x, int64_t ld_x, int32_t x_dtype, int64_t B, int64_t N, int32_t C,
                                   int32_t G, const int32_t* lens, const float* gamma, const float* beta, float eps,
                                   int32_t act, void* y, int64_t ld_y, int32_t y_dtype, void* ws, size_t ws_bytes,
                                   void* stream) {
    MESO_REQUIRE(B >= 0 && N >= 0, MESORASI_EINVAL, "mesorasi_group_norm: negative size");
    MESO_REQUIRE(C >= 1 && G >= 1 && C % G == 0, MESORASI_EINVAL, "mesorasi_group_norm: C = %d, G = %d", C, G);
    MESO_REQUIRE(ld_x >= C && ld_y >= C, MESORASI_EINVAL, "mesorasi_group_norm: leading dimension < C");
    MESO_REQUIRE(act >= MESORASI_ACT_NONE && act <= MESORASI_ACT_GELU, MESORASI_EINVAL, "mesorasi_group_norm: act %d",
                 act);
    MESO_REQUIRE(std::isfinite(eps) && eps >= 0.0f, MESORASI_EINVAL, "mesorasi_group_norm: eps = %g", (double)eps);
    MESO_REQUIRE((x_dtype == MESORASI_F32 || x_dtype == MESORASI_BF16) &&
                     (y_dtype == MESORASI_F32 || y_dtype == MESORASI_BF16),
                 MESORASI_EUNSUPPORTED, "mesorasi_group_norm: dtypes %d, %d", x_dtype, y_dtype);
    MESO_REQUIRE(C <= MESORASI_MAX_C_NORM && N <= 0x7fffffff && B <= 0x7fffffff / G, MESORASI_EUNSUPPORTED,
                 "mesorasi_group_norm: B = %lld, N = %lld, C = %d", (long long)B, (long long)N, C);
    if (B == 0 || N == 0) return MESORASI_OK;
    MESO_REQUIRE(x && y, MESORASI_EINVAL, "mesorasi_group_norm: NULL x or y");
    hipStream_t s = as_stream(stream);
    const dim3 grid((unsigned)(B * G)), block(kGnThreads);
#define MESO_GN(TX, TY)                                                                                          \
    group_norm_kernel<TX, TY><<<grid, block, 0, s>>>(static_cast<const TX*>(x), ld_x, N, C, G, lens, gamma, beta, \
                                                     eps, act, static_cast<TY*>(y), ld_y)
    if (x_dtype == MESORASI_F32) {
        if (y_dtype == MESORASI_F32) MESO_GN(float, float);
        else MESO_GN(float, uint16_t);
    } else {
        if (y_dtype == MESORASI_F32) MESO_GN(uint16_t, float);
        else MESO_GN(uint16_t, uint16_t);
    }
#undef MESO_GN
    return after_launch("mesorasi_group_norm");
}
