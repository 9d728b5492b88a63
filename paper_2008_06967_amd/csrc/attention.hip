// Cross attention to another set of points.
#include <algorithm>
#include <cmath>

#include "common.h"

namespace meso {

namespace {

struct AttnArgs {
    const void* q;
    const void* k;
    const void* v;
    void* o;
    int64_t qb, ql, qh, kb, kl, kh, vb, vl, vh, ob, ol, oh;   // strides: cloud, point, head
    int64_t Nq, Nk, mask_ld;
    int Hq, Hkv, D;
    float scale;
    const int32_t* k_len;
    const uint8_t* k_mask;
};

template <typename T>
__device__ __forceinline__ float at_load(const T* p) {
    if constexpr (sizeof(T) == 4)
        return *p;
    else
        return bf16_to_f32(*p);
}

// One wave per query and head: 64 sources at a time, a source per lane for
// the scores, a channel (two for D > 64) per lane for the output.
template <typename T>
__global__ __launch_bounds__(64) void attention_kernel(AttnArgs a, int64_t total) {
    __shared__ float qs[MESORASI_MAX_D_ATTN];
    __shared__ float ps[64];
    const int lane = threadIdx.x;
    const int64_t e = blockIdx.x;
    const int h = (int)(e % a.Hq);
    const int64_t n = e / a.Hq % a.Nq, b = e / a.Hq / a.Nq;
    const int kvh = h / (a.Hq / a.Hkv);
    const T* q = static_cast<const T*>(a.q) + b * a.qb + n * a.ql + h * a.qh;
    const T* k = static_cast<const T*>(a.k) + b * a.kb + kvh * a.kh;
    const T* v = static_cast<const T*>(a.v) + b * a.vb + kvh * a.vh;
    T* o = static_cast<T*>(a.o) + b * a.ob + n * a.ol + h * a.oh;
    const int64_t len = a.k_len ? min(max((int64_t)a.k_len[b], (int64_t)0), a.Nk) : a.Nk;
    const uint8_t* mask = a.k_mask ? a.k_mask + b * a.mask_ld : nullptr;
    for (int c = lane; c < a.D; c += 64) qs[c] = at_load(q + c) * a.scale;
    __syncthreads();
    float m = -INFINITY, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
    for (int64_t j0 = 0; j0 < len; j0 += 64) {
        const int64_t j = j0 + lane;
        const bool ok = j < len && (!mask || mask[j]);
        float s = -INFINITY;
        if (ok) {
            s = 0.0f;
            for (int c = 0; c < a.D; ++c) s = fmaf(qs[c], at_load(k + j * a.kl + c), s);
        }
        float mt = s;
        for (int w = 32; w; w >>= 1) mt = fmaxf(mt, __shfl_xor(mt, w));
        const float mn = fmaxf(m, mt);
        const float base = mn == -INFINITY ? 0.0f : mn;
        const float p = expf(s - base);
        float lt = p;
        for (int w = 32; w; w >>= 1) lt += __shfl_xor(lt, w);
        const float f = expf(m - base);
        l = l * f + lt;
        o0 *= f;
        o1 *= f;
        m = mn;
        __syncthreads();
        ps[lane] = p;
        __syncthreads();
        const uint64_t okm = ballot(ok);
        for (int i = 0; i < 64; ++i) {
            if (!((okm >> i) & 1)) continue;
            const T* vr = v + (j0 + i) * a.vl;
            if (lane < a.D) o0 = fmaf(ps[i], at_load(vr + lane), o0);
            if (lane + 64 < a.D) o1 = fmaf(ps[i], at_load(vr + lane + 64), o1);
        }
    }
    const float r = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    for (int i = 0; i < 2; ++i) {
        const int c = lane + 64 * i;
        if (c >= a.D) continue;
        const float w = (i ? o1 : o0) * r;
        if constexpr (sizeof(T) == 4)
            o[c] = w;
        else
            o[c] = f32_to_bf16_any(w);
    }
}

}  // namespace

}  // namespace meso

using namespace meso;

extern "C" size_t mesorasi_cross_attention_workspace(int64_t B, int64_t Nq, int64_t Nk, int32_t Hq, int32_t Hkv,
                                                     int32_t D, int32_t dtype) {
    return 0;
}

extern "C" int mesorasi_cross_attention(const void* q, int64_t q_bs, int64_t q_ld, int64_t q_hs, const void* k,
                                        int64_t k_bs, int64_t k_ld, int64_t k_hs, const void* v, int64_t v_bs,
                                        int64_t v_ld, int64_t v_hs, int32_t dtype, int64_t B, int64_t Nq, int64_t Nk,
                                        int32_t Hq, int32_t Hkv, int32_t D, float scale, const int32_t* k_len,
                                        const uint8_t* k_mask, int64_t mask_ld, void* o, int64_t o_bs, int64_t o_ld,
                                        int64_t o_hs, void* ws, size_t ws_bytes, void* stream) {
    MESO_REQUIRE(B >= 0 && Nq >= 0 && Nk >= 0, MESORASI_EINVAL, "mesorasi_cross_attention: negative size");
    MESO_REQUIRE(Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && D >= 1, MESORASI_EINVAL,
                 "mesorasi_cross_attention: Hq = %d, Hkv = %d, D = %d", Hq, Hkv, D);
    MESO_REQUIRE(q_bs >= 0 && q_ld >= 0 && q_hs >= 0 && k_bs >= 0 && k_ld >= 0 && k_hs >= 0 && v_bs >= 0 && v_ld >= 0 &&
                     v_hs >= 0,
                 MESORASI_EINVAL, "mesorasi_cross_attention: negative stride");
    MESO_REQUIRE((B <= 1 || o_bs >= D) && (Nq <= 1 || o_ld >= D) && (Hq <= 1 || o_hs >= D), MESORASI_EINVAL,
                 "mesorasi_cross_attention: an output stride < D");
    MESO_REQUIRE(!k_mask || B <= 1 || mask_ld >= Nk, MESORASI_EINVAL, "mesorasi_cross_attention: mask_ld < Nk");
    MESO_REQUIRE(std::isfinite(scale), MESORASI_EINVAL, "mesorasi_cross_attention: scale = %g", (double)scale);
    MESO_REQUIRE(dtype == MESORASI_F32 || dtype == MESORASI_BF16, MESORASI_EUNSUPPORTED,
                 "mesorasi_cross_attention: dtype %d", dtype);
    MESO_REQUIRE(D <= MESORASI_MAX_D_ATTN, MESORASI_EUNSUPPORTED, "mesorasi_cross_attention: D = %d", D);
    MESO_REQUIRE(Nk <= 0x7fffffff - 1023 && Nq <= (0x7fffffff - 1023) / (Hq / Hkv), MESORASI_EUNSUPPORTED,
                 "mesorasi_cross_attention: Nq = %lld, Nk = %lld", (long long)Nq, (long long)Nk);
    if (B == 0 || Nq == 0) return MESORASI_OK;
    MESO_REQUIRE(q && o && (Nk == 0 || (k && v)), MESORASI_EINVAL, "mesorasi_cross_attention: NULL q, k, v or o");
    AttnArgs a = {q, k, v, o, q_bs, q_ld, q_hs, k_bs, k_ld, k_hs, v_bs, v_ld, v_hs, o_bs, o_ld, o_hs,
                  Nq, Nk, mask_ld, Hq, Hkv, D, scale, k_len, k_mask};
    const int64_t total = B * Nq * Hq;
    MESO_REQUIRE(total <= 0x7fffffff, MESORASI_EUNSUPPORTED, "mesorasi_cross_attention: size");
    if (dtype == MESORASI_F32)
        attention_kernel<float><<<dim3((unsigned)total), dim3(64), 0, as_stream(stream)>>>(a, total);
    else
        attention_kernel<uint16_t><<<dim3((unsigned)total), dim3(64), 0, as_stream(stream)>>>(a, total);
    return after_launch("mesorasi_cross_attention");
}
