// Products in 8-bit integers with a scale for each row and output channel.
#include <algorithm>

#include "common.h"

namespace meso {

namespace {

constexpr int kQuThreads = 256;

template <typename T>
__device__ __forceinline__ float qu_load(const T* p) {
    if constexpr (sizeof(T) == 4)
        return *p;
    else
        return bf16_to_f32(*p);
}

// One wave per row: the largest magnitude, then the row in 8 bits.
template <typename T>
__global__ __launch_bounds__(kQuThreads) void quantize_i8_kernel(const T* __restrict__ x, int64_t ldx, int64_t rows,
                                                                 int C, int8_t* __restrict__ q, int64_t ldq,
                                                                 float* __restrict__ scale) {
    const int64_t r = blockIdx.x * (int64_t)(kQuThreads / 64) + (threadIdx.x >> 6);
    if (r >= rows) return;
    const int lane = threadIdx.x & 63;
    const T* xr = x + r * ldx;
    // magnitudes as bits: NaN above infinity above every finite value
    uint32_t m = 0;
    for (int c = lane; c < C; c += 64) m = max(m, __float_as_uint(qu_load(xr + c)) & 0x7fffffffu);
    for (int o = 32; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    const bool bad = m >= 0x7f800000u;
    const float a = fmaxf(__uint_as_float(m), 0x1p-100f);
    const float inv = 127.0f / a;
    if (lane == 0) scale[r] = bad ? __uint_as_float(0x7fc00000u) : a / 127.0f;
    const int Cp = (C + 15) & ~15;
    for (int c = lane; c < Cp; c += 64) q[r * ldq + c] = c < C && !bad ? (int8_t)(int)rintf(qu_load(xr + c) * inv) : 0;
}

template <typename TY>
__global__ __launch_bounds__(256) void linear_i8_kernel(const int8_t* __restrict__ x, int64_t ldx,
                                                        const float* __restrict__ xs, int64_t rows, int kp,
                                                        const int8_t* __restrict__ W, int64_t ldw,
                                                        const float* __restrict__ wsc, const float* __restrict__ bias,
                                                        int co, int relu, TY* __restrict__ y, int64_t ldy) {
    const int64_t e = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (e >= rows * co) return;
    const int64_t r = e / co;
    const int o = (int)(e - r * co);
    int acc = 0;
    for (int k = 0; k < kp; k += 4) {
        const char4 u = *reinterpret_cast<const char4*>(x + r * ldx + k);
        const char4 w = *reinterpret_cast<const char4*>(W + o * ldw + k);
        acc += u.x * w.x + u.y * w.y + u.z * w.z + u.w * w.w;
    }
    float v = ((float)acc * xs[r]) * wsc[o];
    if (bias) v += bias[o];
    if (relu) v = v < 0.0f ? 0.0f : v;
    if constexpr (sizeof(TY) == 4)
        y[r * ldy + o] = v;
    else
        y[r * ldy + o] = f32_to_bf16_any(v);
}

int64_t i8_pad(int64_t c) { return (c + 15) & ~(int64_t)15; }

}  // namespace

}  // namespace meso

using namespace meso;

extern "C" int mesorasi_quantize_i8(const void* x, int64_t ld_x, int32_t x_dtype, int64_t rows, int32_t C, int8_t* q,
                                    int64_t ld_q, float* scale, void* stream) {
    MESO_REQUIRE(rows >= 0, MESORASI_EINVAL, "mesorasi_quantize_i8: rows = %lld < 0", (long long)rows);
    MESO_REQUIRE(C >= 1 && ld_x >= C, MESORASI_EINVAL, "mesorasi_quantize_i8: C = %d, ld_x = %lld", C, (long long)ld_x);
    MESO_REQUIRE(ld_q >= C && ld_q % 16 == 0, MESORASI_EINVAL,
                 "mesorasi_quantize_i8: ld_q = %lld (at least C and a multiple of 16)", (long long)ld_q);
    MESO_REQUIRE(x_dtype == MESORASI_F32 || x_dtype == MESORASI_BF16, MESORASI_EUNSUPPORTED,
                 "mesorasi_quantize_i8: dtype %d", x_dtype);
    MESO_REQUIRE(C <= MESORASI_MAX_WIDTH_I8 && rows <= 0x7fffffff, MESORASI_EUNSUPPORTED,
                 "mesorasi_quantize_i8: C = %d, rows = %lld", C, (long long)rows);
    if (rows == 0) return MESORASI_OK;
    MESO_REQUIRE(x && q && scale, MESORASI_EINVAL, "mesorasi_quantize_i8: NULL pointer");
    MESO_REQUIRE(aligned(q, 16), MESORASI_EINVAL, "mesorasi_quantize_i8: q is not 16-byte aligned");
    const dim3 grid((unsigned)ceil_div(rows, kQuThreads / 64)), block(kQuThreads);
    if (x_dtype == MESORASI_F32)
        quantize_i8_kernel<float><<<grid, block, 0, as_stream(stream)>>>(static_cast<const float*>(x), ld_x, rows, C, q,
                                                                         ld_q, scale);
    else
        quantize_i8_kernel<uint16_t><<<grid, block, 0, as_stream(stream)>>>(static_cast<const uint16_t*>(x), ld_x, rows,
                                                                            C, q, ld_q, scale);
    return after_launch("mesorasi_quantize_i8");
}

extern "C" size_t mesorasi_linear_i8_workspace(int64_t rows, int32_t c_in, int32_t c_out, int32_t x_dtype) {
    if (rows < 1 || c_in < 1 || c_out < 1 || x_dtype == MESORASI_I8 || c_in > MESORASI_MAX_WIDTH_I8 ||
        c_out > MESORASI_MAX_WIDTH_I8 || rows > 0x7fffffff)
        return 0;
    return (size_t)(rows * i8_pad(c_in) + i8_pad(rows * 4));
}

extern "C" int mesorasi_linear_i8(const void* x, int64_t ld_x, int32_t x_dtype, const float* x_scale, int64_t rows,
                                  int32_t c_in, const int8_t* W, int64_t ld_w, const float* w_scale, const float* bias,
                                  int32_t c_out, int32_t relu, void* y, int64_t ld_y, int32_t y_dtype, void* ws,
                                  size_t ws_bytes, void* stream) {
    MESO_REQUIRE(rows >= 0, MESORASI_EINVAL, "mesorasi_linear_i8: rows = %lld < 0", (long long)rows);
    MESO_REQUIRE(c_in >= 1 && c_out >= 1, MESORASI_EINVAL, "mesorasi_linear_i8: c_in = %d, c_out = %d", c_in, c_out);
    MESO_REQUIRE(ld_x >= c_in && ld_w >= c_in && ld_y >= c_out, MESORASI_EINVAL,
                 "mesorasi_linear_i8: leading dimension < width");
    MESO_REQUIRE((x_dtype == MESORASI_F32 || x_dtype == MESORASI_BF16 || x_dtype == MESORASI_I8) &&
                     (y_dtype == MESORASI_F32 || y_dtype == MESORASI_BF16),
                 MESORASI_EUNSUPPORTED, "mesorasi_linear_i8: dtypes %d, %d", x_dtype, y_dtype);
    MESO_REQUIRE(ld_w % 16 == 0 && (x_dtype != MESORASI_I8 || ld_x % 16 == 0), MESORASI_EINVAL,
                 "mesorasi_linear_i8: an 8-bit leading dimension is no multiple of 16");
    MESO_REQUIRE(c_in <= MESORASI_MAX_WIDTH_I8 && c_out <= MESORASI_MAX_WIDTH_I8 && rows <= 0x7fffffff,
                 MESORASI_EUNSUPPORTED, "mesorasi_linear_i8: c_in = %d, c_out = %d, rows = %lld", c_in, c_out,
                 (long long)rows);
    if (rows == 0) return MESORASI_OK;
    MESO_REQUIRE(x && W && w_scale && y, MESORASI_EINVAL, "mesorasi_linear_i8: NULL pointer");
    MESO_REQUIRE((x_scale != nullptr) == (x_dtype == MESORASI_I8), MESORASI_EINVAL,
                 "mesorasi_linear_i8: x_scale goes with 8-bit rows, and only with them");
    MESO_REQUIRE(aligned(W, 16) && (x_dtype != MESORASI_I8 || aligned(x, 16)), MESORASI_EINVAL,
                 "mesorasi_linear_i8: 8-bit rows are not 16-byte aligned");
    const int8_t* q = static_cast<const int8_t*>(x);
    int64_t ldq = ld_x;
    const float* qs = x_scale;
    if (x_dtype != MESORASI_I8) {
        const size_t need = mesorasi_linear_i8_workspace(rows, c_in, c_out, x_dtype);
        MESO_REQUIRE(ws && ws_bytes >= need, MESORASI_EWORKSPACE, "mesorasi_linear_i8: workspace %zu < %zu bytes",
                     ws ? ws_bytes : (size_t)0, need);
        MESO_REQUIRE(aligned(ws, 16), MESORASI_EINVAL, "mesorasi_linear_i8: ws is not 16-byte aligned");
        ldq = i8_pad(c_in);
        int8_t* qw = static_cast<int8_t*>(ws);
        float* sw = reinterpret_cast<float*>(qw + rows * ldq);
        const int rc = mesorasi_quantize_i8(x, ld_x, x_dtype, rows, c_in, qw, ldq, sw, stream);
        if (rc != MESORASI_OK) return rc;
        q = qw;
        qs = sw;
    }
    const dim3 grid((unsigned)ceil_div(rows * c_out, 256)), block(256);
    if (y_dtype == MESORASI_F32)
        linear_i8_kernel<float><<<grid, block, 0, as_stream(stream)>>>(
            q, ldq, qs, rows, (int)i8_pad(c_in), W, ld_w, w_scale, bias, c_out, relu, static_cast<float*>(y), ld_y);
    else
        linear_i8_kernel<uint16_t><<<grid, block, 0, as_stream(stream)>>>(
            q, ldq, qs, rows, (int)i8_pad(c_in), W, ld_w, w_scale, bias, c_out, relu, static_cast<uint16_t*>(y), ld_y);
    return after_launch("mesorasi_linear_i8");
}
