// Rotary positions with several axes.
//
// Pair j of a head turns by t = pos[r, axis(j)] freq[j], the same for every
// head of row r.  A workgroup forms the angles of its rows once, in LDS:
// the product of two floats is exact in 64 bits, so is its reduction to quarters
// of a revolution and a remainder of at most an eighth to about |t| 2^-53, and
// only that remainder is rounded to fp32 before its sine and cosine -- a far
// coordinate costs no accuracy.
// Then every head's pairs are read, turned in fp32 and written, 16 bytes at
// a time where the layout allows it.
//
// Bound: one read and one write of x from HBM (65536 rows of 8 heads of 128 in
// bf16: 48 us, 5.6 TB/s; 64 in fp32: 46 us, 5.8 TB/s).
#include <algorithm>

#include "common.h"

namespace meso {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotAngles = 2048;     // angles of a workgroup (16 KB of LDS)

struct RotArgs {
    const void* x;
    void* y;
    const float* pos;
    const float* freq;
    int64_t ldx, ldy, ldp, rows;
    int H, D, P;
    int R;                           // rows of a workgroup, R * P <= kRotAngles
    int tpr;                         // threads of a row (a power of two)
    int n_axes;
    int end[MESORASI_MAX_AXES];      // first pair after each axis' section
    int copy;                        // the channels past the pairs have to be copied
};

// Sine and cosine of |x| <= pi / 4, from their power series: the terms left out
// are below x 2e-9 and 2e-10.
__device__ __forceinline__ void rot_sincos(float x, float& s, float& c) {
    const float z = x * x;
    const float p = fmaf(fmaf(fmaf(1.0f / 362880, z, -1.0f / 5040), z, 1.0f / 120), z, -1.0f / 6);
    const float q = fmaf(fmaf(fmaf(-1.0f / 3628800, z, 1.0f / 40320), z, -1.0f / 720), z, 1.0f / 24);
    s = fmaf(x * z, p, x);
    c = fmaf(z, fmaf(z, q, -0.5f), 1.0f);
}

__device__ __forceinline__ float rot_load(const float* p) { return *p; }
__device__ __forceinline__ float rot_load(const uint16_t* p) { return bf16_to_f32(*p); }

template <typename T, int N>
struct alignas(sizeof(T) * N) RotVec {
    T e[N];
};

template <typename T, int N>
__device__ __forceinline__ void rot_read(const T* p, float (&f)[N]) {
    const RotVec<T, N> v = *reinterpret_cast<const RotVec<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = rot_load(&v.e[i]);
}

template <typename T, int N>
__device__ __forceinline__ void rot_write(T* p, const float (&f)[N]) {
    RotVec<T, N> v;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (sizeof(T) == 4)
            v.e[i] = f[i];
        else
            v.e[i] = f32_to_bf16_any(f[i]);
    }
    *reinterpret_cast<RotVec<T, N>*>(p) = v;
}

// VEC pairs at a time: two vectors of VEC channels P apart, or one of 2 VEC
// adjacent channels.
template <typename T, int VEC, bool INTERLEAVED>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotArgs a) {
    __shared__ float2 ang[kRotAngles];
    const int tid = threadIdx.x;
    const int64_t r0 = (int64_t)blockIdx.x * a.R;
    const int nr = (int)min((int64_t)a.R, a.rows - r0);
    for (int i = tid; i < nr * a.P; i += kRotThreads) {
        const int r = i / a.P, j = i - r * a.P;
        int ax = 0;
#pragma unroll
        for (int k = 0; k < MESORASI_MAX_AXES - 1; ++k) ax += j >= a.end[k];
        const double rev = (double)a.pos[(r0 + r) * a.ldp + ax] * (double)a.freq[j] * 0.15915494309189533577;
        const double quarters = rint(4.0 * rev);
        const int q = (int)(quarters - 4.0 * rint(0.25 * quarters)) & 3;
        float s, c;
        rot_sincos((float)((rev - 0.25 * quarters) * 6.28318530717958647693), s, c);
        const float x = q & 1 ? s : c, y = q & 1 ? c : s;        // turned by q quarters
        ang[i] = make_float2(q == 1 || q == 2 ? -x : x, q >= 2 ? -y : y);
    }
    __syncthreads();
    const int nv = a.P / VEC;                                       // vectors of pairs of a head
    const int ih = nv + (a.copy ? (a.D - 2 * a.P) / VEC : 0);       // and of copied channels
    const int lane = tid & (a.tpr - 1);
    const int h0 = lane / ih, v0 = lane - h0 * ih;
    const int dh = a.tpr / ih, dv = a.tpr - dh * ih;
    for (int r = tid / a.tpr; r < nr; r += kRotThreads / a.tpr) {
        const T* __restrict__ xr = static_cast<const T*>(a.x) + (r0 + r) * a.ldx;
        T* yr = static_cast<T*>(a.y) + (r0 + r) * a.ldy;
        const float2* __restrict__ ar = ang + r * a.P;
        int h = h0, v = v0;
        while (h < a.H) {
            const int64_t base = (int64_t)h * a.D;
            if (v >= nv) {
                const int64_t o = base + 2 * a.P + (v - nv) * VEC;
                *reinterpret_cast<RotVec<T, VEC>*>(yr + o) = *reinterpret_cast<const RotVec<T, VEC>*>(xr + o);
            } else if constexpr (INTERLEAVED) {
                float z[2 * VEC];
                const int64_t o = base + 2 * VEC * v;
                if constexpr (VEC == 1) {     // rows of any alignment
                    z[0] = rot_load(xr + o);
                    z[1] = rot_load(xr + o + 1);
                } else {
                    rot_read<T, 2 * VEC>(xr + o, z);
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float2 cs = ar[v * VEC + i];
                    const float u = z[2 * i], w = z[2 * i + 1];
                    z[2 * i] = u * cs.x - w * cs.y;
                    z[2 * i + 1] = u * cs.y + w * cs.x;
                }
                if constexpr (VEC == 1) {
                    rot_write<T, 1>(yr + o, {z[0]});
                    rot_write<T, 1>(yr + o + 1, {z[1]});
                } else {
                    rot_write<T, 2 * VEC>(yr + o, z);
                }
            } else {
                float u[VEC], w[VEC];
                const int64_t o = base + VEC * v;
                rot_read<T, VEC>(xr + o, u);
                rot_read<T, VEC>(xr + o + a.P, w);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float2 cs = ar[v * VEC + i];
                    const float t = u[i];
                    u[i] = t * cs.x - w[i] * cs.y;
                    w[i] = t * cs.y + w[i] * cs.x;
                }
                rot_write<T, VEC>(yr + o, u);
                rot_write<T, VEC>(yr + o + a.P, w);
            }
            h += dh;
            v += dv;
            if (v >= ih) {
                v -= ih;
                ++h;
            }
        }
    }
}

template <typename T, int VEC>
void launch_rotary(const RotArgs& a, bool interleaved, unsigned grid, hipStream_t s) {
    if (interleaved)
        rotary_kernel<T, VEC, true><<<dim3(grid), dim3(kRotThreads), 0, s>>>(a);
    else
        rotary_kernel<T, VEC, false><<<dim3(grid), dim3(kRotThreads), 0, s>>>(a);
}

}  // namespace

}  // namespace meso

using namespace meso;

extern "C" int mesorasi_rotary(const void* x, int64_t ld_x, int32_t dtype, int64_t rows, int32_t H, int32_t D,
                               const float* pos, int64_t ld_pos, int32_t n_axes, const int32_t* sections,
                               const float* freq, int32_t interleaved, void* y, int64_t ld_y, void* stream) {
    MESO_REQUIRE(rows >= 0, MESORASI_EINVAL, "mesorasi_rotary: rows = %lld < 0", (long long)rows);
    MESO_REQUIRE(H >= 1 && D >= 1, MESORASI_EINVAL, "mesorasi_rotary: H = %d, D = %d", H, D);
    MESO_REQUIRE(n_axes >= 1 && n_axes <= MESORASI_MAX_AXES, MESORASI_EUNSUPPORTED, "mesorasi_rotary: %d axes", n_axes);
    MESO_REQUIRE(sections, MESORASI_EINVAL, "mesorasi_rotary: NULL sections");
    MESO_REQUIRE(dtype == MESORASI_F32 || dtype == MESORASI_BF16, MESORASI_EUNSUPPORTED, "mesorasi_rotary: dtype %d",
                 dtype);
    MESO_REQUIRE(D <= MESORASI_MAX_D_ROTARY && H <= 65536 && rows <= 0x7fffffff, MESORASI_EUNSUPPORTED,
                 "mesorasi_rotary: H = %d, D = %d, rows = %lld", H, D, (long long)rows);
    RotArgs a;
    int64_t P = 0;
    for (int i = 0; i < MESORASI_MAX_AXES; ++i) {
        if (i < n_axes) {
            MESO_REQUIRE(sections[i] >= 0, MESORASI_EINVAL, "mesorasi_rotary: sections[%d] = %d", i, sections[i]);
            P += sections[i];
        }
        a.end[i] = i < n_axes - 1 ? (int)std::min<int64_t>(P, D) : 0x7fffffff;
    }
    MESO_REQUIRE(P >= 1 && 2 * P <= D, MESORASI_EINVAL, "mesorasi_rotary: %lld pairs in a head of %d channels",
                 (long long)P, D);
    const int64_t width = (int64_t)H * D;
    MESO_REQUIRE(ld_x >= width && ld_y >= width && ld_pos >= n_axes, MESORASI_EINVAL,
                 "mesorasi_rotary: leading dimension < width");
    MESO_REQUIRE(x != y || ld_x == ld_y || rows == 0, MESORASI_EINVAL,
                 "mesorasi_rotary: y == x with another leading dimension");
    if (rows == 0) return MESORASI_OK;
    MESO_REQUIRE(x && y && pos && freq, MESORASI_EINVAL, "mesorasi_rotary: NULL pointer");
    const int elem = dtype == MESORASI_F32 ? 4 : 2;
    a.x = x; a.y = y; a.pos = pos; a.freq = freq;
    a.ldx = ld_x; a.ldy = ld_y; a.ldp = ld_pos; a.rows = rows;
    a.H = H; a.D = D; a.P = (int)P; a.n_axes = n_axes;
    a.copy = x != y && 2 * P < D;
    // the widest vector that divides every run of channels and is aligned
    int vec = 16 / elem;
    while (vec > 1 && !(P % vec == 0 && D % vec == 0 && ld_x % vec == 0 && ld_y % vec == 0 &&
                        aligned(x, vec * elem) && aligned(y, vec * elem)))
        vec /= 2;
    // an interleaved vector of pairs is twice as long
    const bool inter = interleaved != 0;
    if (inter && vec > 1) vec /= 2;
    // rows of a workgroup: as many as its angles hold, fewer while that leaves compute units without work
    const int ih = (int)(P / vec) + (a.copy ? (int)((D - 2 * P) / vec) : 0);
    int R = (int)std::max<int64_t>(1, std::min<int64_t>(kRotAngles / P, 64));
    while (R > 1 && ceil_div(rows, R) < 2048) R /= 2;
    int tpr = 1;
    while (tpr < kRotThreads && tpr < (int64_t)H * ih) tpr *= 2;
    a.R = R;
    a.tpr = tpr;
    MESO_REQUIRE(launch_fits(ceil_div(rows, R), kRotThreads), MESORASI_EUNSUPPORTED, "mesorasi_rotary: %lld rows of %lld pairs",
                 (long long)rows, (long long)P);
    const Extent ext = rows_extent(y, rows, ld_y, width, elem);
    MESO_REQUIRE((x == y || !overlap(ext, rows_extent(x, rows, ld_x, width, elem))) &&
                     !overlap(ext, rows_extent(pos, rows, ld_pos, n_axes, 4)) && !overlap(ext, rows_extent(freq, 1, P, P, 4)),
                 MESORASI_EINVAL, "mesorasi_rotary: y overlaps an input");
    const unsigned grid = (unsigned)ceil_div(rows, R);
    hipStream_t s = as_stream(stream);
    if (dtype == MESORASI_F32) {
        switch (vec) {
            case 4: launch_rotary<float, 4>(a, inter, grid, s); break;
            case 2: launch_rotary<float, 2>(a, inter, grid, s); break;
            default: launch_rotary<float, 1>(a, inter, grid, s); break;
        }
    } else {
        switch (vec) {
            case 8: launch_rotary<uint16_t, 8>(a, inter, grid, s); break;
            case 4: launch_rotary<uint16_t, 4>(a, inter, grid, s); break;
            case 2: launch_rotary<uint16_t, 2>(a, inter, grid, s); break;
            default: launch_rotary<uint16_t, 1>(a, inter, grid, s); break;
        }
    }
    return after_launch("mesorasi_rotary");
}
