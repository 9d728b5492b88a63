// Products in 8-bit integers with a scale for each row and output channel:
// y = (float(sum_c q_c w_c) s_row) s_channel + b, the sum exact in 32 bits.
//
// Float rows are first brought to 8 bits (quantize_i8_kernel), or, where at
// most 16 rows of at most 2048 columns come, in the product's registers.
//
// Measured.  The large product (16384 x 4096 -> 4096, 8-bit rows): 270 us, 2040
// TOP/s, where the library's int8 product without scales takes 247 us, 2220;
// at 8192 x 8192 -> 8192 2270 against 2470.  The matrix cores are busy 50 % of
// it and L2 serves 2.1 GB of tiles at 8 TB/s, so neither alone bounds it; what
// takes the rest was not isolated.  16368 x 320 -> 256 from fp32: 16 us for the
// 7 of its bytes, two launches and the 8-bit rows' round trip.  Few rows: the
// latency of one chain of loads (13 x 1024 -> 512: 3.0 us from 8-bit rows, 6.0
// from fp32).
#include <algorithm>

#include "common.h"

namespace meso {

namespace {

typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) const char* lds_cptr;

// ---------------------------------------------------------------------------
// rows to 8 bits
// ---------------------------------------------------------------------------

constexpr int kQuThreads = 256;
constexpr int kQuKeep = 8;           // vectors of a row that a lane keeps between the two passes

template <typename T, int N>
struct alignas(sizeof(T) * N) QuVec {
    T e[N];
};

// The same at any element: the hardware's loads and stores need no more.
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) QuLoose {
    T e[N];
};

__device__ __forceinline__ float qu_float(float v) { return v; }
__device__ __forceinline__ float qu_float(uint16_t v) { return bf16_to_f32(v); }

struct QuScale {
    float scale, inv;
    bool bad;
};

// m: the row's largest magnitude as bits (NaN above infinity above every
// finite value).
__device__ __forceinline__ QuScale qu_scale(uint32_t m) {
    const float a = fmaxf(__uint_as_float(m), 0x1p-100f);
    QuScale s;
    s.bad = m >= 0x7f800000u;
    s.scale = s.bad ? __uint_as_float(0x7fc00000u) : a / 127.0f;
    s.inv = s.bad ? 0.0f : 127.0f / a;
    return s;
}

// rint(fl(v inv)) in the low byte: adding 1.5 2^23 rounds to a whole number,
// ties to even.
__device__ __forceinline__ uint32_t qu_byte(float v, float inv) {
    return __float_as_uint(v * inv + 12582912.0f) & 0xffu;
}

template <int N>
__device__ __forceinline__ void qu_store(int8_t* q, const float (&f)[N], const QuScale& s) {
    QuVec<uint32_t, N / 4> w;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        uint32_t u = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) u |= qu_byte(f[4 * i + k], s.inv) << (8 * k);
        w.e[i] = s.bad ? 0u : u;
    }
    *reinterpret_cast<QuVec<uint32_t, N / 4>*>(q) = w;
}

// LPR lanes per row, 16 bytes of a row (of any alignment) at a time; the first
// kQuKeep vectors of a lane stay in registers between the maximum and the
// rounding, longer rows are read again.  Bound: one read of x and one write
// of q (16384 x 4096 bf16: 45 us, 4.5 TB/s
// between products; 32 us repeated on the same rows, which the caches then hold in part).
template <typename T, int LPR>
__global__ __launch_bounds__(kQuThreads) void quantize_i8_kernel(const T* __restrict__ x, int64_t ldx, int64_t rows,
                                                                 int C, int8_t* __restrict__ q, int64_t ldq,
                                                                 float* __restrict__ scale) {
    constexpr int VEC = 16 / sizeof(T);
    const int64_t r = blockIdx.x * (int64_t)(kQuThreads / LPR) + threadIdx.x / LPR;
    const int lane = threadIdx.x % LPR;
    if (r >= rows) return;
    const T* xr = x + r * ldx;
    const int pad = (C + 15) & ~15, nv = pad / VEC;          // the last vectors may end in padding
    float keep[kQuKeep][VEC];
    uint32_t m = 0;
    auto read = [&](int v, float (&f)[VEC]) {
        const int c = v * VEC;
        if (c + VEC <= C) {
            const QuLoose<T, VEC> w = *reinterpret_cast<const QuLoose<T, VEC>*>(xr + c);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = qu_float(w.e[i]);
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = c + i < C ? qu_float(xr[c + i]) : 0.0f;
        }
    };
#pragma unroll
    for (int i = 0; i < kQuKeep; ++i) {
        const int v = i * LPR + lane;
        if (v < nv) {
            read(v, keep[i]);
#pragma unroll
            for (int k = 0; k < VEC; ++k) m = max(m, __float_as_uint(keep[i][k]) & 0x7fffffffu);
        }
    }
    for (int v = kQuKeep * LPR + lane; v < nv; v += LPR) {
        float f[VEC];
        read(v, f);
#pragma unroll
        for (int k = 0; k < VEC; ++k) m = max(m, __float_as_uint(f[k]) & 0x7fffffffu);
    }
#pragma unroll
    for (int o = LPR / 2; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    const QuScale s = qu_scale(m);
    if (lane == 0) scale[r] = s.scale;
    int8_t* qr = q + r * ldq;
#pragma unroll
    for (int i = 0; i < kQuKeep; ++i) {
        const int v = i * LPR + lane;
        if (v < nv) qu_store<VEC>(qr + v * VEC, keep[i], s);
    }
    for (int v = kQuKeep * LPR + lane; v < nv; v += LPR) {
        float f[VEC];
        read(v, f);
        qu_store<VEC>(qr + v * VEC, f, s);
    }
}

// Lanes of a row: as few as keep it in registers, so that short rows share a wave.
int quantize_lanes(int C, int dtype) {
    const int nv = ((C + 15) & ~15) / (dtype == MESORASI_F32 ? 4 : 8);
    return nv <= 4 * kQuKeep ? 4 : nv <= 16 * kQuKeep ? 16 : 64;
}

bool quantize_fits(int64_t rows, int C, int dtype) {
    return launch_fits(ceil_div(rows, kQuThreads / quantize_lanes(C, dtype)), kQuThreads);
}

template <typename T>
void run_quantize(const T* x, int64_t ldx, int64_t rows, int C, int8_t* q, int64_t ldq, float* scale, hipStream_t s) {
    const int lpr = quantize_lanes(C, sizeof(T) == 4 ? MESORASI_F32 : MESORASI_BF16);
    const dim3 grid((unsigned)ceil_div(rows, kQuThreads / lpr)), block(kQuThreads);
    switch (lpr) {
        case 4: quantize_i8_kernel<T, 4><<<grid, block, 0, s>>>(x, ldx, rows, C, q, ldq, scale); break;
        case 16: quantize_i8_kernel<T, 16><<<grid, block, 0, s>>>(x, ldx, rows, C, q, ldq, scale); break;
        default: quantize_i8_kernel<T, 64><<<grid, block, 0, s>>>(x, ldx, rows, C, q, ldq, scale); break;
    }
}

void run_quantize(const void* x, int64_t ldx, int dtype, int64_t rows, int C, int8_t* q, int64_t ldq, float* scale,
                  hipStream_t s) {
    if (dtype == MESORASI_F32)
        run_quantize(static_cast<const float*>(x), ldx, rows, C, q, ldq, scale, s);
    else
        run_quantize(static_cast<const uint16_t*>(x), ldx, rows, C, q, ldq, scale, s);
}

// ---------------------------------------------------------------------------
// the product
// ---------------------------------------------------------------------------

struct LinArgs {
    const int8_t* x;
    const float* xs;
    const int8_t* w;
    const float* wsc;
    const float* bias;
    void* y;
    int64_t ldx, ldw, ldy, rows;
    int kp, co, relu;                // kp: columns, a multiple of 16
    int tiles_r, tiles_c;
    int64_t blocks;
    int per_xcd;
};

__device__ const uint4 kLinZero[1] = {};

constexpr int kLinK = 128;           // bytes of a row in a tile: eight 16-byte chunks

// Slot of a chunk in its row: 16 rows at one chunk lie in different banks.
__device__ __forceinline__ int lin_swz(int row) { return (row >> 1) & 7; }

__device__ __forceinline__ void lin_load_lds(const void* g, uint32_t lds_base) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)(uintptr_t)g,
                                     (__attribute__((address_space(3))) uint32_t*)(uintptr_t)lds_base, 16, 0, 0);
}

// Four channels of a row: scaled, biased (a missing bias is 0: adding it
// turns a -0 into 0 and changes nothing else), clamped and written.
template <typename TY>
__device__ __forceinline__ void lin_out(const LinArgs& a, int64_t row, int ch, i32x4 acc, float xs,
                                        const float (&ws)[4], const float (&bs)[4]) {
    TY* y = static_cast<TY*>(a.y) + row * a.ldy + ch;
    QuLoose<TY, 4> v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float f = ((float)acc[i] * xs) * ws[i] + bs[i];
        if (a.relu) f = f < 0.0f ? 0.0f : f;
        if constexpr (sizeof(TY) == 4)
            v.e[i] = f;
        else
            v.e[i] = f32_to_bf16_any(f);
    }
    if (ch + 3 < a.co) {
        *reinterpret_cast<QuLoose<TY, 4>*>(y) = v;
        asm volatile("");            // keeps this one store apart from those below
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (ch + i < a.co) y[i] = v.e[i];
}

// Y^T = W X^T on v_mfma_i32_32x32x32_i8: a lane's accumulators of a 32 x 32
// block are four runs of 4 channels of its own row, which it scales and
// writes.  Both operands are 16-byte pieces of rows as they lie, from tiles
// of 128 columns that are loaded ahead, two in LDS, and a step's operands are
// read between the products of the step before (when that came in: 468 to
// 282 us for 16384 x 4096 -> 4096).  WC x WR waves, each of BC x BR blocks
// (channels x rows).
template <typename TY, int WC, int WR, int BC, int BR>
__global__ __launch_bounds__(64 * WC * WR, (WC * WR >= 8 ? 2 : 1)) void linear_i8_kernel(LinArgs a) {
    constexpr int kThreads = 64 * WC * WR;
    constexpr int TC = 32 * WC * BC, TR = 32 * WR * BR;
    constexpr int kTile = (TC + TR) * kLinK;
    constexpr int kLoads = kTile / 16 / kThreads;
    static_assert(TC * 8 % kThreads == 0 && TR * 8 % kThreads == 0, "whole loads of either operand");
    extern __shared__ __align__(16) char lds[];
    const int64_t lb = (int64_t)(blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3);
    if (lb >= a.blocks) return;
    // groups of 8 row tiles over all channel tiles: what runs together shares rows and weights in L2
    const int64_t group = lb / (8 * a.tiles_c);
    const int in = (int)(lb - group * 8 * a.tiles_c);
    const int gr = (int)min((int64_t)8, a.tiles_r - group * 8);
    const int64_t row0 = (group * 8 + in % gr) * TR;
    const int ch0 = in / gr * TC;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int half = lane >> 5, col = lane & 31;
    const int wc = wave % WC, wr = wave / WC;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_cptr)lds;

    // chunk p of the tile: row p / 8 (channels, then rows), slot p % 8
    const int8_t* src[kLoads];
    bool in_range[kLoads];
    int chunk[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int p = i * kThreads + tid, r = p >> 3;
        chunk[i] = ((p & 7) ^ lin_swz(r)) * 16;
        if (i * kThreads < TC * 8) {
            in_range[i] = ch0 + r < a.co;
            src[i] = a.w + (int64_t)(ch0 + r) * a.ldw + chunk[i];
        } else {
            const int64_t xr = row0 + (r - TC);
            in_range[i] = xr < a.rows;
            src[i] = a.x + xr * a.ldx + chunk[i];
        }
    }
    auto stage = [&](int t) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const bool ok = in_range[i] && chunk[i] + t * kLinK < a.kp;
            const void* g = ok ? (const void*)(src[i] + (int64_t)t * kLinK) : (const void*)kLinZero;
            lin_load_lds(g, __builtin_amdgcn_readfirstlane(lds0 + (t & 1) * kTile + (i * kThreads + wave * 64) * 16));
        }
    };

    i32x16 acc[BC][BR];
#pragma unroll
    for (int i = 0; i < BC; ++i)
#pragma unroll
        for (int j = 0; j < BR; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
    const int swz = lin_swz(col);
    const int tiles = (a.kp + kLinK - 1) / kLinK;
    stage(0);
    for (int t = 0; t < tiles; ++t) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (t + 1 < tiles) stage(t + 1);
        const char* tw = lds + (t & 1) * kTile + (wc * BC * 32 + col) * kLinK;
        const char* tx = lds + (t & 1) * kTile + (TC + wr * BR * 32 + col) * kLinK;
        // a step's operands are read between the products of the step before
        i32x4 wf[2][BC], xf[2][BR];
        auto read = [&](int s) {
            const int at = ((2 * s + half) ^ swz) << 4;
#pragma unroll
            for (int j = 0; j < BR; ++j) xf[s & 1][j] = *reinterpret_cast<const i32x4*>(tx + j * 32 * kLinK + at);
#pragma unroll
            for (int i = 0; i < BC; ++i) wf[s & 1][i] = *reinterpret_cast<const i32x4*>(tw + i * 32 * kLinK + at);
        };
        read(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < kLinK / 32; ++s) {
            if (s + 1 < kLinK / 32) read(s + 1);
#pragma unroll
            for (int i = 0; i < BC; ++i)
#pragma unroll
                for (int j = 0; j < BR; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[s & 1][i], xf[s & 1][j], acc[i][j], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < BC + BR; ++i) {      // a product, a read, ...
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            if constexpr (BC * BR > BC + BR) __builtin_amdgcn_sched_group_barrier(0x008, BC * BR - BC - BR, 0);
        }
    }
    // A block goes through LDS, so that lanes hold runs of a row's channels:
    // 8 of them write 128 bytes of it.
    __syncthreads();
    constexpr int kPitch = 36;
    int* sh = reinterpret_cast<int*>(lds) + wave * 32 * kPitch;
    const int er = lane >> 3, ec = 4 * (lane & 7);
#pragma unroll
    for (int i = 0; i < BC; ++i) {
        const int ch = ch0 + (wc * BC + i) * 32 + ec;
        float ws[4], bs[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            ws[e] = ch + e < a.co ? a.wsc[ch + e] : 0.0f;
            bs[e] = a.bias && ch + e < a.co ? a.bias[ch + e] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < BR; ++j) {
            const int64_t rb = row0 + (wr * BR + j) * 32;
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<i32x4*>(sh + col * kPitch + 2 * r + 4 * half) =
                    i32x4{acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]};
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const i32x4 v = *reinterpret_cast<const i32x4*>(sh + (8 * k + er) * kPitch + ec);
                const int64_t row = rb + 8 * k + er;
                if (row < a.rows && ch < a.co) lin_out<TY>(a, row, ch, v, a.xs[row], ws, bs);
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
}

template <typename TY, int WC, int WR, int BC, int BR>
int launch_linear(LinArgs& a, hipStream_t s) {
    constexpr int TC = 32 * WC * BC, TR = 32 * WR * BR, bytes = 2 * (TC + TR) * kLinK;
    static const hipError_t attr =
        hipFuncSetAttribute(reinterpret_cast<const void*>(&linear_i8_kernel<TY, WC, WR, BC, BR>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    MESO_REQUIRE(attr == hipSuccess, MESORASI_EHIP, "mesorasi_linear_i8: LDS size attribute: %s",
                 hipGetErrorString(attr));
    a.tiles_r = (int)ceil_div(a.rows, TR);
    a.tiles_c = (int)ceil_div(a.co, TC);
    a.blocks = (int64_t)a.tiles_r * a.tiles_c;
    const int64_t per = ceil_div(a.blocks, 8);
    a.per_xcd = (int)per;
    linear_i8_kernel<TY, WC, WR, BC, BR><<<dim3((unsigned)(8 * per)), dim3(64 * WC * WR), bytes, s>>>(a);
    return MESORASI_OK;
}

// Few rows: a workgroup takes 16 channels and all (at most 16 RB) rows, its
// eight waves share the columns, and the weights go from memory straight to
// the operands of v_mfma_i32_16x16x64_i8 (lane: channel or row lane % 16,
// columns 16 (lane / 16) + 0..15 of 64).  TX float or bf16 (RB = 1): every
// workgroup brings the rows to 8 bits in registers, where their columns'
// operands are; each reads all of x, which its caches hold.
// Bound: one read of W, and the latency of one chain of loads.
constexpr int kFewThreads = 512;
constexpr int kFewSteps = 4;         // steps of 64 columns that a wave holds in registers
constexpr int kFewMaxK = 64 * 8 * kFewSteps;

template <typename TX, typename TY, int RB>
__global__ __launch_bounds__(kFewThreads) void linear_i8_few_kernel(LinArgs a, const TX* __restrict__ xf, int ci) {
    constexpr int kWaves = kFewThreads / 64;
    __shared__ i32x4 part[kWaves][RB][64];
    __shared__ uint32_t top[kWaves][16];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int r16 = lane & 15, grp = lane >> 4;
    const int ch = blockIdx.x * 16 + r16;
    const int steps = (a.kp + 63) / 64, per = (steps + kWaves - 1) / kWaves;
    const int s0 = wave * per, s1 = min(steps, s0 + per);
    const int8_t* wp = a.w + (int64_t)min(ch, a.co - 1) * a.ldw + 16 * grp;
    const i32x4 zero = {0, 0, 0, 0};
    i32x4 acc[RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) acc[j] = zero;
    float scale = 0.0f;
    if constexpr (sizeof(TX) == 1) {
        const int8_t* xp[RB];
#pragma unroll
        for (int j = 0; j < RB; ++j) xp[j] = a.x + min((int64_t)(16 * j + r16), a.rows - 1) * a.ldx + 16 * grp;
        for (int s = s0; s < s1; s += kFewSteps) {
            i32x4 wf[kFewSteps], xq[kFewSteps][RB];
#pragma unroll
            for (int i = 0; i < kFewSteps; ++i) {
                const bool in = s + i < s1 && 64 * (s + i) + 16 * grp < a.kp;
                wf[i] = in ? *reinterpret_cast<const i32x4*>(wp + 64 * (s + i)) : zero;
#pragma unroll
                for (int j = 0; j < RB; ++j)
                    xq[i][j] = in ? *reinterpret_cast<const i32x4*>(xp[j] + 64 * (s + i)) : zero;
            }
#pragma unroll
            for (int i = 0; i < kFewSteps; ++i)
#pragma unroll
                for (int j = 0; j < RB; ++j)
                    acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[i], xq[i][j], acc[j], 0, 0, 0);
        }
    } else {
        i32x4 wf[kFewSteps];
        float v[kFewSteps][16];
        const TX* xp = xf + (int64_t)r16 * a.ldx + 16 * grp;
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kFewSteps; ++i) {
            const int k0 = 64 * (s0 + i) + 16 * grp;
            const bool in = s0 + i < s1 && k0 < a.kp;
            wf[i] = in ? *reinterpret_cast<const i32x4*>(wp + 64 * (s0 + i)) : zero;
            constexpr int V = 16 / sizeof(TX);
            const bool row = in && r16 < a.rows;
            if (row && k0 + 16 <= ci) {
#pragma unroll
                for (int e = 0; e < 16; e += V) {
                    const QuLoose<TX, V> w = *reinterpret_cast<const QuLoose<TX, V>*>(xp + 64 * (s0 + i) + e);
#pragma unroll
                    for (int k = 0; k < V; ++k) v[i][e + k] = qu_float(w.e[k]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) v[i][e] = row && k0 + e < ci ? qu_float(xp[64 * (s0 + i) + e]) : 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < kFewSteps; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) m = max(m, __float_as_uint(v[i][e]) & 0x7fffffffu);
        m = max(m, (uint32_t)__shfl_xor((int)m, 16));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32));
        if (grp == 0) top[wave][r16] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = max(m, top[w][r16]);
        const QuScale q = qu_scale(m);
        scale = q.scale;
#pragma unroll
        for (int i = 0; i < kFewSteps; ++i) {
            i32x4 xq;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t u = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) u |= qu_byte(v[i][4 * w + k], q.inv) << (8 * k);
                xq[w] = q.bad ? 0 : (int)u;
            }
            acc[0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[i], xq, acc[0], 0, 0, 0);
        }
    }
    // lane: channels 4 grp + 0..3 of row lane % 16
#pragma unroll
    for (int j = 0; j < RB; ++j) part[wave][j][lane] = acc[j];
    __syncthreads();
    if (wave >= RB) return;
    i32x4 t = part[0][wave][lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) t += part[w][wave][lane];
    const int64_t row = 16 * wave + r16;
    const int c4 = blockIdx.x * 16 + 4 * grp;
    if (row >= a.rows || c4 >= a.co) return;
    if constexpr (sizeof(TX) == 1) scale = a.xs[row];
    float ws[4], bs[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        ws[e] = c4 + e < a.co ? a.wsc[c4 + e] : 0.0f;
        bs[e] = a.bias && c4 + e < a.co ? a.bias[c4 + e] : 0.0f;
    }
    lin_out<TY>(a, row, c4, t, scale, ws, bs);
}

template <typename TY>
int run_linear(LinArgs& a, hipStream_t s) {
    if (a.rows <= 64) {
        const dim3 grid((unsigned)ceil_div(a.co, 16)), block(kFewThreads);
        if (a.rows <= 16)
            linear_i8_few_kernel<int8_t, TY, 1><<<grid, block, 0, s>>>(a, nullptr, 0);
        else if (a.rows <= 32)
            linear_i8_few_kernel<int8_t, TY, 2><<<grid, block, 0, s>>>(a, nullptr, 0);
        else
            linear_i8_few_kernel<int8_t, TY, 4><<<grid, block, 0, s>>>(a, nullptr, 0);
        return MESORASI_OK;
    }
    // 256 x 256 tiles for long products whose tiles fill at least three quarters of the compute units' turns, else the
    // largest tile that gives most compute units one: 16384 x 1024 -> 1024 takes 32.5 us in the first and 34.6 in the
    // second, 16384 x 320 -> 256 9.2 in the second and 8.6 in the third, 65536 x 128 -> 128 17.0, 11.9 and 11.9,
    // 4096 x 1024 -> 1024 27.5, 11.3 and 12.3
    const int64_t t = ceil_div(a.rows, 256) * ceil_div(a.co, 256);
    if (a.kp >= 1024 && 4 * t >= 3 * 256 * ceil_div(t, 256)) return launch_linear<TY, 2, 4, 4, 2>(a, s);
    if (ceil_div(a.rows, 128) * ceil_div(a.co, 128) >= 192) return launch_linear<TY, 2, 4, 2, 1>(a, s);
    return launch_linear<TY, 2, 2, 1, 1>(a, s);
}

// Few rows that are brought to 8 bits where they are multiplied.
bool linear_few_fused(int64_t rows, int64_t kp, int x_dtype) {
    return x_dtype != MESORASI_I8 && rows <= 16 && kp <= kFewMaxK;
}

template <typename TX, typename TY>
void run_linear_few_fused(const LinArgs& a, const TX* x, int ci, hipStream_t s) {
    linear_i8_few_kernel<TX, TY, 1><<<dim3((unsigned)ceil_div(a.co, 16)), dim3(kFewThreads), 0, s>>>(a, x, ci);
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
    MESO_REQUIRE(C <= MESORASI_MAX_WIDTH_I8 && rows <= 0x7fffffff && quantize_fits(rows, C, x_dtype),
                 MESORASI_EUNSUPPORTED, "mesorasi_quantize_i8: C = %d, rows = %lld", C, (long long)rows);
    if (rows == 0) return MESORASI_OK;
    MESO_REQUIRE(x && q && scale, MESORASI_EINVAL, "mesorasi_quantize_i8: NULL pointer");
    MESO_REQUIRE(aligned(q, 16), MESORASI_EINVAL, "mesorasi_quantize_i8: q is not 16-byte aligned");
    const Extent ext = rows_extent(x, rows, ld_x, C, x_dtype == MESORASI_F32 ? 4 : 2);
    MESO_REQUIRE(!overlap(ext, rows_extent(q, rows, ld_q, i8_pad(C), 1)) && !overlap(ext, rows_extent(scale, rows, 1, 1, 4)),
                 MESORASI_EINVAL, "mesorasi_quantize_i8: q or scale overlaps x");
    run_quantize(x, ld_x, x_dtype, rows, C, q, ld_q, scale, as_stream(stream));
    return after_launch("mesorasi_quantize_i8");
}

extern "C" size_t mesorasi_linear_i8_workspace(int64_t rows, int32_t c_in, int32_t c_out, int32_t x_dtype) {
    if (rows < 1 || c_in < 1 || c_out < 1 || x_dtype == MESORASI_I8 || c_in > MESORASI_MAX_WIDTH_I8 ||
        c_out > MESORASI_MAX_WIDTH_I8 || rows > 0x7fffffff || linear_few_fused(rows, i8_pad(c_in), x_dtype))
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
    // tiles of 128 x 128 in the most workgroups that many rows and channels get
    MESO_REQUIRE(c_in <= MESORASI_MAX_WIDTH_I8 && c_out <= MESORASI_MAX_WIDTH_I8 && rows <= 0x7fffffff &&
                     launch_fits(ceil_div(rows, 128) * ceil_div(c_out, 128) + 7, 512) &&
                     (x_dtype == MESORASI_I8 || quantize_fits(rows, c_in, x_dtype)),
                 MESORASI_EUNSUPPORTED, "mesorasi_linear_i8: c_in = %d, c_out = %d, rows = %lld", c_in, c_out,
                 (long long)rows);
    if (rows == 0) return MESORASI_OK;
    MESO_REQUIRE(x && W && w_scale && y, MESORASI_EINVAL, "mesorasi_linear_i8: NULL pointer");
    MESO_REQUIRE((x_scale != nullptr) == (x_dtype == MESORASI_I8), MESORASI_EINVAL,
                 "mesorasi_linear_i8: x_scale goes with 8-bit rows, and only with them");
    MESO_REQUIRE(aligned(W, 16) && (x_dtype != MESORASI_I8 || aligned(x, 16)), MESORASI_EINVAL,
                 "mesorasi_linear_i8: 8-bit rows are not 16-byte aligned");
    hipStream_t s = as_stream(stream);
    const int kp = (int)i8_pad(c_in);
    const bool f32 = y_dtype == MESORASI_F32;
    const size_t need = mesorasi_linear_i8_workspace(rows, c_in, c_out, x_dtype);
    MESO_REQUIRE(need == 0 || (ws && ws_bytes >= need), MESORASI_EWORKSPACE,
                 "mesorasi_linear_i8: workspace %zu < %zu bytes", ws ? ws_bytes : (size_t)0, need);
    MESO_REQUIRE(need == 0 || aligned(ws, 16), MESORASI_EINVAL, "mesorasi_linear_i8: ws is not 16-byte aligned");
    const int elem = x_dtype == MESORASI_F32 ? 4 : x_dtype == MESORASI_BF16 ? 2 : 1;
    const Extent ext = rows_extent(y, rows, ld_y, c_out, f32 ? 4 : 2);
    MESO_REQUIRE(!overlap(ext, rows_extent(x, rows, ld_x, c_in, elem)) && !overlap(ext, rows_extent(W, c_out, ld_w, c_in, 1)) &&
                     !overlap(ext, rows_extent(x_scale, rows, 1, 1, 4)),
                 MESORASI_EINVAL, "mesorasi_linear_i8: y overlaps an input");
    LinArgs a = {static_cast<const int8_t*>(x), x_scale, W, w_scale, bias, y, ld_x, ld_w, ld_y, rows, kp, c_out, relu};
    if (linear_few_fused(rows, kp, x_dtype)) {
        if (x_dtype == MESORASI_F32) {
            const float* p = static_cast<const float*>(x);
            f32 ? run_linear_few_fused<float, float>(a, p, c_in, s) : run_linear_few_fused<float, uint16_t>(a, p, c_in, s);
        } else {
            const uint16_t* p = static_cast<const uint16_t*>(x);
            f32 ? run_linear_few_fused<uint16_t, float>(a, p, c_in, s)
                : run_linear_few_fused<uint16_t, uint16_t>(a, p, c_in, s);
        }
        return after_launch("mesorasi_linear_i8");
    }
    if (x_dtype != MESORASI_I8) {
        int8_t* q = static_cast<int8_t*>(ws);
        float* qs = reinterpret_cast<float*>(q + rows * kp);
        run_quantize(x, ld_x, x_dtype, rows, c_in, q, kp, qs, s);
        a.x = q;
        a.ldx = kp;
        a.xs = qs;
    }
    const int rc = f32 ? run_linear<float>(a, s) : run_linear<uint16_t>(a, s);
    if (rc != MESORASI_OK) return rc;
    return after_launch("mesorasi_linear_i8");
}
