// Cross attention to another set of points: o_i = sum_j p_ij v_j / sum_j p_ij,
// p_ij = exp(s_ij - m_i), s_ij = scale q_i . k_j.
//
// One pass over the sources with a running reference m_i and sum (the online
// normalizer calculation of Milakov and Gimelshein, 2018): where a
// later score passes m_i by 8 (in powers of two) what was summed is scaled
// down, otherwise m_i stays, so that the weights are at most 256 and most
// tiles rescale nothing.  The queries of all heads that share a source head
// are rows of one product (row = point x heads of the group + head), so K and
// V are read once for them.
//
//   attention_bf16_kernel  bf16 on the matrix cores
//   attention_f32_kernel   fp32 operands in three bf16 parts, many rows
//   attention_f32_few_kernel  fp32 on the fp32 instruction, few rows
//   attention_join_kernel  joins the parts of calls that split the sources
//
// Bounds.  Many rows: 4 D operations a pair on the matrix cores and the
// weights on the vector units, which do not overlap whole.  4 x 16384 queries
// over 4096 sources, 8 heads on 2, bf16: 1.10 ms, 1000 TFLOP/s at 128 channels
// (matrix cores busy 46 %, 7 vector instructions counted a weight), 580 us,
// 948 at 64 (41 %, 5), 392 us, 702 at 32; a large bf16 library product reaches
// 1400.  Few rows: one read of K and V (8 x 1 query over 16384 sources, 8 heads
// of 128: 187 us, 5.7 TB/s in fp32; 107 us, 5.0 TB/s in bf16).
#include <algorithm>
#include <cmath>

#include "common.h"

namespace meso {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
typedef __attribute__((address_space(3))) const char* lds_cptr;

constexpr int kAtThreads = 256;

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
    // the launch
    int rows;           // query rows of a cloud and source head: Nq (Hq / Hkv)
    int row_tiles;      // workgroups over them
    int splits;         // workgroups over the sources
    int64_t blocks;     // pairs * row_tiles * splits
    int per_xcd;
    int Dp;             // channels of a part: D rounded up to 32
    float* part;        // splits > 1: [pair, split, row, Dp] sums, then [pair, split, row, 2] maximum and sum
};


// ---------------------------------------------------------------------------
// bf16
// ---------------------------------------------------------------------------

__device__ const uint4 kAtZero[1] = {};

// Slot of a 16-byte chunk in its row of CH chunks: rows that one read
// touches together lie in different banks (the scores read one chunk of 16
// rows, half of a transposed read four chunks of 4 rows).
template <int CH>
__device__ __forceinline__ int at_swz(int row) {
    const int low = (row >> 2) & 3;
    if constexpr (CH == 16)
        return ((row & 3) << 2) | low;
    else if constexpr (CH == 8)
        return (((row >> 1) & 1) << 2) | low;
    else
        return low;
}

// 16 bytes from each lane's address to LDS at base + 16 lane.  The wait is
// the caller's: at_wait_loads() before the barrier that publishes the tile.
__device__ __forceinline__ void at_load_lds(const void* g, uint32_t lds_base) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)(uintptr_t)g,
                                     (__attribute__((address_space(3))) uint32_t*)(uintptr_t)lds_base, 16, 0, 0);
}
__device__ __forceinline__ void at_wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ float at_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ float at_other_half(float v, float& lo) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    lo = __uint_as_float(r[0]);
    return __uint_as_float(r[1]);
}

// A query's sum of weights from its two lanes'.  Where its reference is
// +infinity (the largest score times the scale passes fp32's range) the weights
// are not defined, though exp2 of differences to it gives 0.
__device__ __forceinline__ float at_weights(float l, float m) {
    float lo;
    const float hi = at_other_half(l, lo);
    return m == INFINITY ? NAN : lo + hi;
}

__device__ __forceinline__ uint32_t at_pack(float a, float b) {
    bf16x2 v;
    v[0] = static_cast<__bf16>(a);
    v[1] = static_cast<__bf16>(b);
    return __builtin_bit_cast(uint32_t, v);
}

// Valid sources among the 64 from j0 on.
__device__ __forceinline__ uint64_t at_count_bits(int64_t j0, int64_t end) {
    const int64_t r = end - j0;
    return r >= 64 ? ~0ull : r <= 0 ? 0ull : (1ull << r) - 1;
}

// The waves that share R rows join: sh [W][Dp][R] their sums, sm [W][R] maxima
// and [W][R] sums of weights.
template <typename T, int Dp, int W, int R>
__device__ __forceinline__ void at_join_waves(const AttnArgs& a, const float* sh, const float* sm, int row0,
                                              int64_t pair, int split, int64_t b, int kvh, int g) {
    const int tid = threadIdx.x, r = tid & (R - 1), row = row0 + r;
    if (row >= a.rows) return;
    float mm[W], M = -INFINITY, L = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, mm[w] = sm[w * R + r]);
    const float base = M == -INFINITY ? 0.0f : M;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        mm[w] = at_exp2(mm[w] - base);
        L += mm[w] * sm[(W + w) * R + r];
    }
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    const int n = row / g, h = kvh * g + (row - n * g);
    T* op = static_cast<T*>(a.o) + b * a.ob + n * a.ol + h * a.oh;
    const int64_t pr = (pair * a.splits + split) * a.rows + row;
    for (int d = tid / R; d < a.D; d += 64 * W / R) {
        float v = 0.0f, part[W];
#pragma unroll
        for (int w = 0; w < W; ++w) part[w] = mm[w] * sh[(w * Dp + d) * R + r];
#pragma unroll
        for (int w = 0; w < W; ++w) v += mm[w] == 0.0f ? 0.0f : part[w];
        if (a.splits > 1) {
            a.part[pr * a.Dp + d] = v;
        } else {
            v = L == 0.0f ? 0.0f : v * inv;      // 0 without a weight, whatever the sums hold
            if constexpr (sizeof(T) == 4)
                op[d] = v;
            else
                op[d] = f32_to_bf16_any(v);
        }
    }
    if (a.splits > 1 && tid < R) {
        float* pm = a.part + (a.blocks / a.row_tiles) * a.rows * a.Dp;
        pm[2 * pr] = M;
        pm[2 * pr + 1] = L;
    }
}

// A row's part: its two lanes' sums, maximum and sum of weights.
template <int DB>
__device__ __forceinline__ void at_write_part(const AttnArgs& a, int64_t pr, const f32x16 (&o)[DB], float m, float l,
                                              int half) {
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            *reinterpret_cast<float4*>(a.part + pr * a.Dp + 32 * d + 2 * r + 4 * half) =
                make_float4(o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]);
    if (half == 0) {
        float* pm = a.part + (a.blocks / a.row_tiles) * a.rows * a.Dp;
        pm[2 * pr] = m;
        pm[2 * pr + 1] = l;
    }
}

// The product taken transposed, S^T = K Q^T and O^T = V^T P^T on
// v_mfma_f32_32x32x16_bf16: a lane's 16 accumulators of a block of 32
// sources belong to its own query (lane % 32), sources 8 (r / 4) + 4 (lane /
// 32) + r % 4.  So the maximum and the sum of a query's weights stay in its
// two lanes, and the weights, rounded to bf16 and packed, are the next
// product's operand as they lie if its step t takes element e of lane half h
// to be source 16 t + 8 (e / 4) + 4 h + e % 4.  V's operand in that order comes
// from LDS by transposed reads.
//
// DB: blocks of 32 channels; QB: blocks of 32 query rows of a wave.  The four
// waves share the tiles of K and V: of 64 sources where each has rows of its
// own, of 128, one block of 32 for each wave, where they share 32 rows (KS).
// GEN: rows of any width and alignment, staged by elements.
//
// Where the waves share rows the weights are kept in two bf16 parts, to 2^-15 of
// each, and V is multiplied by both: such calls wait for memory or for their
// few tiles (8 x 1 query over 16384 sources of 128 channels 106 us either way,
// 1 x 1024 over 1024 of 64 10.8 -> 12.0).  The first part is rounded down and
// the second above 0, so that an infinite v meets no 0 and no other sign.  With
// rows of their own they are rounded to bf16, 2^-8 of each, whose errors average
// out over a row's sources to about the output's own rounding: a second part
// costs what it adds to the matrix cores and the vector units (4 x 16384 over
// 4096, 8 heads on 2: 1120 -> 1530 us at 128 channels, 591 -> 877 at 64).
template <int DB, int QB, bool KS, bool GEN>
__global__ __launch_bounds__(kAtThreads, 2) void attention_bf16_kernel(AttnArgs a) {
    constexpr int CH = DB == 1 ? 4 : DB == 2 ? 8 : 16;       // 16-byte chunks of a row in LDS
    constexpr int KT = KS ? 128 : 64;                        // sources of a tile
    constexpr int NB = KS ? 1 : 2;                           // blocks of 32 of them for a wave
    constexpr int kTile = KT * CH * 16;                      // bytes of K's or V's tile
    constexpr int kLoads = KT * CH / kAtThreads;
    extern __shared__ __align__(16) char lds[];              // [2][K, V]

    const int64_t lb = (int64_t)(blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3);
    if (lb >= a.blocks) return;
    const int split = (int)(lb % a.splits);
    const int64_t rest = lb / a.splits;
    const int tile0 = (int)(rest % a.row_tiles);
    const int64_t pair = rest / a.row_tiles;
    const int64_t b = pair / a.Hkv;
    const int kvh = (int)(pair - b * a.Hkv);
    const int g = a.Hq / a.Hkv;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int half = lane >> 5, col = lane & 31;

    const uint16_t* __restrict__ kp = static_cast<const uint16_t*>(a.k) + b * a.kb + kvh * a.kh;
    const uint16_t* __restrict__ vp = static_cast<const uint16_t*>(a.v) + b * a.vb + kvh * a.vh;
    const uint8_t* __restrict__ mask = a.k_mask ? a.k_mask + b * a.mask_ld : nullptr;
    int64_t end = a.k_len ? min(max((int64_t)a.k_len[b], (int64_t)0), a.Nk) : a.Nk;
    int64_t begin = 0;
    if (a.splits > 1) {
        const int64_t per = ((end + a.splits - 1) / a.splits + KT - 1) / KT * KT;
        begin = min(end, split * per);
        end = min(end, begin + per);
    }
    const int tiles = (int)((end - begin + KT - 1) / KT);

    // scores are exponentiated as powers of two; a negative scale turns the queries around
    const float c0 = a.scale * 1.44269504088896340736f;
    const float c = c0 == 0.0f ? 1.0f : fabsf(c0);
    const uint32_t qflip = c0 < 0.0f ? 0x80008000u : 0u;
    const uint32_t qkeep = c0 == 0.0f ? 0u : ~0u;

    // the wave's queries: operand B, channel 16 s + 8 half + e
    const int row0 = tile0 * (KS ? 32 * QB : 4 * 32 * QB) + (KS ? 0 : wave * 32 * QB);
    bf16x8 qf[QB][2 * DB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int r = min(row0 + 32 * qb + col, a.rows - 1);
        const int n = r / g, h = kvh * g + (r - n * g);
        const uint16_t* qp = static_cast<const uint16_t*>(a.q) + b * a.qb + n * a.ql + h * a.qh;
#pragma unroll
        for (int s = 0; s < 2 * DB; ++s) {
            const int d0 = 16 * s + 8 * half;
            uint4 w = make_uint4(0, 0, 0, 0);
            if constexpr (GEN) {
                uint32_t u[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = d0 + e < a.D ? qp[d0 + e] : 0u;
                w = make_uint4(u[0] | u[1] << 16, u[2] | u[3] << 16, u[4] | u[5] << 16, u[6] | u[7] << 16);
            } else {
                if (d0 < a.D) w = *reinterpret_cast<const uint4*>(qp + d0);
            }
            w.x = (w.x & qkeep) ^ qflip; w.y = (w.y & qkeep) ^ qflip;
            w.z = (w.z & qkeep) ^ qflip; w.w = (w.w & qkeep) ^ qflip;
            qf[qb][s] = __builtin_bit_cast(bf16x8, w);
        }
    }

    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_cptr)lds;
    // one tile of K and V to LDS; rows that are not valid, and chunks past D, come as zeros
    auto stage = [&](int t, const uint64_t (&bits)[KT / 64]) {
        const int64_t j0 = begin + (int64_t)t * KT;
        const uint32_t base = lds0 + (t & 1) * 2 * kTile;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int p = i * kAtThreads + tid;
            const int row = p / CH, ch = (p % CH) ^ at_swz<CH>(row);
            const bool ok = ((bits[KT == 64 ? 0 : row >> 6] >> (row & 63)) & 1) && 8 * ch < a.D;
            const int64_t j = j0 + row;
            if constexpr (GEN) {
                uint32_t u[8], w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool in = ok && 8 * ch + e < a.D;
                    u[e] = in ? kp[j * a.kl + 8 * ch + e] : 0u;
                    w[e] = in ? vp[j * a.vl + 8 * ch + e] : 0u;
                }
                uint4* d = reinterpret_cast<uint4*>(lds + (t & 1) * 2 * kTile) + p;
                d[0] = make_uint4(u[0] | u[1] << 16, u[2] | u[3] << 16, u[4] | u[5] << 16, u[6] | u[7] << 16);
                d[kTile / 16] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
            } else if (DB != 3 || ch < 4 * DB) {
                const void* gk = ok ? (const void*)(kp + j * a.kl + 8 * ch) : (const void*)kAtZero;
                const void* gv = ok ? (const void*)(vp + j * a.vl + 8 * ch) : (const void*)kAtZero;
                const uint32_t l = __builtin_amdgcn_readfirstlane(base + (i * kAtThreads + wave * 64) * 16);
                at_load_lds(gk, l);
                at_load_lds(gv, l + kTile);
            }
        }
    };
    auto valid_bits = [&](int t, uint64_t (&bits)[KT / 64]) {
#pragma unroll
        for (int i = 0; i < KT / 64; ++i) {
            const int64_t j = begin + (int64_t)t * KT + 64 * i;
            bits[i] = at_count_bits(j, end);
            if (mask) bits[i] &= ballot(j + lane < end && mask[j + lane]);
        }
    };

    f32x16 oacc[QB][DB];
    float m[QB], l[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        m[qb] = -INFINITY;
        l[qb] = 0.0f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) oacc[qb][d][r] = 0.0f;
    }

    const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3f803f80u);
    // a lane's place in the tiles
    const int swk = at_swz<CH>(col);
    const int vi = lane & 15, vg = (lane >> 4) & 1;
    const int vrow = 4 * half + (vi >> 2);                     // + 16 t + 8 (e / 4): bits 0..2 of the source
    const int vch = 2 * vg + ((vi & 3) >> 1), vin = 8 * (vi & 1);

    uint64_t cur[KT / 64], nxt[KT / 64] = {};
    if (tiles > 0) {
        valid_bits(0, cur);
        stage(0, cur);
        if (tiles > 1) valid_bits(1, nxt);
    }
    for (int t = 0; t < tiles; ++t) {
        at_wait_loads();
        __syncthreads();
        if (t + 1 < tiles) stage(t + 1, nxt);
        const char* tk = lds + (t & 1) * 2 * kTile;
        const char* tv = tk + kTile;

        // scores: the next block's operands are read between this block's products
        f32x16 s[QB][NB];
        bf16x8 kf[2][2 * DB];
        auto read_k = [&](int kb, int st) {
            const int blk = KS ? wave : kb;
            return *reinterpret_cast<const bf16x8*>(tk + (32 * blk + col) * CH * 16 + (((2 * st + half) ^ swk) << 4));
        };
#pragma unroll
        for (int st = 0; st < 2 * DB; ++st) kf[0][st] = read_k(0, st);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[qb][kb][r] = 0.0f;
#pragma unroll
            for (int st = 0; st < 2 * DB; ++st) {
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
                    s[qb][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kb & 1][st], qf[qb][st], s[qb][kb], 0, 0, 0);
                if (kb + 1 < NB) kf[(kb + 1) & 1][st] = read_k(kb + 1, st);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        // sources that are not valid
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            const int blk = KS ? wave : kb;
            const uint32_t w32 = (uint32_t)(cur[KT == 64 ? 0 : blk >> 1] >> (32 * (blk & 1)));
            if (w32 != 0xffffffffu) {
                const uint32_t w = w32 >> (4 * half);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const bool ok = (w >> (8 * (r / 4) + r % 4)) & 1;
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) s[qb][kb][r] = ok ? s[qb][kb][r] : -INFINITY;
                }
            }
        }
        // weights: the reference m of a query moves when its maximum passes it by 8 (a factor of 256)
        uint32_t pk[QB][NB][8], pl[QB][NB][8];           // pl: the second parts (KS)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            float mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[qb][kb][r]);
            float lo;
            const float hi = at_other_half(mx, lo);
            mx = fmaxf(lo, hi) * c;
            if (ballot(mx > m[qb] + 8.0f)) {
                const float mn = fmaxf(m[qb], mx);
                const float f = mn == -INFINITY ? 1.0f : at_exp2(m[qb] - mn);
                m[qb] = mn;
                l[qb] *= f;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) oacc[qb][d][r] *= f;
            }
            const float base = m[qb] == -INFINITY ? 0.0f : m[qb];
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                for (int r = 0; r < 16; r += 2) {
                    // the sum takes the rounded weights, as the product with V does
                    const float p0 = at_exp2(fmaf(s[qb][kb][r], c, -base));
                    const float p1 = at_exp2(fmaf(s[qb][kb][r + 1], c, -base));
                    const uint32_t b0 = __float_as_uint(p0) & 0xffff0000u, b1 = __float_as_uint(p1) & 0xffff0000u;
                    const uint32_t hi = KS ? b0 >> 16 | b1 : at_pack(p0, p1);
                    pk[qb][kb][r / 2] = hi;
                    l[qb] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, hi), ones, l[qb], false);
                    if constexpr (KS) {
                        // p (1 + 2^-23) - hi
                        const uint32_t lo = at_pack(fmaf(p0, 1.00000012f, -__uint_as_float(b0)),
                                                    fmaf(p1, 1.00000012f, -__uint_as_float(b1)));
                        pl[qb][kb][r / 2] = lo;
                        l[qb] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, lo), ones, l[qb], false);
                    }
                }
        }
        // outputs
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            const int blk = KS ? wave : kb;
#pragma unroll
            for (int st = 0; st < 2; ++st) {
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    s16x4 v[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int row = 32 * blk + 16 * st + 8 * e + vrow;
                        const int ch = (4 * d + vch) ^ (at_swz<CH>(vrow) | 2 * e);
                        v[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            (lds_s16x4)(tv + row * CH * 16 + (ch << 4) + vin));
                    }
                    const uint4 vw = make_uint4(__builtin_bit_cast(uint2, v[0]).x, __builtin_bit_cast(uint2, v[0]).y,
                                                __builtin_bit_cast(uint2, v[1]).x, __builtin_bit_cast(uint2, v[1]).y);
                    const bf16x8 vf = __builtin_bit_cast(bf16x8, vw);
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) {
                        if constexpr (KS) {
                            const uint4 lw = make_uint4(pl[qb][kb][4 * st], pl[qb][kb][4 * st + 1],
                                                        pl[qb][kb][4 * st + 2], pl[qb][kb][4 * st + 3]);
                            oacc[qb][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, lw),
                                                                                  oacc[qb][d], 0, 0, 0);
                        }
                        const uint4 pw = make_uint4(pk[qb][kb][4 * st], pk[qb][kb][4 * st + 1], pk[qb][kb][4 * st + 2],
                                                    pk[qb][kb][4 * st + 3]);
                        oacc[qb][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, pw),
                                                                              oacc[qb][d], 0, 0, 0);
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < KT / 64; ++i) cur[i] = nxt[i];
        if (t + 2 < tiles) valid_bits(t + 2, nxt);
    }

    // the two lanes of a query join their sums
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) l[qb] = at_weights(l[qb], m[qb]);
    if constexpr (KS) {
        constexpr int Dp = 32 * DB;
        // the waves join: [wave][d][32 rows] sums, then their maxima and sums
        float* sh = reinterpret_cast<float*>(lds);
        float* sm = sh + 4 * Dp * 32;
        __syncthreads();
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                sh[(wave * Dp + 32 * d + 8 * (r / 4) + 4 * half + r % 4) * 32 + col] = oacc[0][d][r];
        if (half == 0) {
            sm[wave * 32 + col] = m[0];
            sm[128 + wave * 32 + col] = l[0];
        }
        __syncthreads();
        at_join_waves<uint16_t, Dp, 4, 32>(a, sh, sm, row0, pair, split, b, kvh, g);
    } else {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const int row = row0 + 32 * qb + col;
            if (row >= a.rows) continue;
            if (a.splits > 1) {
                at_write_part<DB>(a, (pair * a.splits + split) * a.rows + row, oacc[qb], m[qb], l[qb], half);
                continue;
            }
            const bool none = l[qb] == 0.0f;         // 0 then, whatever the sums hold
            const float inv = none ? 0.0f : 1.0f / l[qb];
            const int n = row / g, h = kvh * g + (row - n * g);
            uint16_t* op = static_cast<uint16_t*>(a.o) + b * a.ob + n * a.ol + h * a.oh;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int d0 = 32 * d + 2 * r + 4 * half;
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = none ? 0.0f : oacc[qb][d][r + e] * inv;
                    if constexpr (GEN) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (d0 + e < a.D) op[d0 + e] = f32_to_bf16_any(v[e]);
                    } else if (d0 < a.D) {
                        *reinterpret_cast<uint2*>(op + d0) = make_uint2(at_pack(v[0], v[1]), at_pack(v[2], v[3]));
                    }
                }
        }
    }
}

// ---------------------------------------------------------------------------
// fp32
// ---------------------------------------------------------------------------

// v = hi + mid + lo, each in bf16: 8 bits each of a float's 24, with nothing
// left over -- of values from 2^-110 (below, what the last parts lose is at most
// 2^-134) to 3.38e38 (above, and for infinities, the parts are no numbers).
struct AtSplit {
    uint32_t hi, mid, lo;            // of two values
};

__device__ __forceinline__ AtSplit at_split(float a, float b) {
    AtSplit s;
    s.hi = at_pack(a, b);
    a -= __uint_as_float(s.hi << 16);
    b -= __uint_as_float(s.hi & 0xffff0000u);
    s.mid = at_pack(a, b);
    a -= __uint_as_float(s.mid << 16);
    b -= __uint_as_float(s.mid & 0xffff0000u);
    s.lo = at_pack(a, b);
    return s;
}

// Eight values into one operand of each part.
__device__ __forceinline__ void at_split8(const float (&f)[8], uint4 (&w)[3]) {
    AtSplit s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = at_split(f[2 * i], f[2 * i + 1]);
    w[0] = make_uint4(s[0].hi, s[1].hi, s[2].hi, s[3].hi);
    w[1] = make_uint4(s[0].mid, s[1].mid, s[2].mid, s[3].mid);
    w[2] = make_uint4(s[0].lo, s[1].lo, s[2].lo, s[3].lo);
}

// A product of split operands: the six partial products down to 2^-16 of it,
// the small ones first; the three left out are below 2^-24.
__device__ __forceinline__ f32x16 at_mfma6(const bf16x8 (&a)[3], const bf16x8 (&b)[3], f32x16 c) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[2], b[0], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[2], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1], b[1], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1], b[0], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[1], c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[0], c, 0, 0, 0);
}

// The bf16 kernel's scheme with every operand in three bf16 parts and six
// matrix instructions a product: 419 TFLOP/s at most instead of the fp32
// instruction's 157.  K and V are split once a tile, on their way to LDS (the
// next tile's rows wait in registers); Q once, the weights where they form.
// Four waves with 32 rows of their own.  4 x 4096 queries over 1024 sources, 8
// heads of 64: 181 us, 190 TFLOP/s, matrix cores busy 52 %; of 128: 443 us, 155,
// busy 37 %, one wave a SIMD.
//
// Values that the parts do not hold show in the results.  An infinity or a huge
// value in k, or products past fp32's range with parts of either sign, give NaN
// scores and sums; in v infinite or NaN outputs; and where v is so small that
// 2^-134 counts, so are outputs.  A workgroup that finds such a result (from a
// NaN of its inputs too), or a query outside [2^-102, 2^60] and 0, or a scale
// that would show the small parts of k, goes over its tiles again with the fp32
// instruction, for those queries alone.  (Testing every tile's values as they
// are split instead took 7 to 17 % of the time.)
constexpr float kAtLargeQ = 0x1p60f, kAtSmallQ = 0x1p-102f, kAtSmallOut = 0x1p-108f, kAtMaxScale = 0x1p20f;

template <int DB>
struct AtF32 {
    static constexpr int KT = DB > 2 ? 32 : 64;                         // sources of a tile
    static constexpr int CH = DB == 1 ? 4 : DB == 2 ? 8 : 16;           // 16-byte chunks of a row of one part
    static constexpr int kPart = KT * CH * 16;                          // bytes of one part of a tile
    static constexpr int kUnits = KT * CH / kAtThreads;                 // chunks of K (and of V) a thread stages
    static constexpr int kRow = 8 * CH + 4;                             // floats of a row that is not split
    static constexpr int kFlags = 6 * kPart;                            // the waves' flags
    static constexpr int kLds = kFlags + 16;
    static_assert(2 * KT * kRow * 4 <= kFlags, "K and V in fp32 fit the parts' place");
};

// A workgroup's place: cloud, source head, part of the sources, query rows.
struct AtPlace {
    int64_t pair, b, begin, end;
    int split, row0, kvh, g, tiles;
    const uint8_t* mask;
    __device__ __forceinline__ AtPlace(const AttnArgs& a, int64_t lb, int kt, int rows) {
        split = (int)(lb % a.splits);
        const int64_t rest = lb / a.splits;
        row0 = (int)(rest % a.row_tiles) * rows;
        pair = rest / a.row_tiles;
        b = pair / a.Hkv;
        kvh = (int)(pair - b * a.Hkv);
        g = a.Hq / a.Hkv;
        mask = a.k_mask ? a.k_mask + b * a.mask_ld : nullptr;
        begin = 0;
        end = a.k_len ? min(max((int64_t)a.k_len[b], (int64_t)0), a.Nk) : a.Nk;
        if (a.splits > 1) {
            const int64_t per = ((end + a.splits - 1) / a.splits + kt - 1) / kt * kt;
            begin = min(end, split * per);
            end = min(end, begin + per);
        }
        tiles = (int)((end - begin + kt - 1) / kt);
    }
};

// Eight channels from d0 on, zeros past D; without GEN D is a multiple of 4.
template <bool GEN>
__device__ __forceinline__ void at_read8(const AttnArgs& a, const float* p, int d0, bool ok, float (&f)[8]) {
    if constexpr (GEN) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = ok && d0 + e < a.D ? p[d0 + e] : 0.0f;
    } else {
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (ok && d0 + e < a.D) v = *reinterpret_cast<const float4*>(p + d0 + e);
            f[e] = v.x; f[e + 1] = v.y; f[e + 2] = v.z; f[e + 3] = v.w;
        }
    }
}

// A wave's 32 queries in fp32: running reference and sums, the scores' factor c
// (of a power of two), the queries' factor (a negative scale turns them around,
// a scale of 0 clears them).
template <int DB>
struct AtRows {
    f32x16 oacc[DB];
    float m, l, c, qmul;
    __device__ __forceinline__ explicit AtRows(const AttnArgs& a) : m(-INFINITY), l(0.0f) {
        const float c0 = a.scale * 1.44269504088896340736f;
        c = c0 == 0.0f ? 1.0f : fabsf(c0);
        qmul = c0 == 0.0f ? 0.0f : c0 < 0.0f ? -1.0f : 1.0f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) oacc[d][r] = 0.0f;
    }
    // sources of a block of 32 that are not valid
    static __device__ __forceinline__ void drop(f32x16& s, uint32_t w32, int half) {
        if (w32 != 0xffffffffu) {
            const uint32_t w = w32 >> (4 * half);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = (w >> (8 * (r / 4) + r % 4)) & 1 ? s[r] : -INFINITY;
        }
    }
    // The reference m moves when a block's maximum passes it by 8; gives the factor of what was summed before.
    __device__ __forceinline__ float advance(const f32x16& s) {
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        float lo;
        const float hi = at_other_half(mx, lo);
        mx = fmaxf(lo, hi) * c;
        const float mn = mx > m + 8.0f ? mx : m;
        const float f = mn == m ? 1.0f : at_exp2(m - mn);
        m = mn;
        return f;
    }
    __device__ __forceinline__ float base() const { return m == -INFINITY ? 0.0f : m; }
    __device__ __forceinline__ void rescale(float f) {
        if (ballot(f != 1.0f)) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) oacc[d][r] *= f;
        }
    }
    __device__ __forceinline__ void join_halves() { l = at_weights(l, m); }
    // a row without a weight is 0, whatever its sums hold
    template <bool GEN>
    __device__ __forceinline__ void write(const AttnArgs& a, const AtPlace& p, int row, int half) const {
        if (row >= a.rows) return;
        if (a.splits > 1) {
            at_write_part<DB>(a, (p.pair * a.splits + p.split) * a.rows + row, oacc, m, l, half);
            return;
        }
        const bool none = l == 0.0f;
        const float inv = none ? 0.0f : 1.0f / l;
        const int n = row / p.g, h = p.kvh * p.g + (row - n * p.g);
        float* op = static_cast<float*>(a.o) + p.b * a.ob + n * a.ol + h * a.oh;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int d0 = 32 * d + 2 * r + 4 * half;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = none ? 0.0f : oacc[d][r + e] * inv;
                if constexpr (GEN) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (d0 + e < a.D) op[d0 + e] = v[e];
                } else if (d0 < a.D) {
                    *reinterpret_cast<float4*>(op + d0) = make_float4(v[0], v[1], v[2], v[3]);
                }
            }
    }
};

// A wave's queries in `again` on v_mfma_f32_32x32x2_f32, which takes any value:
// a lane supplies row or column lane % 32 and k = lane / 32.  Scores: channels
// 8 i + 4 (lane / 32) + e are step (i, e).  Outputs: step r takes the sources of
// the lane's own weights.  Block, thread and the kernel's arguments (its only
// parameter) are taken through an empty asm, so that the kernel before it keeps
// none of this in registers (it was 4 to 8 % slower with them).
template <int DB, bool GEN>
__device__ __forceinline__ void attention_f32_plain(int block, int tid, uint32_t again, char* lds) {
    using P = AtF32<DB>;
    constexpr int CH = P::CH, KT = P::KT;
    static_assert(sizeof(AttnArgs) % 8 == 0, "whole words");
    struct Words {
        uint64_t w[sizeof(AttnArgs) / 8];
    } words;
    auto* args = (__attribute__((address_space(4))) const uint64_t*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(block), "+v"(tid), "+s"(args));
#pragma unroll
    for (int i = 0; i < (int)(sizeof(AttnArgs) / 8); ++i) words.w[i] = args[i];
    const AttnArgs a = __builtin_bit_cast(AttnArgs, words);
    const AtPlace p(a, (int64_t)(block & 7) * a.per_xcd + (block >> 3), KT, 128);
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, half = lane >> 5, col = lane & 31;
    const float* __restrict__ kp = static_cast<const float*>(a.k) + p.b * a.kb + p.kvh * a.kh;
    const float* __restrict__ vp = static_cast<const float*>(a.v) + p.b * a.vb + p.kvh * a.vh;
    const int row = p.row0 + wave * 32 + col, rc = min(row, a.rows - 1), n = rc / p.g, h = p.kvh * p.g + (rc - n * p.g);
    const float* qp = static_cast<const float*>(a.q) + p.b * a.qb + n * a.ql + h * a.qh;
    float* pk = reinterpret_cast<float*>(lds);
    float* pv = pk + KT * P::kRow;
    AtRows<DB> o(a);
#pragma unroll 1
    for (int t = 0; t < p.tiles; ++t) {
        const int64_t j0 = p.begin + (int64_t)t * KT;
        uint64_t bits = at_count_bits(j0, p.end);
        if (p.mask) bits &= ballot(j0 + lane < p.end && p.mask[j0 + lane]);
        __syncthreads();             // the tile before has been read
#pragma unroll 1
        for (int i = 0; i < P::kUnits; ++i) {
            const int u = i * kAtThreads + tid, r = u / CH, ch = u % CH;
            const bool ok = (bits >> r) & 1;
            float x[8], y[8];
            at_read8<GEN>(a, kp + (j0 + r) * a.kl, 8 * ch, ok, x);
            at_read8<GEN>(a, vp + (j0 + r) * a.vl, 8 * ch, ok, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                pk[r * P::kRow + 8 * ch + e] = x[e];
                pv[r * P::kRow + 8 * ch + e] = y[e];
            }
        }
        __syncthreads();
#pragma unroll 1
        for (int kb = 0; kb < KT / 32; ++kb) {
            f32x16 s;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = 0.0f;
#pragma unroll 1
            for (int i = 0; i < 4 * DB; ++i) {
                float q[8];
                at_read8<GEN>(a, qp, 8 * i, o.qmul != 0.0f, q);
                const float4 k = *reinterpret_cast<const float4*>(pk + (32 * kb + col) * P::kRow + 8 * i + 4 * half);
                s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.x, (half ? q[4] : q[0]) * o.qmul, s, 0, 0, 0);
                s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.y, (half ? q[5] : q[1]) * o.qmul, s, 0, 0, 0);
                s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.z, (half ? q[6] : q[2]) * o.qmul, s, 0, 0, 0);
                s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.w, (half ? q[7] : q[3]) * o.qmul, s, 0, 0, 0);
            }
            AtRows<DB>::drop(s, (uint32_t)(bits >> (32 * kb)), half);
            const float f = o.advance(s), base = o.base();
            o.rescale(f);
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = at_exp2(fmaf(s[r], o.c, -base));
                sum += s[r];
            }
            o.l = o.l * f + sum;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float* v = pv + (32 * kb + 8 * (r / 4) + 4 * half + r % 4) * P::kRow + col;
#pragma unroll
                for (int d = 0; d < DB; ++d)
                    o.oacc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[32 * d], s[r], o.oacc[d], 0, 0, 0);
            }
        }
    }
    o.join_halves();
    if ((again >> col) & 1) o.template write<GEN>(a, p, row, half);
}

template <int DB, bool GEN>
__global__ __launch_bounds__(kAtThreads, (DB > 2 ? 1 : DB == 2 ? 2 : 3)) void attention_f32_kernel(AttnArgs a) {
    using P = AtF32<DB>;
    constexpr int CH = P::CH, KT = P::KT, NB = KT / 32;
    extern __shared__ __align__(16) char lds[];              // K's three parts, then V's; the waves' flags

    const int64_t lb = (int64_t)(blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3);
    if (lb >= a.blocks) return;
    const AtPlace p(a, lb, KT, 128);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int half = lane >> 5, col = lane & 31;

    const float* __restrict__ kp = static_cast<const float*>(a.k) + p.b * a.kb + p.kvh * a.kh;
    const float* __restrict__ vp = static_cast<const float*>(a.v) + p.b * a.vb + p.kvh * a.vh;
    const int64_t begin = p.begin, end = p.end;
    const int tiles = p.tiles;
    AtRows<DB> o(a);
    const float c = o.c;

    // the wave's queries: operand B, channel 16 s + 8 half + e
    const int row = p.row0 + wave * 32 + col;
    bf16x8 qf[2 * DB][3];
    float qtop = 0.0f;
    uint32_t qlow = ~0u;             // of magnitudes that are not 0: twice their bits, less 1
    {
        const int r = min(row, a.rows - 1), n = r / p.g, h = p.kvh * p.g + (r - n * p.g);
        const float* qp = static_cast<const float*>(a.q) + p.b * a.qb + n * a.ql + h * a.qh;
#pragma unroll
        for (int s = 0; s < 2 * DB; ++s) {
            float f[8];
            uint4 w[3];
            at_read8<GEN>(a, qp, 16 * s + 8 * half, o.qmul != 0.0f, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                f[e] *= o.qmul;
                qtop = fmaxf(qtop, fabsf(f[e]));
                qlow = min(qlow, (__float_as_uint(f[e]) << 1) - 1u);
            }
            at_split8(f, w);
#pragma unroll
            for (int i = 0; i < 3; ++i) qf[s][i] = __builtin_bit_cast(bf16x8, w[i]);
        }
    }
    const uint64_t q_lanes = ballot(c > kAtMaxScale || qtop > kAtLargeQ ||
                                    qlow < (__builtin_bit_cast(uint32_t, kAtSmallQ) << 1) - 1u);

    auto valid_bits = [&](int t) {
        const int64_t j = begin + (int64_t)t * KT;
        uint64_t bits = at_count_bits(j, end);
        if (p.mask) bits &= ballot(j + lane < end && p.mask[j + lane]);
        return bits;
    };
    float kr[P::kUnits][8], vr[P::kUnits][8];
    auto fetch = [&](int t, uint64_t bits) {
        const int64_t j0 = begin + (int64_t)t * KT;
#pragma unroll
        for (int i = 0; i < P::kUnits; ++i) {
            const int u = i * kAtThreads + tid, r = u / CH, ch = (u % CH) ^ at_swz<CH>(r);
            const bool ok = (bits >> r) & 1;
            at_read8<GEN>(a, kp + (j0 + r) * a.kl, 8 * ch, ok, kr[i]);
            at_read8<GEN>(a, vp + (j0 + r) * a.vl, 8 * ch, ok, vr[i]);
        }
    };
    auto store = [&]() {
#pragma unroll
        for (int i = 0; i < P::kUnits; ++i) {
            uint4 w[3], x[3];
            at_split8(kr[i], w);
            at_split8(vr[i], x);
            char* d = lds + (i * kAtThreads + tid) * 16;
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                *reinterpret_cast<uint4*>(d + k * P::kPart) = w[k];
                *reinterpret_cast<uint4*>(d + (3 + k) * P::kPart) = x[k];
            }
        }
    };

    const int swk = at_swz<CH>(col);
    const int vi = lane & 15, vg = (lane >> 4) & 1;
    const int vrow = 4 * half + (vi >> 2);
    const int vch = 2 * vg + ((vi & 3) >> 1), vin = 8 * (vi & 1);

    uint64_t cur = 0, nxt = 0;
    if (tiles > 0) {
        cur = valid_bits(0);
        fetch(0, cur);
    }
    for (int t = 0; t < tiles; ++t) {
        __syncthreads();             // the tile before has been read
        store();
        __syncthreads();
        if (t + 1 < tiles) {
            nxt = valid_bits(t + 1);
            fetch(t + 1, nxt);
        }
        const char* tk = lds;
        const char* tv = lds + 3 * P::kPart;

        // One block of 32 sources after another, so that a block's weights form between the products of its neighbors:
        // scores 0, scores 1 with weights 0, outputs 0 with weights 1, outputs 1.
        f32x16 s[NB];
        bf16x8 pb[2][3];
        float f;
        auto scores = [&](int kb) {
            const char* base = tk + (32 * kb + col) * CH * 16;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kb][r] = 0.0f;
            bf16x8 kf[2][3];
            auto read_k = [&](int st) {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    kf[st & 1][i] =
                        *reinterpret_cast<const bf16x8*>(base + i * P::kPart + (((2 * st + half) ^ swk) << 4));
            };
            read_k(0);
#pragma unroll
            for (int st = 0; st < 2 * DB; ++st) {
                if (st + 1 < 2 * DB) read_k(st + 1);
                s[kb] = at_mfma6(kf[st & 1], qf[st], s[kb]);
            }
        };
        // weights in three parts, and the factor f of what was summed before
        auto weights = [&](int kb, bf16x8 (&p)[2][3]) {
            f = o.advance(s[kb]);
            const float base = o.base();
            float sum = 0.0f;
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                // a step's 16 weights: sources 16 st + 8 (e / 4) + 4 half + e % 4
                float pf[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) pf[e] = at_exp2(fmaf(s[kb][8 * st + e], c, -base));
#pragma unroll
                for (int e = 0; e < 8; e += 2) sum += pf[e] + pf[e + 1];
                uint4 pw[3];
                at_split8(pf, pw);
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    // formed here, between the products, and not where the outputs take them
                    asm volatile("" : "+v"(pw[i].x), "+v"(pw[i].y), "+v"(pw[i].z), "+v"(pw[i].w));
                    p[st][i] = __builtin_bit_cast(bf16x8, pw[i]);
                }
            }
            o.l = o.l * f + sum;
        };
        auto outputs = [&](int kb, const bf16x8 (&p)[2][3]) {
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    bf16x8 vf[3];
#pragma unroll
                    for (int i = 0; i < 3; ++i) {
                        s16x4 v[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int vr0 = 32 * kb + 16 * st + 8 * e + vrow;
                            const int ch = (4 * d + vch) ^ (at_swz<CH>(vrow) | 2 * e);
                            v[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                (lds_s16x4)(tv + i * P::kPart + vr0 * CH * 16 + (ch << 4) + vin));
                        }
                        const uint4 vw =
                            make_uint4(__builtin_bit_cast(uint2, v[0]).x, __builtin_bit_cast(uint2, v[0]).y,
                                       __builtin_bit_cast(uint2, v[1]).x, __builtin_bit_cast(uint2, v[1]).y);
                        vf[i] = __builtin_bit_cast(bf16x8, vw);
                    }
                    o.oacc[d] = at_mfma6(vf, p[st], o.oacc[d]);
                }
        };
        scores(0);
        o.drop(s[0], (uint32_t)cur, half);
        if constexpr (NB == 2) {
            bf16x8 pb1[2][3];
            scores(1);
            weights(0, pb);
            o.rescale(f);
            o.drop(s[1], (uint32_t)(cur >> 32), half);
            outputs(0, pb);
            weights(1, pb1);
            o.rescale(f);
            outputs(1, pb1);
        } else {
            weights(0, pb);
            o.rescale(f);
            outputs(0, pb);
        }
        cur = nxt;
    }

    o.join_halves();

    // results that ask for the fp32 instruction: times 0 they are not 0, or they are small but not 0
    float nan = o.l * 0.0f;
    uint32_t low = ~0u;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            nan = fmaf(o.oacc[d][r], 0.0f, nan);
            low = min(low, (__float_as_uint(o.oacc[d][r]) << 1) - 1u);
        }
    const uint64_t lanes =
        q_lanes | ballot(nan != 0.0f || low < (__float_as_uint(o.l * kAtSmallOut) << 1) - 1u);
    const uint32_t again = (uint32_t)lanes | (uint32_t)(lanes >> 32);        // of the wave's queries
    if (lane == 0) reinterpret_cast<uint32_t*>(lds + P::kFlags)[wave] = again;
    if (!((again >> col) & 1)) o.template write<GEN>(a, p, row, half);
    __syncthreads();
    const uint4 all = *reinterpret_cast<const uint4*>(lds + P::kFlags);
    if (__builtin_amdgcn_readfirstlane(all.x | all.y | all.z | all.w))
        attention_f32_plain<DB, GEN>(blockIdx.x, threadIdx.x, again, lds);
}

// Few rows in fp32: 16 RB query rows, the fp32 instruction, and K and V from
// memory straight to its operands, so that nothing waits for a tile: the
// waves take blocks of 16 sources in turn and join at the end.  On
// v_mfma_f32_16x16x4_f32 a lane supplies row or column lane % 16 and one k, lane
// / 16 = g.  Scores: the k of a step are channels 16 i + 4 g + e, so that a
// lane's 16 bytes of its source's row are four steps; a lane's four scores are
// sources 4 g + r of query lane % 16.  Outputs: step r takes source 4 g + r,
// and 16 bytes of its row, channels 64 q + 4 (lane % 16) + e, are four blocks'
// operands.
// Bound: one read of K and V (157 TFLOP/s hold 20 bytes a clock and compute
// unit for 16 rows).
template <int DQ, int RB, bool GEN>
__global__ __launch_bounds__(kAtThreads, (DQ * RB > 2 ? 1 : 2)) void attention_f32_few_kernel(AttnArgs a) {
    constexpr int R = 16 * RB, W = kAtThreads / 64;
    extern __shared__ __align__(16) char lds[];              // the waves' sums, then their maxima and sums of weights
    float* sh = reinterpret_cast<float*>(lds);
    float* sm = sh + W * 64 * DQ * R;
    const int64_t lb = (int64_t)(blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3);
    if (lb >= a.blocks) return;
    const int split = (int)(lb % a.splits);
    const int64_t rest = lb / a.splits;
    const int tile0 = (int)(rest % a.row_tiles);
    const int64_t pair = rest / a.row_tiles;
    const int64_t b = pair / a.Hkv;
    const int kvh = (int)(pair - b * a.Hkv), g = a.Hq / a.Hkv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int l16 = lane & 15, grp = lane >> 4;

    const float* __restrict__ kp = static_cast<const float*>(a.k) + b * a.kb + kvh * a.kh;
    const float* __restrict__ vp = static_cast<const float*>(a.v) + b * a.vb + kvh * a.vh;
    const uint8_t* __restrict__ mask = a.k_mask ? a.k_mask + b * a.mask_ld : nullptr;
    int64_t end = a.k_len ? min(max((int64_t)a.k_len[b], (int64_t)0), a.Nk) : a.Nk;
    int64_t begin = 0;
    if (a.splits > 1) {
        const int64_t per = ((end + a.splits - 1) / a.splits + 63) / 64 * 64;
        begin = min(end, split * per);
        end = min(end, begin + per);
    }
    const float c0 = a.scale * 1.44269504088896340736f;
    const float c = c0 == 0.0f ? 1.0f : fabsf(c0);
    auto read4 = [&](const float* p, int d0, bool ok) {
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (GEN) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (ok && d0 + e < a.D) v[e] = p[d0 + e];
        } else {                     // D is a multiple of 4
            if (ok && d0 < a.D) v = *reinterpret_cast<const f32x4*>(p + d0);
        }
        return v;
    };
    f32x4 qf[RB][4 * DQ];
#pragma unroll
    for (int j = 0; j < RB; ++j) {
        const int r = min(tile0 * R + 16 * j + l16, a.rows - 1), n = r / g, h = kvh * g + (r - n * g);
        const float* qp = static_cast<const float*>(a.q) + b * a.qb + n * a.ql + h * a.qh;
#pragma unroll
        for (int i = 0; i < 4 * DQ; ++i) {
            qf[j][i] = read4(qp, 16 * i + 4 * grp, true);
#pragma unroll
            for (int e = 0; e < 4; ++e) qf[j][i][e] = c0 == 0.0f ? 0.0f : c0 < 0.0f ? -qf[j][i][e] : qf[j][i][e];
        }
    }
    f32x4 o[RB][DQ][4];
    float m[RB], l[RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) {
        m[j] = -INFINITY;
        l[j] = 0.0f;
#pragma unroll
        for (int q = 0; q < DQ; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[j][q][e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    f32x4 kn[4 * DQ], vn[4][DQ];
    uint32_t bits_n = 0;
    auto fetch = [&](int64_t j0) {
        const bool ok = j0 + l16 < end && (!mask || mask[j0 + l16]);
        bits_n = (uint32_t)ballot(ok) & 0xffffu;
#pragma unroll
        for (int i = 0; i < 4 * DQ; ++i) kn[i] = read4(kp + (j0 + l16) * a.kl, 16 * i + 4 * grp, ok);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int q = 0; q < DQ; ++q)
                vn[r][q] = read4(vp + (j0 + 4 * grp + r) * a.vl, 64 * q + 4 * l16, (bits_n >> (4 * grp + r)) & 1);
    };
    if (begin + 16 * wave < end) fetch(begin + 16 * wave);
    for (int64_t j0 = begin + 16 * wave; j0 < end; j0 += 16 * W) {
        // the next block's rows come while this one's are multiplied
        const uint32_t bits = bits_n;
        f32x4 kf[4 * DQ], vf[4][DQ];
#pragma unroll
        for (int i = 0; i < 4 * DQ; ++i) kf[i] = kn[i];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int q = 0; q < DQ; ++q) vf[r][q] = vn[r][q];
        if (j0 + 16 * W < end) fetch(j0 + 16 * W);
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            f32x4 s0 = {0.0f, 0.0f, 0.0f, 0.0f}, s1 = s0;
#pragma unroll
            for (int i = 0; i < 4 * DQ; ++i) {
                if (16 * i >= a.D) break;
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i][e], qf[j][i][e], s0, 0, 0, 0);
                    s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i][e + 1], qf[j][i][e + 1], s1, 0, 0, 0);
                }
            }
            float mx = -INFINITY;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s0[r] = (bits >> (4 * grp + r)) & 1 ? s0[r] + s1[r] : -INFINITY;
                mx = fmaxf(mx, s0[r]);
            }
            const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
            float lo;
            const float hi = at_other_half(mx, lo);
            mx = fmaxf(lo, hi) * c;
            if (ballot(mx > m[j] + 8.0f)) {
                const float mn = fmaxf(m[j], mx);
                const float f = mn == -INFINITY ? 1.0f : at_exp2(m[j] - mn);
                m[j] = mn;
                l[j] *= f;
#pragma unroll
                for (int q = 0; q < DQ; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[j][q][e] *= f;
            }
            const float base = m[j] == -INFINITY ? 0.0f : m[j];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float p = at_exp2(fmaf(s0[r], c, -base));
                l[j] += p;
#pragma unroll
                for (int q = 0; q < DQ; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[j][q][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[r][q][e], p, o[j][q][e], 0, 0, 0);
            }
        }
    }
    // a query's four lanes join their sums, then the waves
#pragma unroll
    for (int j = 0; j < RB; ++j) {
        const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(l[j]), __float_as_uint(l[j]), false, false);
        l[j] = at_weights(__uint_as_float(x[0]) + __uint_as_float(x[1]), m[j]);
#pragma unroll
        for (int q = 0; q < DQ; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    sh[(wave * 64 * DQ + 64 * q + 16 * grp + 4 * r + e) * R + 16 * j + l16] = o[j][q][e][r];
        if (grp == 0) {
            sm[wave * R + 16 * j + l16] = m[j];
            sm[(W + wave) * R + 16 * j + l16] = l[j];
        }
    }
    __syncthreads();
    at_join_waves<float, 64 * DQ, W, R>(a, sh, sm, tile0 * R, pair, split, b, kvh, g);
}

constexpr int kAtMaxSplits = 256;

// The splits' results of one row, joined: their weights first, a split per
// thread, then the sums, 32 lanes of 4 channels over every eighth split.
template <typename T>
__global__ __launch_bounds__(kAtThreads) void attention_join_kernel(AttnArgs a) {
    __shared__ float w[kAtMaxSplits], red[4];
    __shared__ float4 sum[kAtThreads / 32][32];
    const int tid = threadIdx.x, lane = tid & 31, grp = tid >> 5;
    const int64_t pair = blockIdx.x / a.rows;
    const int row = (int)(blockIdx.x - pair * a.rows);
    const int64_t first = pair * a.splits * a.rows + row;
    const float* pm = a.part + (int64_t)gridDim.x * a.splits * a.Dp;
    float m = -INFINITY, l = 0.0f;
    if (tid < a.splits) {
        const float2 v = *reinterpret_cast<const float2*>(pm + 2 * (first + tid * (int64_t)a.rows));
        m = v.x;
        l = v.y;
    }
    float M = wave_max_f32(m);
    if ((tid & 63) == 0) red[tid >> 6] = M;
    __syncthreads();
    M = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    // a split without any source has l = 0; its sums may not have been written
    const float f = l == 0.0f ? 0.0f : at_exp2(m - (M == -INFINITY ? 0.0f : M));
    w[tid] = f;
    float L = f * l;
    for (int o = 32; o; o >>= 1) L += __shfl_xor(L, o);
    __syncthreads();
    if ((tid & 63) == 0) red[tid >> 6] = L;
    __syncthreads();
    L = (red[0] + red[1]) + (red[2] + red[3]);
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (4 * lane < a.D) {
#pragma unroll 4
        for (int s = grp; s < a.splits; s += kAtThreads / 32) {
            const float fs = w[s];
            if (fs == 0.0f) continue;
            const float4 x = *reinterpret_cast<const float4*>(a.part + (first + s * (int64_t)a.rows) * a.Dp + 4 * lane);
            v.x += fs * x.x; v.y += fs * x.y; v.z += fs * x.z; v.w += fs * x.w;
        }
    }
    sum[grp][lane] = v;
    __syncthreads();
    if (tid >= a.D) return;
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < kAtThreads / 32; ++i) t += reinterpret_cast<const float*>(sum[i])[tid];
    t *= L == 0.0f ? 0.0f : 1.0f / L;
    const int g = a.Hq / a.Hkv, n = row / g;
    const int64_t b = pair / a.Hkv;
    const int h = (int)(pair - b * a.Hkv) * g + (row - n * g);
    T* op = static_cast<T*>(a.o) + b * a.ob + n * a.ol + h * a.oh;
    if constexpr (sizeof(T) == 4)
        op[tid] = t;
    else
        op[tid] = f32_to_bf16_any(t);
}

// How a call is split: QB blocks of query rows per wave, or the waves sharing
// 32 rows (qb = 0), and `splits` workgroups over the sources.
struct AttnPlan {
    int qb, rb, row_tiles, splits, Dp;      // rb: blocks of 16 shared rows of the fp32 form
    int64_t blocks;
};

constexpr int kAtCus = 256;

AttnPlan plan_attention(int64_t B, int64_t Nq, int64_t Nk, int Hq, int Hkv, int D, int dtype) {
    AttnPlan p;
    const int64_t pairs = B * Hkv, rows = Nq * (Hq / Hkv);
    const int64_t wg1 = pairs * ceil_div(rows, 128);
    p.Dp = (D + 31) / 32 * 32;
    p.splits = 1;
    p.rb = 0;
    // Parts of 128 sources and up, and the launch that joins them, past 512 sources (2 x 12 heads of 64 over 722, fp32:
    // 10.1 us in parts of 128, 12.1 of 256, 14.3 of 512; 3 x 12 queries over 486, bf16: 9.1 us whole, 9.9 in parts of 128).
    auto splits = [&](int64_t wg) {
        return Nk <= 512 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(kAtMaxSplits / wg, ceil_div(Nk, 128)));
    };
    // Two blocks a wave read the sources' operands half as often (64 channels: 652 -> 608 us for 4 x 16384 over 4096, 8
    // heads) but above 64 channels leave one wave a SIMD (128: 1080 -> 1260 us).  Below a workgroup for most compute
    // units, waves that share 32 rows and split the sources finish sooner (1 x 1024 over 1024, 8 heads of 64: 12 us
    // instead of 22); in fp32, whose shared form is the slower instruction, only for few rows (4 x 349 over 10357, 4
    // heads on 2, of 24: 74 us with rows of their own, 229 shared).  Up to 32 rows, one shared tile, share it however many
    // clouds and heads there are: three waves of four would have no rows (32 x 1 over 4096, 8 heads of 128: fp32 417 us
    // with rows of their own, 179 shared, bf16 104 and 102; 32 x 32 over 2048, 8 heads of 64: 98 and 59, 36 and 26; the
    // other way about 64 x 1 over 1024 of 128 in bf16, 46 and 50; and past 32 rows fp32 64 x 64 over 257 of 32, 22 and 32).
    if (rows <= 32)
        p.qb = 0;
    else if (dtype == MESORASI_BF16 && D <= 64 && pairs * ceil_div(rows, 256) >= 2 * kAtCus)
        p.qb = 2;
    else if (wg1 >= kAtCus * 3 / 4 || (dtype == MESORASI_F32 && rows > 64))
        p.qb = 1;
    else
        p.qb = 0;
    int tile = 128 * p.qb;
    if (p.qb == 0) {
        if (dtype == MESORASI_F32) p.rb = rows <= 16 ? 1 : 2;
        tile = p.rb == 1 ? 16 : 32;
    }
    p.row_tiles = (int)ceil_div(rows, tile);
    const int64_t wg = pairs * p.row_tiles;
    if (p.qb < 2) p.splits = splits(wg);
    p.blocks = wg * p.splits;
    return p;
}

size_t attention_ws(const AttnPlan& p, int64_t rows, int64_t pairs) {
    return p.splits > 1 ? (size_t)(pairs * p.splits * rows * (p.Dp + 2)) * 4 : 0;
}

template <int DB, int QB, bool KS, bool GEN>
int launch_attention_bf16(const AttnArgs& a, unsigned grid, hipStream_t s) {
    constexpr int CH = DB == 1 ? 4 : DB == 2 ? 8 : 16;
    constexpr int tiles = 2 * 2 * (KS ? 128 : 64) * CH * 16;
    constexpr int join = KS ? 4 * 32 * DB * 32 * 4 + 2 * 128 * 4 : 0;
    constexpr int bytes = tiles > join ? tiles : join;
    static const hipError_t attr =
        hipFuncSetAttribute(reinterpret_cast<const void*>(&attention_bf16_kernel<DB, QB, KS, GEN>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    MESO_REQUIRE(attr == hipSuccess, MESORASI_EHIP, "mesorasi_cross_attention: LDS size attribute: %s",
                 hipGetErrorString(attr));
    attention_bf16_kernel<DB, QB, KS, GEN><<<dim3(grid), dim3(kAtThreads), bytes, s>>>(a);
    return MESORASI_OK;
}

template <int DB, bool GEN>
int launch_attention_bf16(const AttnArgs& a, int qb, unsigned grid, hipStream_t s) {
    if constexpr (DB <= 2)
        if (qb == 2) return launch_attention_bf16<DB, 2, false, GEN>(a, grid, s);
    if (qb == 1) return launch_attention_bf16<DB, 1, false, GEN>(a, grid, s);
    return launch_attention_bf16<DB, 1, true, GEN>(a, grid, s);
}

template <bool GEN>
int launch_attention_bf16(const AttnArgs& a, int qb, unsigned grid, hipStream_t s) {
    switch ((a.D + 31) / 32) {
        case 1: return launch_attention_bf16<1, GEN>(a, qb, grid, s);
        case 2: return launch_attention_bf16<2, GEN>(a, qb, grid, s);
        case 3: return launch_attention_bf16<3, GEN>(a, qb, grid, s);
        default: return launch_attention_bf16<4, GEN>(a, qb, grid, s);
    }
}

template <int DB, bool GEN>
int launch_attention_f32(const AttnArgs& a, unsigned grid, hipStream_t s) {
    using P = AtF32<DB>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&attention_f32_kernel<DB, GEN>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, P::kLds);
    MESO_REQUIRE(attr == hipSuccess, MESORASI_EHIP, "mesorasi_cross_attention: LDS size attribute: %s",
                 hipGetErrorString(attr));
    attention_f32_kernel<DB, GEN><<<dim3(grid), dim3(kAtThreads), P::kLds, s>>>(a);
    return MESORASI_OK;
}

template <int DQ, int RB, bool GEN>
int launch_attention_f32_few(const AttnArgs& a, unsigned grid, hipStream_t s) {
    constexpr int bytes = kAtThreads / 64 * (64 * DQ + 2) * 16 * RB * 4;
    static const hipError_t attr =
        hipFuncSetAttribute(reinterpret_cast<const void*>(&attention_f32_few_kernel<DQ, RB, GEN>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    MESO_REQUIRE(attr == hipSuccess, MESORASI_EHIP, "mesorasi_cross_attention: LDS size attribute: %s",
                 hipGetErrorString(attr));
    attention_f32_few_kernel<DQ, RB, GEN><<<dim3(grid), dim3(kAtThreads), bytes, s>>>(a);
    return MESORASI_OK;
}

template <bool GEN>
int launch_attention_f32(const AttnArgs& a, const AttnPlan& p, unsigned grid, hipStream_t s) {
    if (p.qb == 0) {
        if (a.D <= 64)
            return p.rb == 1 ? launch_attention_f32_few<1, 1, GEN>(a, grid, s) : launch_attention_f32_few<1, 2, GEN>(a, grid, s);
        return p.rb == 1 ? launch_attention_f32_few<2, 1, GEN>(a, grid, s) : launch_attention_f32_few<2, 2, GEN>(a, grid, s);
    }
    switch ((a.D + 31) / 32) {
        case 1: return launch_attention_f32<1, GEN>(a, grid, s);
        case 2: return launch_attention_f32<2, GEN>(a, grid, s);
        case 3: return launch_attention_f32<3, GEN>(a, grid, s);
        default: return launch_attention_f32<4, GEN>(a, grid, s);
    }
}

}  // namespace

}  // namespace meso

using namespace meso;

extern "C" size_t mesorasi_cross_attention_workspace(int64_t B, int64_t Nq, int64_t Nk, int32_t Hq, int32_t Hkv,
                                                     int32_t D, int32_t dtype) {
    if (B < 1 || Nq < 1 || Nk < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || D < 1 || D > MESORASI_MAX_D_ATTN ||
        Nk > 0x7fffffff - 1023 || Nq > (0x7fffffff - 1023) / (Hq / Hkv) || B > 0x7fffffff / Hkv)
        return 0;
    if (dtype != MESORASI_BF16 && dtype != MESORASI_F32) return 0;
    return attention_ws(plan_attention(B, Nq, Nk, Hq, Hkv, D, dtype), Nq * (Hq / Hkv), B * Hkv);
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
    MESO_REQUIRE(!k_mask || B <= 1 || mask_ld == 0 || mask_ld >= Nk, MESORASI_EINVAL, "mesorasi_cross_attention: mask_ld < Nk");
    MESO_REQUIRE(std::isfinite(scale * 1.4426951f), MESORASI_EINVAL, "mesorasi_cross_attention: scale = %g", (double)scale);
    MESO_REQUIRE(dtype == MESORASI_F32 || dtype == MESORASI_BF16, MESORASI_EUNSUPPORTED,
                 "mesorasi_cross_attention: dtype %d", dtype);
    MESO_REQUIRE(D <= MESORASI_MAX_D_ATTN, MESORASI_EUNSUPPORTED, "mesorasi_cross_attention: D = %d", D);
    MESO_REQUIRE(Nk <= 0x7fffffff - 1023 && Nq <= (0x7fffffff - 1023) / (Hq / Hkv), MESORASI_EUNSUPPORTED,
                 "mesorasi_cross_attention: Nq = %lld, Nk = %lld", (long long)Nq, (long long)Nk);
    if (B == 0 || Nq == 0) return MESORASI_OK;
    MESO_REQUIRE(q && o && (Nk == 0 || (k && v)), MESORASI_EINVAL, "mesorasi_cross_attention: NULL q, k, v or o");
    MESO_REQUIRE(B <= 0x7fffffff / Hkv, MESORASI_EUNSUPPORTED, "mesorasi_cross_attention: B = %lld", (long long)B);
    AttnArgs a = {q, k, v, o, q_bs, q_ld, q_hs, k_bs, k_ld, k_hs, v_bs, v_ld, v_hs, o_bs, o_ld, o_hs,
                  Nq, Nk, mask_ld, Hq, Hkv, D, scale, k_len, k_mask};
    hipStream_t s = as_stream(stream);
    const AttnPlan p = plan_attention(B, Nq, Nk, Hq, Hkv, D, dtype);
    const int64_t pairs = B * Hkv;
    a.rows = (int)(Nq * (Hq / Hkv));
    const size_t need = attention_ws(p, a.rows, pairs);
    MESO_REQUIRE(need == 0 || (ws && ws_bytes >= need), MESORASI_EWORKSPACE,
                 "mesorasi_cross_attention: workspace %zu < %zu bytes", ws ? ws_bytes : (size_t)0, need);
    MESO_REQUIRE(need == 0 || aligned(ws, 16), MESORASI_EINVAL, "mesorasi_cross_attention: ws is not 16-byte aligned");
    a.row_tiles = p.row_tiles;
    a.splits = p.splits;
    a.blocks = p.blocks;
    a.Dp = p.Dp;
    a.part = p.splits > 1 ? static_cast<float*>(ws) : nullptr;
    const int64_t per = ceil_div(p.blocks, 8);
    MESO_REQUIRE(launch_fits(8 * per, kAtThreads), MESORASI_EUNSUPPORTED, "mesorasi_cross_attention: %lld workgroups",
                 (long long)p.blocks);
    a.per_xcd = (int)per;
    const int elem = dtype == MESORASI_F32 ? 4 : 2;
    auto extent = [&](const void* t, int64_t n, int64_t heads, int64_t bs, int64_t ld, int64_t hs) {
        return Extent{t, (int64_t)D * elem, {B, n, heads}, {bs * elem, ld * elem, hs * elem}};
    };
    const Extent ext = extent(o, Nq, Hq, o_bs, o_ld, o_hs);
    MESO_REQUIRE(!overlap(ext, extent(q, Nq, Hq, q_bs, q_ld, q_hs)) && !overlap(ext, extent(k, Nk, Hkv, k_bs, k_ld, k_hs)) &&
                     !overlap(ext, extent(v, Nk, Hkv, v_bs, v_ld, v_hs)),
                 MESORASI_EINVAL, "mesorasi_cross_attention: o overlaps q, k or v");
    // 16-byte pieces of every row, runs of 4 channels of the output
    const bool f32 = dtype == MESORASI_F32;
    const int64_t st = q_bs | q_ld | q_hs | k_bs | k_ld | k_hs | v_bs | v_ld | v_hs | D;
    const bool vec = st % (f32 ? 4 : 8) == 0 && (o_bs | o_ld | o_hs) % 4 == 0 && aligned(q, 16) && aligned(k, 16) &&
                     aligned(v, 16) && aligned(o, f32 ? 16 : 8);
    const unsigned grid = (unsigned)(8 * per);
    const int rc = f32 ? (vec ? launch_attention_f32<false>(a, p, grid, s) : launch_attention_f32<true>(a, p, grid, s))
                       : (vec ? launch_attention_bf16<false>(a, p.qb, grid, s)
                              : launch_attention_bf16<true>(a, p.qb, grid, s));
    if (rc != MESORASI_OK) return rc;
    if (p.splits > 1) {
        const dim3 jgrid((unsigned)(pairs * a.rows)), block(kAtThreads);
        if (f32)
            attention_join_kernel<float><<<jgrid, block, 0, s>>>(a);
        else
            attention_join_kernel<uint16_t><<<jgrid, block, 0, s>>>(a);
    }
    return after_launch("mesorasi_cross_attention");
}
