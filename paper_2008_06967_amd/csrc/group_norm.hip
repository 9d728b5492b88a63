// Group normalisation with an activation, channels last.
//
// Mean and variance are joined from parts, each (count, mean, sum of squared
// differences to that mean), so that nothing cancels.  A mean is a sum of two
// floats, the second what the first's rounding leaves, and every join takes
// differences to a first estimate of the mean and corrects it by their own mean:
// so neither an offset of the data nor single values far from the others cost
// the others accuracy, wherever they stand.  Parts are joined in a fixed order.
//
// Two forms.  Where the rows of a run of whole groups fit the registers of
// one workgroup, it reads them once, and one launch does all.  Otherwise one
// launch forms the parts of chunks of rows and another joins them and
// writes; its writes pass the caches by, which leaves them to x (138 us
// instead of 167 for 16 x 16384 x 256 in fp32, gelu, the same x repeated).
//
// Bound: one read and one write of HBM, and a second read where x is larger
// than the caches (16 x 16384 x 256 fp32: 43 + 100 us, 6.3 and 5.4 TB/s).  The
// small form is bound by its chain of loads, two sums over the workgroup and
// stores (16 x 1023 x 192 bf16: 12.9 us, 128 x 128: 5.3).
#include <algorithm>
#include <cmath>

#include "common.h"

namespace meso {

namespace {

constexpr int kGnThreads = 256;      // of the two-launch form
constexpr int kGnOneThreads = 512;   // of the one-launch form
constexpr int kGnKeep = 16;          // vectors of a thread in the one-launch form, at most
constexpr int kGnBlocks = 1024;      // workgroups of the two-launch form: four a compute unit (2048: 157 us for 136)

template <typename T, int N>
struct alignas(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) GnVec {
    T e[N];
};

// Mean (hi + lo, hi the nearest float) and sum of squared differences to it.
struct GnPart {
    float hi, lo, m2;
};

struct GnArgs {
    const void* x;
    void* y;
    const int32_t* lens;
    const float* gamma;
    const float* beta;
    GnPart* part;                    // [B, chunks, groups, pieces]
    int64_t ldx, ldy, B, N;
    int C, G, c;
    float eps;
    int act;
    int slab;                        // channels of a workgroup: whole groups, or a piece of one
    int slabs, pieces;               // slabs of a row; slabs of a group (1: whole groups in a slab)
    int chunks;
    int64_t chunk_rows;
    int blocks, per_xcd;             // workgroups; of an XCD, in the one-launch form
    FastDiv by_chunks, by_slabs, by_pieces, by_c;
    FastDiv by_rows;                 // rows of a chunk
    FastDiv by_nv;                   // vectors of a full slab
};

__device__ __forceinline__ float gn_float(float v) { return v; }
__device__ __forceinline__ float gn_float(uint16_t v) { return bf16_to_f32(v); }

template <typename T>
__device__ __forceinline__ T gn_round(float v) {
    if constexpr (sizeof(T) == 4)
        return v;
    else
        return f32_to_bf16_any(v);
}

// erfc(z), z >= 0, as 2 to a polynomial: a least-maximum fit of log2(erfc) on
// [0, 4] weighted for z erfc(z) (within 5e-8 in fp32); past 4 it falls faster
// than log2(erfc), where z erfc(z) is below 7e-8.
__device__ __forceinline__ float gn_erfc(float z) {
    float p = -1.7592439007785288e-06f;
    p = fmaf(p, z, 3.0905426683602855e-05f);
    p = fmaf(p, z, -0.00024038320407271385f);
    p = fmaf(p, z, 0.0010606396244838834f);
    p = fmaf(p, z, -0.002575934398919344f);
    p = fmaf(p, z, 0.00033866698504425585f);
    p = fmaf(p, z, 0.02760038711130619f);
    p = fmaf(p, z, -0.14827527105808258f);
    p = fmaf(p, z, -0.9184468388557434f);
    p = fmaf(p, z, -1.627907156944275f);
    return __builtin_amdgcn_exp2f(p * z);
}

// A store that passes the caches by.
template <typename T, int N>
__device__ __forceinline__ void gn_store(T* p, const GnVec<T, N>& v) {
    if constexpr (sizeof(T) * N >= 4) {
        typedef uint32_t words __attribute__((ext_vector_type(sizeof(T) * N >= 16 ? 4 : sizeof(T) * N / 4)));
        const words* w = reinterpret_cast<const words*>(&v);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) * N / sizeof(words)); ++i)
            __builtin_nontemporal_store(w[i], reinterpret_cast<words*>(p) + i);
    } else {
        __builtin_nontemporal_store(v.e[0], p);
    }
}

template <int ACT>
__device__ __forceinline__ float gn_act(float v) {
    if constexpr (ACT == MESORASI_ACT_RELU) return v < 0.0f ? 0.0f : v;
    if constexpr (ACT == MESORASI_ACT_SILU)
        return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504f));
    if constexpr (ACT == MESORASI_ACT_GELU) {
        const float e = gn_erfc(fabsf(v) * 0.70710678f);
        return 0.5f * v * (v < 0.0f ? e : 2.0f - e);
    }
    return v;
}

// Lanes that share a group's parts: all threads at work at once, at most a wave for a group.
template <int THREADS>
__device__ __forceinline__ int gn_lanes(int groups, int parts) {
    int w = 1;
    while (w < 64 && w < parts && 2 * w * groups <= THREADS) w *= 2;
    return __builtin_amdgcn_readfirstlane(w);
}

// a + b as the nearest float and what it leaves (Knuth's two-sum).
__device__ __forceinline__ void gn_two_sum(float a, float b, float& hi, float& lo) {
    hi = a + b;
    const float t = hi - a;
    lo = (a - (hi - t)) + (b - t);
}

// v, or 0 where roundings left less; NaN stays.
__device__ __forceinline__ float gn_positive(float v) { return v < 0.0f ? 0.0f : v; }

__device__ __forceinline__ float gn_diff(const GnPart& a, const GnPart& b) { return (a.hi - b.hi) + (a.lo - b.lo); }

// m's mean moved by d.
__device__ __forceinline__ void gn_move(GnPart& m, float d) { gn_two_sum(m.hi, m.lo + d, m.hi, m.lo); }

// The groups' parts in LDS, joined: part (s, e), e < per, of a group counts
// n(s) values and is get(g, s, e); put(g, part) takes the result.
template <int THREADS, typename Count, typename Get, typename Put>
__device__ __forceinline__ void gn_join(int groups, int slots, int per, Count n, Get get, Put put) {
    const int w = gn_lanes<THREADS>(groups, slots * per);
    int we = 1;
    while (we < w && we < per) we *= 2;
    const int lw = __builtin_ctz(w), le = __builtin_ctz(we);
    const int lane = threadIdx.x & (w - 1), ws = w >> le, s0 = lane >> le, e0 = lane & (we - 1);
    for (int g = threadIdx.x >> lw; g < groups; g += THREADS >> lw) {
        GnPart m = get(g, 0, 0);
        float cnt = 0.0f, sum = 0.0f;
        for (int s = s0; s < slots; s += ws)
            for (int e = e0; e < per; e += we) {
                const float k = n(s);
                cnt += k;
                sum += k * gn_diff(get(g, s, e), m);
            }
        cnt = lane_sum(cnt, w);
        gn_move(m, lane_sum(sum, w) / cnt);
        float m2 = 0.0f;
        sum = 0.0f;
        for (int s = s0; s < slots; s += ws)
            for (int e = e0; e < per; e += we) {
                const GnPart v = get(g, s, e);
                const float t = gn_diff(v, m), nt = n(s) * t;
                sum += nt;
                m2 += v.m2 + nt * t;
            }
        sum = lane_sum(sum, w);
        m2 = lane_sum(m2, w);
        const float d = sum / cnt;
        gn_move(m, d);
        m.m2 = gn_positive(m2 - sum * d);
        if (lane == 0) put(g, m);
    }
}

// A workgroup's place: cloud, slab, valid rows, and each thread's vector of
// channels and rows.
template <int THREADS, int VEC>
struct GnPlace {
    int64_t b, len;
    int slab, ch0, width, slots, slot, vec, first, groups;
    bool on;
    __device__ GnPlace(const GnArgs& a, int blk) {     // cloud and slab
        b = a.by_slabs.div(blk, slab);
        len = a.lens ? min(max((int64_t)a.lens[b], (int64_t)0), a.N) : a.N;
        if (a.pieces > 1) {
            int piece;
            first = a.by_pieces.div(slab, piece);
            ch0 = first * a.c + piece * a.slab;
            width = min(a.slab, a.c - piece * a.slab);
            groups = 1;
        } else {
            ch0 = slab * a.slab;
            width = min(a.slab, a.C - ch0);
            first = a.by_c.div(ch0);
            groups = a.by_c.div(width);
        }
        // a narrower slab leaves lanes of a row without work
        slots = THREADS / (int)a.by_nv.d;
        slot = a.by_nv.div(threadIdx.x, vec);
        on = slot < slots && vec * VEC < width;
    }
    // the groups, within the slab, of the thread's channels
    __device__ void channel_groups(const GnArgs& a, int (&g)[VEC]) const {
        int n = 0, r = 0;
        if (on && a.pieces == 1) {
            n = a.by_c.div(vec * VEC, r);
        }
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            g[k] = n;
            if (++r == a.c && a.pieces == 1) {
                ++n;
                r = 0;
            }
        }
    }
};

// A thread's channels: their groups, gamma and beta, and what is taken from
// their values (the group's first value, then its mean).
template <int VEC>
struct GnChannels {
    int grp[VEC];
    float ref[VEC], gamma[VEC], beta[VEC];
};

template <typename TX, int VEC, typename P>
__device__ __forceinline__ void gn_channels(const GnArgs& a, const P& p, GnChannels<VEC>& c) {
    // the one-launch form's first estimate of a group's mean is taken from its first value on
    const TX* x0 = static_cast<const TX*>(a.x) + p.b * a.N * a.ldx + (int64_t)p.first * a.c;
    p.channel_groups(a, c.grp);
#pragma unroll
    for (int k = 0; k < VEC; ++k) c.ref[k] = 0.0f;
    if (p.on && p.len > 0)
#pragma unroll
        for (int k = 0; k < VEC; ++k) c.ref[k] = gn_float(x0[c.grp[k] * a.c]);
}

template <int VEC, typename P>
__device__ __forceinline__ void gn_affine(const GnArgs& a, const P& p, GnChannels<VEC>& c) {
    const int ch = p.ch0 + p.vec * VEC;
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        c.gamma[k] = 1.0f;
        c.beta[k] = 0.0f;
    }
    if (p.on && a.gamma)
#pragma unroll
        for (int k = 0; k < VEC; ++k) c.gamma[k] = a.gamma[ch + k];
    if (p.on && a.beta)
#pragma unroll
        for (int k = 0; k < VEC; ++k) c.beta[k] = a.beta[ch + k];
}

// The thread's channels' parts to LDS: channels of one group join at once.
template <int VEC>
__device__ __forceinline__ void gn_put_parts(bool merged, float n, const GnPart (&c)[VEC], GnPart* ent) {
    if (!merged) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) ent[k] = c[k];
        return;
    }
    float d = 0.0f, q = 0.0f;
#pragma unroll
    for (int k = 1; k < VEC; ++k) d += gn_diff(c[k], c[0]);
    d *= 1.0f / VEC;
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        const float t = gn_diff(c[k], c[0]) - d;
        q += c[k].m2 + n * t * t;
    }
    GnPart m = c[0];
    gn_move(m, d);
    m.m2 = q;
    *ent = m;
}

template <typename TX, int VEC>
__global__ __launch_bounds__(kGnThreads) void gn_parts_kernel(GnArgs a) {
    __shared__ GnPart ent[kGnThreads * VEC];
    int chunk;
    const int rest = a.by_chunks.div((int)blockIdx.x, chunk);
    const GnPlace<kGnThreads, VEC> p(a, rest);
    const int64_t r0 = chunk * a.chunk_rows, r1 = min(p.len, r0 + a.chunk_rows);
    if (r0 >= r1) return;                        // no valid row: the join knows
    const int nrows = (int)(r1 - r0);
    const bool merged = a.pieces > 1 || a.c % VEC == 0;
    float sum[VEC] = {}, sq[VEC] = {}, f[VEC] = {};
    GnPart part[VEC] = {};
    const int full = nrows / p.slots, tail = nrows - full * p.slots;      // rows of every slot, slots with one more
    const int mine = p.on ? full + (p.slot < tail) : 0;
    if (mine > 0) {
        const TX* xp = static_cast<const TX*>(a.x) + (p.b * a.N + r0 + p.slot) * a.ldx + p.ch0 + p.vec * VEC;
        const int64_t step = (int64_t)p.slots * a.ldx;
        // The differences are taken to the median of a channel's first three values: to one far from the others they
        // would all be rounded as coarsely as it, and so would their sum.
        GnVec<TX, VEC> w[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) w[i] = *reinterpret_cast<const GnVec<TX, VEC>*>(xp + min(i, mine - 1) * step);
#pragma unroll
        for (int k = 0; k < VEC; ++k)
            f[k] = __builtin_amdgcn_fmed3f(gn_float(w[0].e[k]), gn_float(w[1].e[k]), gn_float(w[2].e[k]));
        auto add = [&](const GnVec<TX, VEC>& v) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                const float d = gn_float(v.e[k]) - f[k];
                sum[k] += d;
                sq[k] = fmaf(d, d, sq[k]);
            }
        };
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < mine) add(w[i]);
#pragma unroll 4
        for (int i = 3; i < mine; ++i) add(*reinterpret_cast<const GnVec<TX, VEC>*>(xp + i * step));
        const float n = (float)mine;
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const float d = sum[k] / n;
            gn_two_sum(f[k], d, part[k].hi, part[k].lo);
            part[k].m2 = gn_positive(sq[k] - sum[k] * d);
        }
    }
    const int nv = (int)a.by_nv.d;
    if (p.on) gn_put_parts<VEC>(merged, (float)mine, part, ent + (p.slot * nv + p.vec) * (merged ? 1 : VEC));
    __syncthreads();
    const int per_slot = merged ? nv : nv * VEC;             // parts of a slot
    const int per = merged ? (a.pieces > 1 ? p.width : a.c) / VEC : a.c;   // of them, a group's
    const float each = merged ? (float)VEC : 1.0f;
    const int groups_all = a.G * a.pieces;
    GnPart* out = a.part + (p.b * a.chunks + chunk) * groups_all +
                  (a.pieces > 1 ? p.slab : p.first);
    gn_join<kGnThreads>(
        p.groups, min(p.slots, nrows), per,
        [&](int s) { return (float)(s < tail ? full + 1 : full) * each; },
        [&](int g, int s, int e) { return ent[s * per_slot + g * per + e]; },
        [&](int g, const GnPart& m) { out[g] = m; });
}

// y = act((x - hi) A + S): A = gamma / sqrt(var + eps), S = beta - lo A, from the
// mean hi + lo and st = (lo, 1 / sqrt(var + eps)).
__device__ __forceinline__ void gn_factor(float2 st, float gamma, float beta, float& A, float& S) {
    A = st.y * gamma;
    S = fmaf(-st.x, A, beta);
}

// The cloud's parts in memory, joined: (lo, 1 / deviation) and hi of the slab's
// groups.  The first kGnBatch parts of a lane are all on their way at once.
constexpr int kGnBatch = 8;

template <typename P>
__device__ __forceinline__ void gn_join_chunks(const GnArgs& a, const P& p, float2* stat, float* hi) {
    const int groups_all = a.G * a.pieces;
    const int used = a.by_rows.div((int)p.len - 1) + 1, total = used * a.pieces;
    const int w = gn_lanes<kGnThreads>(p.groups, total);
    const int lane = threadIdx.x & (w - 1), lw = __builtin_ctz(w);
    for (int g = threadIdx.x >> lw; g < p.groups; g += kGnThreads >> lw) {
        const GnPart* in = a.part + p.b * a.chunks * groups_all + (p.first + g) * a.pieces;
        auto get = [&](int i) {
            const int chunk = a.pieces > 1 ? a.by_pieces.div(i) : i;
            return in[(int64_t)chunk * groups_all + (i - chunk * a.pieces)];
        };
        auto count = [&](int i) {
            const int chunk = a.pieces > 1 ? a.by_pieces.div(i) : i, piece = i - chunk * a.pieces;
            const int width = a.pieces > 1 ? min(a.slab, a.c - piece * a.slab) : a.c;
            return (float)min(a.chunk_rows, p.len - chunk * a.chunk_rows) * (float)width;
        };
        GnPart keep[kGnBatch];
#pragma unroll
        for (int k = 0; k < kGnBatch; ++k) keep[k] = get(min(lane + k * w, total - 1));
        GnPart m = get(0);
        float cnt = 0.0f, sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kGnBatch; ++k)
            if (lane + k * w < total) {
                const float n = count(lane + k * w);
                cnt += n;
                sum += n * gn_diff(keep[k], m);
            }
        for (int i = lane + kGnBatch * w; i < total; i += w) {
            const float n = count(i);
            cnt += n;
            sum += n * gn_diff(get(i), m);
        }
        cnt = lane_sum(cnt, w);
        gn_move(m, lane_sum(sum, w) / cnt);
        float m2 = 0.0f;
        sum = 0.0f;
        auto add = [&](const GnPart& v, float n) {
            const float t = gn_diff(v, m), nt = n * t;
            sum += nt;
            m2 += v.m2 + nt * t;
        };
#pragma unroll
        for (int k = 0; k < kGnBatch; ++k)
            if (lane + k * w < total) add(keep[k], count(lane + k * w));
        for (int i = lane + kGnBatch * w; i < total; i += w) add(get(i), count(i));
        sum = lane_sum(sum, w);
        m2 = lane_sum(m2, w);
        const float d = sum / cnt, var = gn_positive(m2 - sum * d) / cnt;
        gn_move(m, d);
        if (lane == 0) {
            stat[g] = make_float2(m.lo, 1.0f / sqrtf(var + a.eps));
            hi[g] = m.hi;
        }
    }
}

template <typename TX, typename TY, int VEC, int ACT>
__global__ __launch_bounds__(kGnThreads) void gn_apply_kernel(GnArgs a) {
    __shared__ float2 stat[kGnThreads * VEC];    // a slab's groups: at most its channels
    __shared__ float hi[kGnThreads * VEC];
    int chunk;
    const int rest = a.by_chunks.div((int)blockIdx.x, chunk);
    const GnPlace<kGnThreads, VEC> p(a, rest);
    const int64_t r0 = chunk * a.chunk_rows, r1 = min(a.N, r0 + a.chunk_rows);
    GnChannels<VEC> c;
    float A[VEC] = {}, S[VEC] = {};
    if (r0 < p.len) {
        p.channel_groups(a, c.grp);
        gn_affine<VEC>(a, p, c);
        gn_join_chunks(a, p, stat, hi);
        __syncthreads();
        if (p.on) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                c.ref[k] = hi[c.grp[k]];
                gn_factor(stat[c.grp[k]], c.gamma[k], c.beta[k], A[k], S[k]);
            }
        }
    }
    if (!p.on) return;
    const TX* __restrict__ xp = static_cast<const TX*>(a.x) + p.b * a.N * a.ldx + p.ch0 + p.vec * VEC;
    TY* __restrict__ yp = static_cast<TY*>(a.y) + p.b * a.N * a.ldy + p.ch0 + p.vec * VEC;
    const int64_t valid = min(r1, p.len);
    int64_t r = r0 + p.slot;
#pragma unroll 4
    for (; r < valid; r += p.slots) {
        const GnVec<TX, VEC> w = *reinterpret_cast<const GnVec<TX, VEC>*>(xp + r * a.ldx);
        GnVec<TY, VEC> o;
#pragma unroll
        for (int k = 0; k < VEC; ++k) o.e[k] = gn_round<TY>(gn_act<ACT>(fmaf(gn_float(w.e[k]) - c.ref[k], A[k], S[k])));
        gn_store(yp + r * a.ldy, o);
    }
    for (; r < r1; r += p.slots) gn_store(yp + r * a.ldy, GnVec<TY, VEC>{});
}

// Sums over the workgroup of each group's values (one or two of each channel),
// finished once a group: a thread's per channel, or of its channels in one
// group where a vector lies in one or at most two; then over the rows of its
// wave, then over waves and entries.  nvp lanes (a power of two) hold a row: a
// wave several rows, or a row several waves.
template <int VEC, int VALUES, typename P, typename Finish>
__device__ __forceinline__ void gn_group_sums(const GnArgs& a, const P& p, int nvp, const int (&grp)[VEC],
                                              float (&v)[VALUES][VEC], float* ent, Finish finish) {
    struct alignas(4 * VALUES) Entry {
        float e[VALUES];
    };
    Entry* at = reinterpret_cast<Entry*>(ent);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    // entries of a vector: its groups, or its channels.  Vectors start at multiples of gcd(c, VEC) in their first group.
    const int low = a.c & -a.c, gcd = low < VEC ? low : VEC;
    const int units = VEC == 1 || gcd == VEC ? 1 : VEC - gcd <= a.c ? 2 : VEC;
    if (VEC > 1 && units <= 2) {
#pragma unroll
        for (int i = 0; i < VALUES; ++i) {
            float s0 = v[i][0], s1 = 0.0f;
            if (units == 1) {
#pragma unroll
                for (int k = 1; k < VEC; ++k) s0 += v[i][k];
            } else {
#pragma unroll
                for (int k = 1; k < VEC; ++k) {
                    s0 += grp[k] == grp[0] ? v[i][k] : 0.0f;
                    s1 += grp[k] == grp[0] ? 0.0f : v[i][k];
                }
                v[i][VEC > 1 ? 1 : 0] = wave_sum_from(s1, nvp);
            }
            v[i][0] = wave_sum_from(s0, nvp);
        }
    } else {
#pragma unroll
        for (int i = 0; i < VALUES; ++i)
#pragma unroll
            for (int k = 0; k < VEC; ++k) v[i][k] = wave_sum_from(v[i][k], nvp);
    }
    const int slots = nvp <= 64 ? kGnOneThreads / 64 : p.slots, row = (int)a.by_nv.d * units;
    const int slot = nvp <= 64 ? wave : p.slot;
    __syncthreads();
    if (p.vec * VEC < p.width && (nvp > 64 || lane < nvp))
#pragma unroll
        for (int k = 0; k < VEC; ++k)
            if (k < units) {
                Entry t;
#pragma unroll
                for (int i = 0; i < VALUES; ++i) t.e[i] = v[i][k];
                at[slot * row + p.vec * units + k] = t;
            }
    __syncthreads();
    const int most = units == 1 ? a.c / VEC : units == 2 ? (a.c + VEC - 2) / VEC + 1 : a.c;      // entries of a group
    const int w = gn_lanes<kGnOneThreads>(p.groups, slots * most);
    int we = 1;
    while (we < w && we < most) we *= 2;
    const int lw = __builtin_ctz(w), le = __builtin_ctz(we);
    const int l = threadIdx.x & (w - 1), ws = w >> le, s0 = l >> le, e0 = l & (we - 1);
    for (int g = threadIdx.x >> lw; g < p.groups; g += kGnOneThreads >> lw) {
        float sum[VALUES] = {};
        const int first = g * a.c / VEC, per = units == 2 ? (g * a.c + a.c - 1) / VEC - first + 1 : most;
        for (int s = s0; s < slots; s += ws)
            for (int e = e0; e < per; e += we) {
                const int in = units == 2 ? 2 * (first + e) + (a.by_c.div((first + e) * VEC) != g) : g * most + e;
                const Entry t = at[s * row + in];
#pragma unroll
                for (int i = 0; i < VALUES; ++i) sum[i] += t.e[i];
            }
#pragma unroll
        for (int i = 0; i < VALUES; ++i) sum[i] = lane_sum(sum[i], w);
        if (l == 0) finish(g, sum);
    }
    __syncthreads();
}

// Packed rows stay packed: what one pass unpacked is not kept for the next.
template <typename T, int N>
__device__ __forceinline__ void gn_keep(GnVec<T, N>& v) {
    if constexpr (sizeof(T) == 2 && N == 8) {
        uint4& r = reinterpret_cast<uint4&>(v);
        asm volatile("" : "+v"(r.x), "+v"(r.y), "+v"(r.z), "+v"(r.w));
    }
}

// One launch: the slab's valid rows stay in registers between the
// statistics and the output.  The first sums estimate the mean, the second ones
// are of differences to that estimate: their mean corrects it, their squares
// give the variance.
template <typename TX, typename TY, int VEC, int ACT, int KEEP>
__global__ __launch_bounds__(kGnOneThreads) void gn_one_kernel(GnArgs a) {
    __shared__ float ent[2 * kGnOneThreads * VEC];   // [slots][width], at most two values for each thread and channel
    __shared__ float2 sums[16 * VEC];    // a slab's groups: at most VEC, or the channels of 16 vectors (the plan)
    const int nv = (int)a.by_nv.d;
    const int shift = nv > 1 ? 32 - __builtin_clz(nv - 1) : 0, nvp = 1 << shift;     // lanes of a row
    // a cloud's slabs share lines of its rows: they go to one XCD
    const int blk = (int)(blockIdx.x & 7) * a.per_xcd + (int)(blockIdx.x >> 3);
    if (blk >= a.blocks) return;
    GnPlace<kGnOneThreads, VEC> p(a, blk);
    p.slots = kGnOneThreads >> shift;
    p.slot = threadIdx.x >> shift;
    p.vec = threadIdx.x & (nvp - 1);
    p.on = p.vec < nv;
    const int nrows = (int)p.len;
    const int mine = p.on && p.slot < nrows ? ((nrows - 1 - p.slot) >> (__builtin_ctz(kGnOneThreads) - shift)) + 1 : 0;
    const TX* __restrict__ xp = static_cast<const TX*>(a.x) + (p.b * a.N + p.slot) * a.ldx + p.ch0 + p.vec * VEC;
    TY* __restrict__ yp = static_cast<TY*>(a.y) + (p.b * a.N + p.slot) * a.ldy + p.ch0 + p.vec * VEC;
    GnChannels<VEC> c;
    gn_channels<TX, VEC>(a, p, c);
    if (KEEP < kGnKeep) gn_affine<VEC>(a, p, c);       // the long form has no registers for them yet
    GnVec<TX, VEC> w[KEEP];
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (i < mine) w[i] = *reinterpret_cast<const GnVec<TX, VEC>*>(xp + (int64_t)i * p.slots * a.ldx);
    float A[VEC] = {}, S[VEC] = {};
    if (nrows > 0) {
        const float inv = 1.0f / ((float)nrows * (float)a.c);
        float v[1][VEC] = {};
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (i < mine)
#pragma unroll
                for (int k = 0; k < VEC; ++k) v[0][k] += gn_float(w[i].e[k]) - c.ref[k];
        gn_group_sums<VEC, 1>(a, p, nvp, c.grp, v, ent, [&](int g, const float (&s)[1]) { sums[g].x = s[0] * inv; });
        float d[2][VEC] = {};
#pragma unroll
        for (int k = 0; k < VEC; ++k) c.ref[k] += sums[c.grp[k]].x;
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (i < mine) {
                gn_keep(w[i]);
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    const float t = gn_float(w[i].e[k]) - c.ref[k];
                    d[0][k] += t;
                    d[1][k] = fmaf(t, t, d[1][k]);
                }
            }
        if (KEEP == kGnKeep) gn_affine<VEC>(a, p, c);
        gn_group_sums<VEC, 2>(a, p, nvp, c.grp, d, ent, [&](int g, const float (&s)[2]) {
            const float lo = s[0] * inv, var = gn_positive(s[1] * inv - lo * lo);
            sums[g] = make_float2(lo, 1.0f / sqrtf(var + a.eps));
        });
#pragma unroll
        for (int k = 0; k < VEC; ++k) gn_factor(sums[c.grp[k]], c.gamma[k], c.beta[k], A[k], S[k]);
    }
    if (!p.on) return;
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (i < mine) {
            gn_keep(w[i]);
            GnVec<TY, VEC> o;
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                o.e[k] = gn_round<TY>(gn_act<ACT>(fmaf(gn_float(w[i].e[k]) - c.ref[k], A[k], S[k])));
            *reinterpret_cast<GnVec<TY, VEC>*>(yp + (int64_t)i * p.slots * a.ldy) = o;
        }
    for (int64_t r = (int64_t)p.slot + (int64_t)mine * p.slots; r < a.N; r += p.slots)
        *reinterpret_cast<GnVec<TY, VEC>*>(yp + (r - p.slot) * a.ldy) = GnVec<TY, VEC>{};
}

// How a call is cut.
struct GnPlan {
    int keep;            // one launch, with this many vectors a thread; 0: two launches
    int slab, slabs, pieces, chunks;
    int64_t chunk_rows;
};

int64_t gn_gcd(int64_t a, int64_t b) { return b ? gn_gcd(b, a % b) : a; }

GnPlan plan_group_norm(int64_t B, int64_t N, int C, int G, int vec) {
    GnPlan p;
    const int c = C / G;
    p.pieces = 1;
    p.chunks = 1;
    p.chunk_rows = N;
    // the shortest run of whole groups and whole vectors (C is a multiple of both)
    const int64_t base = (int64_t)c / gn_gcd(c, vec) * vec;
    const int64_t room = (int64_t)kGnOneThreads * kGnKeep;
    auto lanes = [&](int64_t slab) {         // of a row, a power of two
        int64_t n = 1;
        while (n < slab / vec) n *= 2;
        return n;
    };
    auto fits = [&](int64_t slab) {
        return lanes(slab) <= kGnOneThreads && ceil_div(N, kGnOneThreads / lanes(slab)) <= kGnKeep;
    };
    p.keep = 0;
    if (base <= C && N <= room && fits(base)) {
        // longer runs read whole lines; not past 256 bytes, nor below a workgroup for each compute unit
        int64_t slab = base;
        while (2 * slab <= C && C % (2 * slab) == 0 && 2 * slab / vec <= 16 && fits(2 * slab) &&
               B * (C / (2 * slab)) >= 256)
            slab *= 2;
        p.slab = (int)slab;
        p.slabs = (int)(C / slab);
        p.keep = ceil_div(N, kGnOneThreads / lanes(slab)) <= kGnKeep / 4 ? kGnKeep / 4 : kGnKeep;
        return p;
    }
    const int64_t most = (int64_t)kGnThreads * vec;
    if (base <= most && base <= C) {
        int64_t slab = base;
        while (slab + base <= most && slab + base <= C) slab += base;
        p.slab = (int)slab;
        p.slabs = (int)ceil_div(C, slab);
    } else {
        // a group wider than the threads' vectors, in pieces (c is then a multiple of vec, or vec is 1)
        p.slab = (int)most;
        p.pieces = (int)ceil_div(c, most);
        p.slabs = G * p.pieces;
    }
    const int64_t slots = std::max<int64_t>(1, kGnThreads / ceil_div(std::min<int64_t>(p.slab, C), vec));
    // Every workgroup of the second launch joins all chunks of its cloud, 16 parts a thread at most: 256 chunks for 8
    // groups (1 x 65536 x 64: 16 us, with 128 20), 128 for 32 (1 x 16384 x 256: 26 us, with 256 31).  A thread's chain
    // of sums stays within 128 rows; at least 8 rows a thread.
    const int64_t most_chunks = std::max<int64_t>(64, std::min<int64_t>(256, 4096 / std::max(1, p.slab / c)));
    const int64_t want = std::min(most_chunks, std::max<int64_t>(1, kGnBlocks / std::max<int64_t>(1, B * p.slabs)));
    int64_t rows = std::max<int64_t>(ceil_div(N, want), 8 * slots);
    rows = std::max<int64_t>(std::min<int64_t>(rows, 128 * slots), ceil_div(N, 4096));
    p.chunk_rows = rows;
    p.chunks = (int)ceil_div(N, rows);
    return p;
}

size_t group_norm_ws(const GnPlan& p, int64_t B, int G) {
    return p.keep ? 0 : ((size_t)(B * p.chunks * G * p.pieces) * sizeof(GnPart) + 15) / 16 * 16;
}

// Widest vector: 16 bytes of x where C allows them, else single values.
int group_norm_vec(int C, int G, int x_dtype) {
    const int vec = x_dtype == MESORASI_F32 ? 4 : 8;
    const int64_t c = C / G;
    // whole vectors in a row, and in a group, or in a run of groups within the threads' vectors
    return C % vec == 0 && (c % vec == 0 || c / gn_gcd(c, vec) <= kGnThreads) ? vec : 1;
}

template <typename TX, typename TY, int VEC, int ACT>
void launch_group_norm(const GnArgs& a, const GnPlan& p, hipStream_t s) {
    if (p.keep) {
        const dim3 grid(8u * (unsigned)a.per_xcd), block(kGnOneThreads);
        if (p.keep < kGnKeep)
            gn_one_kernel<TX, TY, VEC, ACT, kGnKeep / 4><<<grid, block, 0, s>>>(a);
        else
            gn_one_kernel<TX, TY, VEC, ACT, kGnKeep><<<grid, block, 0, s>>>(a);
        return;
    }
    gn_parts_kernel<TX, VEC><<<dim3((unsigned)a.blocks), dim3(kGnThreads), 0, s>>>(a);
    gn_apply_kernel<TX, TY, VEC, ACT><<<dim3((unsigned)a.blocks), dim3(kGnThreads), 0, s>>>(a);
}

template <typename TX, typename TY, int VEC>
void launch_group_norm(const GnArgs& a, const GnPlan& p, hipStream_t s) {
    switch (a.act) {
        case MESORASI_ACT_RELU: launch_group_norm<TX, TY, VEC, MESORASI_ACT_RELU>(a, p, s); break;
        case MESORASI_ACT_SILU: launch_group_norm<TX, TY, VEC, MESORASI_ACT_SILU>(a, p, s); break;
        case MESORASI_ACT_GELU: launch_group_norm<TX, TY, VEC, MESORASI_ACT_GELU>(a, p, s); break;
        default: launch_group_norm<TX, TY, VEC, MESORASI_ACT_NONE>(a, p, s); break;
    }
}

}  // namespace

}  // namespace meso

using namespace meso;

static bool group_norm_sizes_ok(int64_t B, int64_t N, int32_t C, int32_t G) {
    return B >= 1 && N >= 1 && C >= 1 && G >= 1 && C % G == 0 && C <= MESORASI_MAX_C_NORM && N <= 0x7fffffff &&
           B <= 0x7fffffff / G;
}

extern "C" size_t mesorasi_group_norm_workspace(int64_t B, int64_t N, int32_t C, int32_t G, int32_t x_dtype) {
    if (!group_norm_sizes_ok(B, N, C, G) || (x_dtype != MESORASI_F32 && x_dtype != MESORASI_BF16)) return 0;
    // rows of any alignment: the larger of both vector widths' needs
    const size_t a = group_norm_ws(plan_group_norm(B, N, C, G, 1), B, G);
    const int vec = group_norm_vec(C, G, x_dtype);
    return std::max(a, group_norm_ws(plan_group_norm(B, N, C, G, vec), B, G));
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
    const int ex = x_dtype == MESORASI_F32 ? 4 : 2, ey = y_dtype == MESORASI_F32 ? 4 : 2;
    int vec = group_norm_vec(C, G, x_dtype);
    if (vec > 1 && !(ld_x % vec == 0 && ld_y % vec == 0 && aligned(x, vec * ex) && aligned(y, std::min(16, vec * ey))))
        vec = 1;
    const GnPlan p = plan_group_norm(B, N, C, G, vec);
    const size_t need = group_norm_ws(p, B, G);
    MESO_REQUIRE(need == 0 || (ws && ws_bytes >= need), MESORASI_EWORKSPACE,
                 "mesorasi_group_norm: workspace %zu < %zu bytes", ws ? ws_bytes : (size_t)0, need);
    MESO_REQUIRE(need == 0 || aligned(ws, 16), MESORASI_EINVAL, "mesorasi_group_norm: ws is not 16-byte aligned");
    MESO_REQUIRE(launch_fits(ceil_div(B * p.slabs * p.chunks, 8) * 8, p.keep ? kGnOneThreads : kGnThreads), MESORASI_EUNSUPPORTED, "mesorasi_group_norm: B = %lld, N = %lld",
                 (long long)B, (long long)N);
    MESO_REQUIRE(!overlap(rows_extent(x, B * N, ld_x, C, ex), rows_extent(y, B * N, ld_y, C, ey)), MESORASI_EINVAL,
                 "mesorasi_group_norm: y overlaps x");
    const int blocks = (int)(B * p.slabs * p.chunks);
    const GnArgs a = {x, y, lens, gamma, beta, static_cast<GnPart*>(ws), ld_x, ld_y, B, N, C, G, C / G, eps, act,
                      p.slab, p.slabs, p.pieces, p.chunks, p.chunk_rows, blocks, (int)ceil_div(blocks, 8), FastDiv(p.chunks), FastDiv(p.slabs),
                      FastDiv(p.pieces), FastDiv(C / G), FastDiv((unsigned)p.chunk_rows), FastDiv((unsigned)ceil_div(p.slab, vec))};
    hipStream_t s = as_stream(stream);
#define MESO_GN(TX, TY, V)                                              \
    do {                                                                \
        if (vec > 1) launch_group_norm<TX, TY, V>(a, p, s);             \
        else launch_group_norm<TX, TY, 1>(a, p, s);                     \
    } while (0)
    if (x_dtype == MESORASI_F32) {
        if (y_dtype == MESORASI_F32) MESO_GN(float, float, 4);
        else MESO_GN(float, uint16_t, 4);
    } else {
        if (y_dtype == MESORASI_F32) MESO_GN(uint16_t, float, 8);
        else MESO_GN(uint16_t, uint16_t, 8);
    }
#undef MESO_GN
    return after_launch("mesorasi_group_norm");
}
