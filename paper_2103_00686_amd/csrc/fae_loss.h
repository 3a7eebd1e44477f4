// Softmax cross entropy over the rows of a table: the kernel that the forward and the classes' gradient share (gfx950).
#pragma once

#include "fae_rows.h"

// Both directions stream rows past rows that a wave holds: Z = (streamed rows) x (held rows)^T by matrix instructions, P = a function of Z in
// registers, O += (streamed rows)^T x P by matrix instructions.
//   LOSS_STATS  held: x, streamed: w; running maximum and sum of 2^Z for every row of x, and the target's Z
//   LOSS_MEAN   the same, and O = the sum of 2^Z w of all classes but the target
//   LOSS_GRAD   held: w, streamed: x; P = gloss (2^(Z - lse) - (class is the target)), O = the sum of P x, and the sum of P (bias)
// Z is in units of log 2 throughout.
enum { LOSS_STATS, LOSS_MEAN, LOSS_GRAD };

struct loss_args {
    const void *st, *own; // streamed rows, held rows
    int64_t st_stride, own_stride;
    int32_t n_st, n_own, width;
    int32_t flip;         // scale < 0: the held rows are negated
    float c;              // |scale| * log2(e)
    const float *bias;    // fp32[n_classes] or NULL
    const void *targets;  // forward
    int32_t target_bits, n_classes;
    const float *nlse, *g;  // gradient, per streamed row: -lse * log2(e), gloss (0 without a target)
    const int32_t *t;       // ... and its target or -1
    const uint32_t *g_most; // fp16: the bits of the largest |gloss|
    uint32_t *status;
    float *stat; // forward: [n_split][n_own][2]: reference, sum of 2^(Z - reference)
    float *zt;   // forward: [n_own] Z of the target
    float *part; // [n_split][n_own][pitch] O
    float *psum; // gradient: [n_split][n_own] sums of P, or NULL
    void *out;   // gradient, one split: gw
    int64_t out_stride;
    float *out_sum; // ... and gbias or NULL
    float scale;
    int32_t pitch, tiles; // tiles: of streamed rows
    uint32_t n_blocks, n_split;
};

static inline int loss_padded(int32_t width) { return width <= 32 ? 32 : width <= 64 ? 64 : width <= 96 ? 96 : width <= 128 ? 128 : width <= 192 ? 192 : 256; }
static inline int loss_tile(int32_t type, int dp) { return type == FAE_F32 && dp > 128 ? 32 : 64; }
#define LOSS_WAVES 4
#define LOSS_HELD (LOSS_WAVES * 32) // held rows of a workgroup

void loss_launch_f32(fae_ctx *ctx, int mode, const loss_args &a);
void loss_launch_bf16(fae_ctx *ctx, int mode, const loss_args &a);
void loss_launch_f16(fae_ctx *ctx, int mode, const loss_args &a);

// a row's target, or -1; one that is no class is reported
#ifdef __HIPCC__
__device__ __forceinline__ int32_t loss_target(const void *targets, int32_t bits, int64_t r, int32_t n_classes, uint32_t *status)
{
    const int64_t t = bits == 64 ? ((const int64_t *)targets)[r] : ((const int32_t *)targets)[r];
    if (t >= n_classes)
        fae_flag(status, FAE_STATUS_ERANGE);
    return t < 0 || t >= n_classes ? -1 : (int32_t)t;
}
#endif

#ifdef LOSS_KERNELS

typedef float loss_f16v __attribute__((ext_vector_type(16)));
typedef float loss_f4 __attribute__((ext_vector_type(4)));

// How a type enters the matrix instructions: as PLANES numbers of E, whose sum is the value (fp32: 24 bits are three times eight;
// fp32's own matrix instructions have a sixteenth of bf16's rate, six products of bf16 take three eighths of their time).
// SHIFT: probabilities are multiplied by 2^SHIFT (fp16 has nothing below 2^-24, and a million classes have probabilities of 2^-20).
// SLACK: how far above 1 they may be before the reference moves (a running maximum that moves rarely).
template <typename T> struct loss_type;
template <> struct loss_type<fae_bf16> {
    typedef fae_bf16 E;
    static constexpr int PLANES = 1, PRODUCTS = 1, SHIFT = 0, SLACK = 16;
};
template <> struct loss_type<fae_f16> {
    typedef fae_f16 E;
    static constexpr int PLANES = 1, PRODUCTS = 1, SHIFT = 12, SLACK = 3;
};
template <> struct loss_type<float> {
    typedef fae_bf16 E;
    static constexpr int PLANES = 3, PRODUCTS = 6, SHIFT = 0, SLACK = 16;
};
// the products of planes that are summed, small ones first; with one plane the last
static constexpr int LOSS_PA[6] = {2, 1, 0, 1, 0, 0}, LOSS_PB[6] = {0, 1, 2, 0, 1, 0};

template <typename E> struct loss_vec {
    typedef E v8 __attribute__((ext_vector_type(8)));
    typedef E v4 __attribute__((ext_vector_type(4)));
};

__device__ __forceinline__ loss_f16v loss_mfma(loss_vec<fae_bf16>::v8 a, loss_vec<fae_bf16>::v8 b, loss_f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ loss_f16v loss_mfma(loss_vec<fae_f16>::v8 a, loss_vec<fae_f16>::v8 b, loss_f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// fp32 values as three bf16 numbers each (rounded to nearest, so that what is left out has either sign)
template <typename T, typename E> __device__ __forceinline__ void loss_split(const float (&v)[8], typename loss_vec<E>::v8 (&o)[loss_type<T>::PLANES])
{
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        r[e] = v[e];
#pragma unroll
    for (int p = 0; p < loss_type<T>::PLANES; ++p) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            o[p][e] = (E)r[e];
        if (p + 1 < loss_type<T>::PLANES) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                r[e] -= (float)o[p][e];
        }
    }
}

// eight values of a row as they are in memory; zeros where there are none
template <typename T> struct loss_raw {
    T v[8];
};
template <typename T> __device__ __forceinline__ loss_raw<T> loss_load(const T *row, int col, int width, bool there)
{
    loss_raw<T> o;
    if (there && col + 8 <= width) {
        typedef typename fae_vec<T, 16 / sizeof(T)>::loose loose;
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
            const auto x = *(const loose *)(row + col + h * (16 / sizeof(T)));
#pragma unroll
            for (int e = 0; e < (int)(16 / sizeof(T)); ++e)
                o.v[h * (16 / sizeof(T)) + e] = x[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            o.v[e] = there && col + e < width ? row[col + e] : (T)0.f;
    }
    return o;
}
template <typename T, typename E> __device__ __forceinline__ void loss_planes(const loss_raw<T> &x, typename loss_vec<E>::v8 (&o)[loss_type<T>::PLANES])
{
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            o[0][e] = x.v[e];
    } else {
        loss_split<T, E>(x.v, o);
    }
}

// A tile's row lies in LDS without padding; its 16-byte pieces are placed by an exclusive or with some bits of the row, so that both kinds of reads
// spread over all banks: 16 rows' piece of one number (Z), and 4 rows' 4 neighbouring pieces (O, transposed on the way).
template <int DP> __device__ __forceinline__ int loss_swizzle(int m)
{
    constexpr int u = DP / 8 % 16;
    return u == 0 ? ((m & 3) << 2) | ((m >> 2) & 3) : u == 8 ? ((m & 2) << 1) | ((m >> 2) & 3) : (m >> 2) & 3;
}

template <typename T, int DP, int MODE> __global__ __launch_bounds__(LOSS_WAVES * 64) void loss_kernel(loss_args a)
{
    typedef typename loss_type<T>::E E;
    typedef typename loss_vec<E>::v8 v8;
    typedef typename loss_vec<E>::v4 v4;
    constexpr int P = loss_type<T>::PLANES, NP = loss_type<T>::PRODUCTS, THREADS = LOSS_WAVES * 64;
    constexpr int TM = P == 3 && DP > 128 ? 32 : 64;
    constexpr int KS = DP / 16, NC = TM * DP / 8 / THREADS;
    constexpr bool HAS_O = MODE != LOSS_STATS;
    static_assert(TM * DP / 8 % THREADS == 0, "whole pieces per thread");
    __shared__ E tile[2][P][TM * DP];
    __shared__ float side[2][3][TM]; // forward: bias; gradient: -lse, gloss, target

    const int lane = fae_lane(), wave = threadIdx.x / 64, ln = lane & 31, half = lane >> 5;
    uint32_t block, split;
    if (a.n_split % 8 == 0) { // the workgroups of one part of the chip stream the same rows
        const uint32_t i = blockIdx.x >> 3;
        split = i / a.n_blocks * 8 + (blockIdx.x & 7);
        block = i % a.n_blocks;
    } else {
        split = blockIdx.x / a.n_blocks;
        block = blockIdx.x % a.n_blocks;
    }
    const int tile0 = (int)((int64_t)a.tiles * split / a.n_split), tile1 = (int)((int64_t)a.tiles * (split + 1) / a.n_split);
    const int n = (int)(block * LOSS_HELD) + wave * 32 + ln; // this lane's held row (may lie behind the last)
    const bool there = n < a.n_own;

    // the held row: value 16 k + 8 half + j is element j of operand k
    v8 q[KS][P];
    {
        const T *row = (const T *)a.own + (int64_t)n * a.own_stride;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            loss_raw<T> x = loss_load<T>(row, k * 16 + half * 8, a.width, there);
            if (a.flip) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x.v[e] = -x.v[e];
            }
            loss_planes<T, E>(x, q[k]);
        }
    }
    int32_t target = -1;
    if (MODE != LOSS_GRAD && there)
        target = loss_target(a.targets, a.target_bits, n, a.n_classes, a.status);
    float own_bias = 0.f, g_scale = 1.f;
    if (MODE == LOSS_GRAD) {
        if (there && a.bias)
            own_bias = a.bias[n] * 1.44269504f;
        if (loss_type<T>::SHIFT) {
            const float most = __uint_as_float(*a.g_most);
            // 2^SHIFT is the largest P
            g_scale = most > 0.f && most < INFINITY ? __builtin_amdgcn_ldexpf(1.f, loss_type<T>::SHIFT - __builtin_amdgcn_frexp_expf(most)) : 1.f;
        }
    }

    loss_raw<T> next[NC];
    int32_t next_t[NC];
    float next_side[3];
    auto fetch = [&](int tl) {
        const int m0 = tl * TM;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int piece = i * THREADS + threadIdx.x, m = piece / (DP / 8), c = piece % (DP / 8);
            next[i] = loss_load<T>((const T *)a.st + (int64_t)(m0 + m) * a.st_stride, c * 8, a.width, m0 + m < a.n_st);
            if (MODE == LOSS_GRAD)
                next_t[i] = m0 + m < a.n_st ? a.t[m0 + m] : -1;
        }
        if (threadIdx.x < TM) {
            const int m = m0 + threadIdx.x;
            const bool in = m < a.n_st;
            if (MODE == LOSS_GRAD) {
                next_side[0] = in ? a.nlse[m] : -INFINITY;
                next_side[1] = in ? a.g[m] * g_scale : 0.f;
                next_side[2] = __int_as_float(in ? a.t[m] : -1);
            } else
                next_side[0] = !in ? -INFINITY : (a.bias ? a.bias[m] * 1.44269504f : 0.f);
        }
    };
    auto place = [&](int buf) {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int piece = i * THREADS + threadIdx.x, m = piece / (DP / 8), c = piece % (DP / 8);
            v8 o[P];
            if (MODE == LOSS_GRAD) { // a row without a target may hold anything, and 0 times that is not always 0
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    next[i].v[e] = next_t[i] < 0 ? (T)0.f : next[i].v[e];
            }
            loss_planes<T, E>(next[i], o);
#pragma unroll
            for (int p = 0; p < P; ++p)
                *(v8 *)&tile[buf][p][m * DP + (c ^ loss_swizzle<DP>(m)) * 8] = o[p];
        }
        if (threadIdx.x < TM) {
            side[buf][0][threadIdx.x] = next_side[0];
            if (MODE == LOSS_GRAD) {
                side[buf][1][threadIdx.x] = next_side[1];
                side[buf][2][threadIdx.x] = next_side[2];
            }
        }
    };

    loss_f16v o[HAS_O ? DP / 32 : 1];
    if (HAS_O) {
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
            o[d] = (loss_f16v)(0.f);
    }
    // Forward: 2^(Z - ref) is what is summed.  Gradient: sum is that of P.
    float ref = -3.402823466e38f, sum = 0.f;
    if (tile0 < tile1) {
        fetch(tile0);
        place(0);
    }
    __syncthreads();
    for (int tl = tile0; tl < tile1; ++tl) {
        const int buf = (tl - tile0) & 1;
        const bool more = tl + 1 < tile1;
        if (more)
            fetch(tl + 1);
#pragma unroll 1
        for (int sb = 0; sb < TM / 32; ++sb) {
            // Z: element i is streamed row 8 (i / 4) + 4 half + i % 4 and held row ln
            loss_f16v z = (loss_f16v)(0.f);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                v8 x[P];
#pragma unroll
                for (int p = 0; p < P; ++p)
                    x[p] = *(const v8 *)&tile[buf][p][(sb * 32 + ln) * DP + ((k * 2 + half) ^ loss_swizzle<DP>(ln)) * 8];
#pragma unroll
                for (int u = 6 - NP; u < 6; ++u)
                    z = loss_mfma(x[LOSS_PA[u]], q[k][LOSS_PB[u]], z);
            }
            float pr[16];
            const float *sd = &side[buf][0][sb * 32 + half * 4];
            if (MODE == LOSS_GRAD) {
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const loss_f4 nl = *(const loss_f4 *)(sd + b * 8), g = *(const loss_f4 *)(sd + TM + b * 8);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = b * 4 + e;
                        pr[i] = __builtin_amdgcn_exp2f(fmaf(z[i], a.c, own_bias + nl[e])) * g[e];
                    }
                }
                // a target in this wave's classes
                const int32_t mine = __float_as_int(side[buf][2][sb * 32 + ln]);
                const int first = (int)(block * LOSS_HELD) + wave * 32;
                if (__any(mine >= first && mine < first + 32)) {
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const loss_f4 g = *(const loss_f4 *)(sd + TM + b * 8), t = *(const loss_f4 *)(sd + 2 * TM + b * 8);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            pr[b * 4 + e] -= __float_as_int(t[e]) == n ? g[e] : 0.f;
                    }
                }
                float some = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    some += pr[i];
                sum += some;
            } else {
                float most = -INFINITY;
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const loss_f4 bs = *(const loss_f4 *)(sd + b * 8);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        z[b * 4 + e] = fmaf(z[b * 4 + e], a.c, bs[e]);
                        most = fmaxf(most, z[b * 4 + e]);
                    }
                }
                if (__any(most > ref + (float)loss_type<T>::SLACK)) {
                    most = fmaxf(most, __shfl_xor(most, 32, 64));
                    const float to = most > ref + (float)loss_type<T>::SLACK ? most : ref;
                    const float f = __builtin_amdgcn_exp2f(ref - to);
                    ref = to;
                    sum *= f;
                    if (HAS_O) {
#pragma unroll
                        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                o[d][i] *= f;
                    }
                }
                float some = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    pr[i] = __builtin_amdgcn_exp2f(z[i] - (ref - (float)loss_type<T>::SHIFT));
                    some += pr[i];
                }
                sum += some;
                const int at = target - tl * TM - sb * 32;
                if (__any((unsigned)at < 32u)) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (8 * (i / 4) + 4 * half + i % 4 == at) {
                            a.zt[n] = z[i];
                            pr[i] = 0.f;
                        }
                }
            }
            if (HAS_O) {
                // eight streamed rows of a lane are the eight of an operand: rows 16 t + 4 half + {0..3, 8..11}
                v8 pb[2][P];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[e] = pr[t * 8 + e];
                    loss_split<T, E>(v, pb[t]);
                }
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        v8 x[P];
#pragma unroll
                        for (int p = 0; p < P; ++p) {
                            typedef short s4 __attribute__((ext_vector_type(4)));
                            typedef __attribute__((address_space(3))) s4 *lds4;
                            s4 w[2];
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                // 16 lanes take 4 rows of 16 columns; each gets its column's 4 values
                                const int m = sb * 32 + t * 16 + u * 8 + half * 4 + ((lane & 15) >> 2);
                                const int c = d * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
                                E *at = &tile[buf][p][m * DP + (c ^ loss_swizzle<DP>(m)) * 8 + (lane & 1) * 4];
                                w[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)at);
                            }
                            x[p] = __builtin_shufflevector(__builtin_bit_cast(v4, w[0]), __builtin_bit_cast(v4, w[1]), 0, 1, 2, 3, 4, 5, 6, 7);
                        }
#pragma unroll
                        for (int u = 6 - NP; u < 6; ++u)
                            o[d] = loss_mfma(x[LOSS_PA[u]], pb[t][LOSS_PB[u]], o[d]);
                    }
                }
            }
        }
        if (more)
            place(buf ^ 1);
        __syncthreads();
    }

    sum += __shfl_xor(sum, 32, 64);
    if (!there)
        return;
    const int64_t at = (int64_t)split * a.n_own + n;
    if (MODE != LOSS_GRAD) {
        if (half == 0) {
            a.stat[at * 2] = ref - (float)loss_type<T>::SHIFT;
            a.stat[at * 2 + 1] = sum;
        }
    } else if (half == 0) {
        if (a.n_split > 1 && a.psum)
            a.psum[at] = sum / g_scale;
        else if (a.n_split == 1 && a.out_sum)
            a.out_sum[n] = sum / g_scale;
    }
    if (HAS_O) {
        const bool direct = MODE == LOSS_GRAD && a.n_split == 1;
        const float f = MODE == LOSS_GRAD ? (direct ? a.scale : 1.f) / g_scale : 1.f;
        if (direct && !a.out)
            return;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int c = d * 32 + b * 8 + half * 4;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = o[d][b * 4 + e] * f;
                if (!direct) {
                    if (c < a.pitch && a.part)
                        *(loss_f4 *)(a.part + at * a.pitch + c) = loss_f4{v[0], v[1], v[2], v[3]};
                } else {
                    fae_place<4> p;
                    p.set(c, a.width);
                    fae_store<T, 4, FAE_ANY>((T *)a.out + (int64_t)n * a.out_stride, v, p);
                }
            }
        }
    }
}

template <typename T, int DP> static void loss_launch_mode(fae_ctx *ctx, int mode, const loss_args &a)
{
    const dim3 grid(a.n_blocks * a.n_split), block(LOSS_WAVES * 64);
    if (mode == LOSS_STATS)
        FAE_LAUNCH(ctx, (loss_kernel<T, DP, LOSS_STATS>), grid, block, 0, ctx->stream, a);
    else if (mode == LOSS_MEAN)
        FAE_LAUNCH(ctx, (loss_kernel<T, DP, LOSS_MEAN>), grid, block, 0, ctx->stream, a);
    else
        FAE_LAUNCH(ctx, (loss_kernel<T, DP, LOSS_GRAD>), grid, block, 0, ctx->stream, a);
}
template <typename T> static void loss_launch(fae_ctx *ctx, int mode, const loss_args &a)
{
    switch (loss_padded(a.width)) {
    case 32: return loss_launch_mode<T, 32>(ctx, mode, a);
    case 64: return loss_launch_mode<T, 64>(ctx, mode, a);
    case 96: return loss_launch_mode<T, 96>(ctx, mode, a);
    case 128: return loss_launch_mode<T, 128>(ctx, mode, a);
    case 192: return loss_launch_mode<T, 192>(ctx, mode, a);
    default: return loss_launch_mode<T, 256>(ctx, mode, a);
    }
}

#endif // LOSS_KERNELS
