// Softmax cross entropy over the rows of a table: the kernel that the forward and the classes' gradient share (gfx950).
#pragma once

#include "fae_rows.h"

// Both directions stream rows past rows that a wave holds: Z = (streamed rows) x (held rows)^T by matrix instructions, P = a function of Z in
// registers, O += (streamed rows)^T x P by matrix instructions.
//   LOSS_STATS  held: x, streamed: w; reference and sum of 2^(Z - reference) of all classes but the target for every row of x, and the target's Z
//               (the reference is one of the others too: the target's may lie far above)
//   LOSS_MEAN   the same, and O = the sum of 2^(Z - reference) w of all classes but the target; of 16-bit types also the sum of P as rounded for O
//   LOSS_GRAD   held: w, streamed: x; P = gloss 2^(Z - lse), or what the row leaves to its target, O = the sum of P x, and the sum of P (bias)
// Z is in units of log 2 throughout.
//   LOSS_FEW    what LOSS_STATS finds, for few rows
enum { LOSS_STATS, LOSS_MEAN, LOSS_GRAD, LOSS_FEW };

struct loss_args {
    const void *st, *own; // streamed rows, held rows
    int64_t st_stride, own_stride;
    int32_t n_st, n_own, width;
    int32_t flip;         // scale < 0: the held rows are negated
    float c;              // |scale| * log2(e)
    const float *bias;    // fp32[n_classes] or NULL
    const void *targets;  // forward
    int32_t target_bits, n_classes;
    const float *st_most; // fp32 as fp16 numbers: n_most values, the largest of them is the largest streamed value
    const float *g_most;  // gradient of fp16: the same of |gloss|
    int32_t n_most;
    const float *nlse, *gt; // gradient, per streamed row: -lse * log2(e) + log2 |gloss|, P of its target (-infinity and -0 without one)
    const int32_t *t;      // ... and its target or -1
    uint32_t *status;
    float *stat; // forward: [n_split][n_own][2]: reference, sum of 2^(Z - reference)
    float *zt;   // forward: [n_own] Z of the target
    float *part; // [n_split][n_own][pitch] O
    float *psum; // [n_split][n_own]: gradient, sums of P, or NULL; means of 16-bit types, sums of P as it entered O
    void *out;   // gradient, one split: gw
    int64_t out_stride;
    float *out_sum; // ... and gbias or NULL
    float scale;
    int32_t pitch, tiles; // tiles: of streamed rows
    uint32_t n_blocks, n_split;
    int32_t spread; // forward: all waves hold the same rows (there are no more than one holds), and take the streamed blocks of 32 in turn
};

// What a kernel is built for: the types, and fp32 in two ways (loss_type says how).
enum { LOSS_F32, LOSS_BF16, LOSS_F16, LOSS_F32_WIDE };
constexpr int loss_planes_of(int how) { return how == LOSS_F32 ? 3 : how == LOSS_F32_WIDE ? 2 : 1; }
static inline int loss_padded(int32_t width) { return width <= 32 ? 32 : width <= 64 ? 64 : width <= 96 ? 96 : width <= 128 ? 128 : width <= 192 ? 192 : 256; }
#define LOSS_F32_WIDTH 64 // LOSS_F32 for wider rows is for few rows alone
constexpr int loss_tile(int how, int dp) { return dp > 128 && loss_planes_of(how) > 1 ? 32 : 64; }
// held rows of a wave, in blocks of 32: two where their registers leave room for two waves on a SIMD
constexpr int loss_blocks(int how, int dp, int mode)
{
    return loss_planes_of(how) > 1 ? (dp <= 32 ? 2 : 1) : (dp <= (mode == LOSS_STATS ? 128 : 64) ? 2 : 1);
}
// Waves that hold the same rows, each with a share of O's columns: two for wide rows, whose O would leave room for one wave alone on a SIMD
// (both take all scores and powers: 48 matrix instructions for 32 x 32 scores where 32 are needed, and still a step of 8192 x 32 768 x 256 bf16
// took 910 us instead of 1130 when this was chosen).
constexpr int loss_shares(int how, int dp, int mode) { return mode != LOSS_STATS && dp > 128 ? 2 : 1; }
// Waves per SIMD that registers are left for: three of 168 registers, else two of 256.
// Two and three, when this was chosen: loss of 16 384 x 131 072 x 64 bf16 512 and 447 us, the gradient of 2048 x 100 000 x 64 fp32 218 and 203; but
// with spills (fp32 means of width 32) 870 and 1120.  What the compiler spills all the same: means of 16-bit types of width 32, 42 registers
// with a bias and 5 without; fp32 of width 64 to 192 up to 27, of 256 37 to 89 (9 for the loss with a bias).
constexpr int loss_waves(int how, int dp, int mode)
{
    if (how == LOSS_F32)
        return 2;
    const bool three = dp <= 32 ? mode != LOSS_MEAN || how != LOSS_F32_WIDE : dp <= 64 && (mode == LOSS_STATS || how == LOSS_F32_WIDE);
    return three ? 3 : 2;
}
#define LOSS_WAVES 4
constexpr int loss_held(int how, int dp, int mode) { return LOSS_WAVES * 32 * loss_blocks(how, dp, mode); }

// few rows, LOSS_FEW_ROWS at most: blocks of 32 that a wave holds, and the workgroups of a launch.  Where a wave holds one block (fp32
// padded to 96 and more, 16 bits padded to 256), 33 to 64 rows are two of them, and the classes are read twice.  Spilled: 16 bits of width 129 to 192 in two blocks 163 registers
// with a bias and 53 without, fp32 of width 193 to 256 65 and 43.
constexpr int loss_few_blocks(int how, int dp) { return loss_planes_of(how) * dp <= 192 ? 2 : 1; }
#define LOSS_FEW_ROWS 64
#define LOSS_FEW_GROUPS 512 // two for each compute unit

void loss_launch_f32(fae_ctx *ctx, int mode, const loss_args &a);
void loss_launch_bf16(fae_ctx *ctx, int mode, const loss_args &a);
void loss_launch_f16(fae_ctx *ctx, int mode, const loss_args &a);
void loss_launch_f32_wide(fae_ctx *ctx, int mode, const loss_args &a);

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

// How values enter the matrix instructions: as PLANES numbers of E whose sum is the value, with the PRODUCTS largest products of them.  fp32's
// own matrix instructions have a sixteenth of bf16's rate.
//   LOSS_F32       three bf16 numbers, 24 bits with fp32's range: six products
//   LOSS_F32_WIDE  two fp16 numbers, 22 bits and more (rounded to nearest both times), three products; values are multiplied by a power of two
//                  first that brings the largest of a held row, or of all streamed rows, to 2^14 .. 2^15, where values down
//                  to 2^-18 of it keep all their bits.  Costs a look at all streamed rows before.
// SHIFT: probabilities are multiplied by 2^SHIFT (fp16 has nothing below 2^-24, and a million classes have probabilities of 2^-20).
// MOST: the reference (in fp32's gradient, a class's power of two) moves when a lane's sum of 16 of them reaches it.  They are then below fp16's
// 65504; the other types, with fp32's range, let the reference lag far behind the maximum, which costs no precision and spares them the
// search for it.
template <int HOW> struct loss_type;
template <> struct loss_type<LOSS_BF16> {
    typedef fae_bf16 T, E;
    static constexpr int PLANES = 1, PRODUCTS = 1, SHIFT = 0;
    static constexpr float MOST = 0x1p24f;
};
template <> struct loss_type<LOSS_F16> {
    typedef fae_f16 T, E;
    static constexpr int PLANES = 1, PRODUCTS = 1, SHIFT = 10;
    static constexpr float MOST = 0x1p15f;
};
template <> struct loss_type<LOSS_F32> {
    typedef float T;
    typedef fae_bf16 E;
    static constexpr int PLANES = 3, PRODUCTS = 6, SHIFT = 0;
    static constexpr float MOST = 0x1p24f;
};
template <> struct loss_type<LOSS_F32_WIDE> {
    typedef float T;
    typedef fae_f16 E;
    static constexpr int PLANES = 2, PRODUCTS = 3, SHIFT = 10;
    static constexpr float MOST = 0x1p15f;
};
// the products of planes that are summed, small ones first: the last PRODUCTS of these
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

// A step of a score.  Wide fp32 rows: the small products of planes go to a sum of their own, so that the large one is rounded once per 16
// values and not three or six times (an addition per score more; 3863 x 132 x 224 2e-6 off without, 6e-7 with).
template <int HOW, int KS> constexpr bool loss_apart() { return loss_type<HOW>::PLANES > 1 && KS > 4; }
template <int HOW, int KS, typename V, int P> __device__ __forceinline__ void loss_score(const V (&x)[P], const V (&q)[P], loss_f16v &z, loss_f16v &less)
{
#pragma unroll
    for (int u = 6 - loss_type<HOW>::PRODUCTS; u < 6; ++u) {
        loss_f16v &to = loss_apart<HOW, KS>() && u < 5 ? less : z;
        to = loss_mfma(x[LOSS_PA[u]], q[LOSS_PB[u]], to);
    }
}

// eight fp32 values as planes, each rounded to nearest so that what is left has either sign (SCALED, two fp16 numbers alone: times a power of two)
template <int HOW, bool SCALED = false>
__device__ __forceinline__ void loss_split(const float (&v)[8], typename loss_vec<typename loss_type<HOW>::E>::v8 (&o)[loss_type<HOW>::PLANES], float up = 1.f)
{
    typedef typename loss_type<HOW>::E E;
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        r[e] = v[e];
#pragma unroll
    for (int p = 0; p < loss_type<HOW>::PLANES; ++p) {
        if constexpr (SCALED) {
            if (p == 0) { // a mixed product and sum rounds to either half of a register
                typedef uint32_t words __attribute__((ext_vector_type(4)));
                words w;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    uint32_t two;
                    asm("v_fma_mixlo_f16 %0, %1, %2, 0" : "=v"(two) : "v"(r[e]), "v"(up));
                    asm("v_fma_mixhi_f16 %0, %1, %2, 0" : "+v"(two) : "v"(r[e + 1]), "v"(up));
                    w[e / 2] = two;
                    asm("v_fma_mix_f32 %0, %0, %2, -%1 op_sel_hi:[0,0,1]" : "+v"(r[e]) : "v"(two), "v"(up));
                    asm("v_fma_mix_f32 %0, %0, %2, -%1 op_sel:[0,0,1] op_sel_hi:[0,0,1]" : "+v"(r[e + 1]) : "v"(two), "v"(up));
                }
                o[0] = __builtin_bit_cast(typename loss_vec<E>::v8, w);
                continue;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            o[p][e] = (E)r[e];
        if (p + 1 < loss_type<HOW>::PLANES) {
            if constexpr (HOW == LOSS_F32_WIDE) { // a mixed product and sum reads the fp16 number where it is: one instruction
                typedef uint32_t words __attribute__((ext_vector_type(4)));
                const words w = __builtin_bit_cast(words, o[p]);
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    asm("v_fma_mix_f32 %0, %0, 1.0, -%1 op_sel_hi:[0,0,1]" : "+v"(r[e]) : "v"(w[e / 2]));
                    asm("v_fma_mix_f32 %0, %0, 1.0, -%1 op_sel:[0,0,1] op_sel_hi:[0,0,1]" : "+v"(r[e + 1]) : "v"(w[e / 2]));
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    r[e] -= (float)o[p][e];
            }
        }
    }
}

// eight values of a row as they are in memory; zeros where there are none
template <typename T> struct loss_raw {
    T v[8];
};
template <typename T> __device__ __forceinline__ loss_raw<T> loss_load_whole(const T *at)
{
    typedef typename fae_vec<T, 16 / sizeof(T)>::loose loose;
    loss_raw<T> o;
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
        const auto x = *(const loose *)(at + h * (16 / sizeof(T)));
#pragma unroll
        for (int e = 0; e < (int)(16 / sizeof(T)); ++e)
            o.v[h * (16 / sizeof(T)) + e] = x[e];
    }
    return o;
}
template <typename T> __device__ __forceinline__ loss_raw<T> loss_load(const T *row, int col, int width, bool there)
{
    if (there && col + 8 <= width)
        return loss_load_whole(row + col);
    loss_raw<T> o;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        o.v[e] = there && col + e < width ? row[col + e] : (T)0.f;
    return o;
}
// the same with a row's end by four values first: for where few rows are missing
template <typename T> __device__ __forceinline__ loss_raw<T> loss_load_ends(const T *row, int col, int width, bool there)
{
    if (there && col + 8 <= width)
        return loss_load_whole(row + col);
    loss_raw<T> o;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        o.v[e] = (T)0.f;
    if (there && col < width) { // a row's end
        const int left = width - col;
        int done = 0;
        if (left >= 4) {
            const auto x = *(const typename fae_vec<T, 4>::loose *)(row + col);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                o.v[e] = x[e];
            done = 4;
        }
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (done + e < left) {
                const T x = row[col + done + e];
                if (done)
                    o.v[4 + e] = x;
                else
                    o.v[e] = x;
            }
    }
    return o;
}
// zeros instead, by whole words
template <typename T> __device__ __forceinline__ loss_raw<T> loss_clear(const loss_raw<T> &x, bool clear)
{
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(x) / 4)));
    words w = __builtin_bit_cast(words, x);
#pragma unroll
    for (int i = 0; i < (int)sizeof(x) / 4; ++i)
        w[i] = clear ? 0u : w[i];
    return __builtin_bit_cast(loss_raw<T>, w);
}
// a sum, and eight probabilities as they enter a product
__device__ __forceinline__ float loss_add(const loss_vec<fae_bf16>::v8 &p, float s)
{
    typedef fae_bf16 two __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int e = 0; e < 8; e += 2)
        s = __builtin_amdgcn_fdot2_f32_bf16(two{p[e], p[e + 1]}, two{(fae_bf16)1.f, (fae_bf16)1.f}, s, false);
    return s;
}
__device__ __forceinline__ float loss_add(const loss_vec<fae_f16>::v8 &p, float s)
{
    typedef fae_f16 two __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int e = 0; e < 8; e += 2)
        s = __builtin_amdgcn_fdot2(two{p[e], p[e + 1]}, two{(fae_f16)1.f, (fae_f16)1.f}, s, false);
    return s;
}

template <int HOW>
__device__ __forceinline__ void loss_planes(const loss_raw<typename loss_type<HOW>::T> &x, float scale,
                                            typename loss_vec<typename loss_type<HOW>::E>::v8 (&o)[loss_type<HOW>::PLANES])
{
    if constexpr (HOW == LOSS_BF16 || HOW == LOSS_F16) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            o[0][e] = x.v[e];
    } else {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = HOW == LOSS_F32_WIDE ? x.v[e] * scale : x.v[e];
        loss_split<HOW>(v, o);
    }
}

// the power of two that brings `most` to 2^(top - 1) .. 2^top, and none for 0 and what is not finite
__device__ __forceinline__ int loss_power(float most, int top)
{
    const int up = top - __builtin_amdgcn_frexp_expf(most);
    return most > 0.f && most < INFINITY ? (up < 120 ? up : 120) : 0;
}

// A tile's row lies in LDS without padding; its 16-byte pieces are placed by an exclusive or with some bits of the row, so that both kinds of reads
// spread over all banks: 16 rows' piece of one number (Z), and 4 rows' 4 neighbouring pieces (O, transposed on the way).
template <int DP> __device__ __forceinline__ int loss_swizzle(int m)
{
    constexpr int u = DP / 8 % 16;
    return u == 0 ? ((m & 3) << 2) | ((m >> 2) & 3) : u == 8 ? ((m & 2) << 1) | ((m >> 2) & 3) : (m >> 2) & 3;
}

// (the gradient's, in pairs: a chain of 16 additions would wait for each of them; the forward's powers are added in a chain)
__device__ __forceinline__ float loss_sum(const float (&v)[16])
{
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        s[i] = v[i] + v[i + 8];
    return ((s[0] + s[4]) + (s[2] + s[6])) + ((s[1] + s[5]) + (s[3] + s[7]));
}

__device__ __forceinline__ float loss_sum_abs(const float (&v)[16])
{
    float a[16];
#pragma unroll
    for (int i = 0; i < 16; ++i)
        a[i] = fabsf(v[i]);
    return loss_sum(a);
}

#define LOSS_LDS(T) __attribute__((address_space(3))) T

template <int HOW, int DP, int MODE, bool BIAS>
__global__ __launch_bounds__(LOSS_WAVES * 64 * loss_shares(HOW, DP, MODE)) __attribute__((amdgpu_waves_per_eu(loss_waves(HOW, DP, MODE)))) void loss_kernel(loss_args a)
{
    typedef loss_type<HOW> H;
    typedef typename H::T T;
    typedef typename H::E E;
    typedef typename loss_vec<E>::v8 v8;
    typedef typename loss_vec<E>::v4 v4;
    typedef short s4 __attribute__((ext_vector_type(4)));
    constexpr int P = H::PLANES, NP = H::PRODUCTS, NB = loss_blocks(HOW, DP, MODE), TM = loss_tile(HOW, DP);
    constexpr int SHARES = loss_shares(HOW, DP, MODE), THREADS = LOSS_WAVES * 64 * SHARES;
    constexpr int KS = DP / 16, DS = DP / 32 / SHARES, PIECES = TM * DP / 8, NC = (PIECES + THREADS - 1) / THREADS;
    constexpr int PLANE = TM * DP * 2, TILE = P * PLANE; // bytes
    constexpr bool HAS_O = MODE != LOSS_STATS, ROUNDED = MODE == LOSS_MEAN && P == 1;
    constexpr bool MOVES = MODE == LOSS_GRAD && HOW == LOSS_F32_WIDE;
    __shared__ __attribute__((aligned(16))) char tiles[2 * TILE];
    __shared__ float side[2][3][TM]; // forward: bias; gradient: -lse + log |gloss|, P of the target, target
    __shared__ float mosts[2][LOSS_WAVES * SHARES];

    const int lane = fae_lane(), wave = threadIdx.x / 64 % LOSS_WAVES, share = threadIdx.x / (LOSS_WAVES * 64), ln = lane & 31, half = lane >> 5;
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
    const int first = (int)(block * (LOSS_WAVES * 32 * NB)) + (MODE != LOSS_GRAD && a.spread ? 0 : wave * 32 * NB); // the wave's held rows; this lane's are first + ln + 32 b (they may lie behind the last)

    // What was found before: the largest streamed value (fp32) or gradient (fp16), to bring fp16 numbers to a range that keeps them.
    float st_scale = 1.f, g_scale = 1.f, g_log = 0.f, c_all = a.c, back = 1.f;
    int st_up = 0;
    if (HOW == LOSS_F32_WIDE || (HOW == LOSS_F16 && MODE == LOSS_GRAD)) {
        float most[2] = {0.f, 0.f};
        for (int i = threadIdx.x; i < a.n_most; i += THREADS) {
            if (HOW == LOSS_F32_WIDE)
                most[0] = fmaxf(most[0], a.st_most[i]);
            if (HOW == LOSS_F16)
                most[1] = fmaxf(most[1], a.g_most[i]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int d = 32; d > 0; d >>= 1)
                most[k] = fmaxf(most[k], __shfl_xor(most[k], d, 64));
            if (lane == 0)
                mosts[k][threadIdx.x / 64] = most[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < LOSS_WAVES * SHARES; ++i)
                most[k] = fmaxf(most[k], mosts[k][i]);
        if (HOW == LOSS_F32_WIDE) {
            st_up = loss_power(most[0], 15);
            st_scale = __builtin_amdgcn_ldexpf(1.f, st_up);
            back = __builtin_amdgcn_ldexpf(1.f, -st_up);
            c_all *= back;
        }
        if (HOW == LOSS_F16) {
            // The largest P is below 2^15, and from 2^-39 of it on P is lost.  What gw then lacks is below half its own smallest step of 2^-24 as long as
            // rows x |gloss| |x| |scale| is below 2^14; sums that reach that far are about to leave fp16 on the other side.
            const int up = loss_power(most[1], 15);
            g_scale = __builtin_amdgcn_ldexpf(1.f, up);
            g_log = (float)up;
        }
    }

    // held rows: value 16 k + 8 half + j is element j of operand k
    v8 q[NB][KS][P];
    int32_t target[NB];
    float own_bias[NB], c[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int n = first + b * 32 + ln;
        own_bias[b] = MODE == LOSS_GRAD && BIAS && n < a.n_own ? a.bias[n] * 1.44269504f : 0.f;
        const bool there = n < a.n_own && own_bias[b] != -INFINITY;
        const T *row = (const T *)a.own + (int64_t)n * a.own_stride;
        float scale = a.flip ? -1.f : 1.f;
        c[b] = c_all;
        if (HOW == LOSS_F32_WIDE) {
            float most = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const loss_raw<T> x = loss_load<T>(row, k * 16 + half * 8, a.width, there);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    most = fmaxf(most, fabsf((float)x.v[e]));
            }
            most = fmaxf(most, __shfl_xor(most, 32, 64));
            const int up = loss_power(most, 15);
            scale = __builtin_amdgcn_ldexpf(scale, up);
            c[b] = __builtin_amdgcn_ldexpf(c_all, -up);
        }
        c[b] = fmaxf(c[b], 0x1p-149f); // a scale of 0: no score is off by more than 2^-21, and minus infinity stays what it is
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            loss_raw<T> x = loss_load<T>(row, k * 16 + half * 8, a.width, there);
            if (HOW != LOSS_F32_WIDE && a.flip) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x.v[e] = -x.v[e];
            }
            loss_planes<HOW>(x, scale, q[b][k]);
        }
        target[b] = MODE != LOSS_GRAD && there ? loss_target(a.targets, a.target_bits, n, a.n_classes, a.status) : -1;
    }

    // the next tile on its way from memory to LDS
    loss_raw<T> next[NC];
    // A row without a target, or a class that is not offered, may hold anything, and 0 times that is not always 0: it is staged as zeros.  Which
    // rows these are every wave finds with one load (forward of 4096 x 60 000 x 128 bf16 166 us instead of 202), or in the gradient every
    // piece with its own (2 to 5 % faster there, but for the widest fp32 rows, whose registers are all taken: 1146 us instead of 847).
    constexpr bool BY_PIECE = MODE == LOSS_GRAD && !(HOW == LOSS_F32_WIDE && DP > 192), BY_WAVE = (MODE == LOSS_GRAD || BIAS) && !BY_PIECE;
    int32_t next_t[BY_PIECE ? NC : 1];
    bool next_gone = false; // of row `lane` of the tile
    float next_side[3];
    auto fetch = [&](int tl) {
        const int m0 = tl * TM;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int piece = i * THREADS + threadIdx.x, m = piece / (DP / 8), p = piece % (DP / 8);
            next[i] = loss_load<T>((const T *)a.st + (int64_t)(m0 + m) * a.st_stride, p * 8, a.width, m0 + m < a.n_st && (PIECES % THREADS == 0 || piece < PIECES));
            if (BY_PIECE)
                next_t[BY_PIECE ? i : 0] = m0 + m < a.n_st ? a.t[m0 + m] : -1;
        }
        if (BY_WAVE) {
            const int m = m0 + (lane & (TM - 1));
            next_gone = m < a.n_st && (MODE == LOSS_GRAD ? a.t[m] < 0 : a.bias[m] * 1.44269504f == -INFINITY);
        }
        if (threadIdx.x < TM) {
            const int m = m0 + threadIdx.x;
            const bool in = m < a.n_st;
            if (MODE == LOSS_GRAD) {
                next_side[0] = in ? a.nlse[m] + g_log : -INFINITY;
                next_side[1] = in ? a.gt[m] * g_scale : -0.f;
                next_side[2] = __int_as_float(in ? a.t[m] : -1);
            } else
                next_side[0] = !in ? -INFINITY : (BIAS ? a.bias[m] * 1.44269504f : 0.f);
        }
    };
    auto place = [&](int buf) {
        const uint64_t gone = BY_WAVE ? __ballot(next_gone) : 0; // (tiles of 32: both halves alike)
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int piece = i * THREADS + threadIdx.x, m = piece / (DP / 8), p = piece % (DP / 8);
            v8 o[P];
            if (BY_PIECE)
                next[i] = loss_clear(next[i], next_t[BY_PIECE ? i : 0] < 0);
            else if (gone != 0)
                next[i] = loss_clear(next[i], (gone >> m) & 1);
            loss_planes<HOW>(next[i], st_scale, o);
#pragma unroll
            for (int k = 0; k < P; ++k)
                if (PIECES % THREADS == 0 || piece < PIECES)
                    *(v8 *)&tiles[buf * TILE + k * PLANE + m * DP * 2 + (p ^ loss_swizzle<DP>(m)) * 16] = o[k];
        }
        if (threadIdx.x < TM) {
            side[buf][0][threadIdx.x] = next_side[0];
            if (MODE == LOSS_GRAD) {
                side[buf][1][threadIdx.x] = next_side[1];
                side[buf][2][threadIdx.x] = next_side[2];
            }
        }
    };

    // where this lane reads in a tile: for Z 16 bytes of row ln; for O 16 lanes take 4 rows of 16 columns, and each gets its column's 4 values
    uint32_t z_at[KS], o_at[DS][2];
#pragma unroll
    for (int k = 0; k < KS; ++k)
        z_at[k] = ln * DP * 2 + ((k * 2 + half) ^ loss_swizzle<DP>(ln)) * 16;
#pragma unroll
    for (int d = 0; d < DS; ++d)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int m = u * 8 + half * 4 + ((lane & 15) >> 2), p = (share * DS + d) * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
            o_at[d][u] = m * DP * 2 + (p ^ loss_swizzle<DP>(m)) * 16 + (lane & 1) * 8;
        }
    LOSS_LDS(char) *const lds = (LOSS_LDS(char) *)tiles;

    loss_f16v o[NB][HAS_O ? DS : 1];
    // Forward: 2^(Z - ref) is what is summed.  Gradient: sum is that of P.
    float ref[NB], sum[NB], rounded[NB];
    // Gradient, P as two fp16 numbers: every class has a power of two of its own, which falls when its P grow, and keeps all digits of its sum beside
    // others' of any size (a step of 2048 x 1 000 000 x 32 1740 us, 1665 with one power for all, where P below 2^-39 of the largest was lost).
    float up[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int d = 0; d < (HAS_O ? DS : 1); ++d)
            o[b][d] = (loss_f16v)(0.f);
        ref[b] = -3.402823466e38f;
        sum[b] = rounded[b] = 0.f;
        up[b] = 0x1p120f;
    }
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
        const bool biased = BIAS || (tl + 1) * (int64_t)TM > a.n_st; // forward: also where the last tile has fewer rows
#pragma unroll 1
        for (int sb = 0; sb < TM / 32; ++sb) {
            if (MODE != LOSS_GRAD && a.spread && ((tl * (TM / 32) + sb) & (LOSS_WAVES - 1)) != wave)
                continue;
            // Z: element i is streamed row 8 (i / 4) + 4 half + i % 4 and held row ln.  One held block after the other: a matrix instruction that
            // waits for the one before leaves the vector unit to the SIMD's other waves, one that waits for the matrix unit does not
            // (24 of them, then 200 vector instructions: 515 ns in one chain and 577 in two at two waves per SIMD, 503 and 544 at four).
            loss_f16v z[NB];
            auto streamed = [&](int k, v8 (&x)[P]) {
#pragma unroll
                for (int p = 0; p < P; ++p)
                    x[p] = *(LOSS_LDS(const v8) *)(lds + (z_at[k] + buf * TILE) + (p * PLANE + sb * 32 * DP * 2));
            };
            v8 x[NB > 1 ? KS : 1][P];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                loss_f16v less = (loss_f16v)(0.f);
                z[b] = (loss_f16v)(0.f);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    v8(&xk)[P] = x[NB > 1 ? k : 0];
                    if (b == 0)
                        streamed(k, xk);
                    loss_score<HOW, KS>(xk, q[b][k], z[b], less);
                }
                if (loss_apart<HOW, KS>())
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        z[b][i] += less[i];
            }
            float pr[NB][16];
            bool again = false;
            const float *sd = &side[buf][0][sb * 32 + half * 4];
            if (MODE == LOSS_GRAD) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const loss_f4 nl = *(const loss_f4 *)(sd + j * 8);
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            pr[b][j * 4 + e] = __builtin_amdgcn_exp2f(fmaf(z[b][j * 4 + e], c[b], BIAS ? own_bias[b] + nl[e] : nl[e]));
                }
                // A target in this wave's classes, or a gradient below 0: seldom.  P of a target is gloss (p - 1), of the other sign than gloss also where it
                // is 0; p - 1 has been found before, as the exponential here and 1 would leave nothing of it in a row that is sure of its target.
                const int32_t mine = __float_as_int(side[buf][2][sb * 32 + ln]);
                const bool mine_hit = mine >= first && mine < first + 32 * NB;
                const bool seldom = __any(mine_hit || __float_as_int(side[buf][1][sb * 32 + ln]) >= 0);
                if (seldom) {
                    again = __any(mine_hit);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const loss_f4 gt = *(const loss_f4 *)(sd + TM + j * 8), t = *(const loss_f4 *)(sd + 2 * TM + j * 8);
#pragma unroll
                        for (int b = 0; b < NB; ++b)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float v = pr[b][j * 4 + e];
                                pr[b][j * 4 + e] = __float_as_int(t[e]) == first + b * 32 + ln ? gt[e] : __float_as_int(gt[e]) >= 0 ? -v : v;
                            }
                    }
                }
                bool over = false;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const float some = loss_sum(pr[b]);
                    sum[b] += some;
                    if (MOVES)
                        over = over || !((seldom ? loss_sum_abs(pr[b]) : some) * up[b] < H::MOST);
                }
                if (MOVES && __any(over)) {
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        float most = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            most = fmaxf(most, fabsf(pr[b][i]));
                        most = fmaxf(most, __shfl_xor(most, 32, 64));
                        const float to = fminf(up[b], __builtin_amdgcn_ldexpf(1.f, H::SHIFT - __builtin_amdgcn_frexp_expf(most)));
                        const float f = to / up[b];
                        up[b] = to;
#pragma unroll
                        for (int d = 0; d < (HAS_O ? DS : 1); ++d)
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                o[b][d][i] *= f;
                    }
                }
            } else {
                // The target's score goes out by itself, and is minus infinity from here on (c is never 0).  It has no part in sum and mean, nor in
                // the reference: 2^10 above the others' largest, as in a row that is sure of its target, it would leave their powers
                // fewer fp16 bits, and none from 2^35 on.
                bool hit = false;
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    hit = hit || (unsigned)(target[b] - tl * TM - sb * 32) < 32u;
                if (__any(hit)) {
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        const int at = target[b] - tl * TM - sb * 32;
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (8 * (i / 4) + 4 * half + i % 4 == at) {
                                if (share == 0)
                                    a.zt[first + b * 32 + ln] = fmaf(z[b][i], c[b], sd[i / 4 * 8 + i % 4]);
                                z[b][i] = -INFINITY;
                            }
                    }
                }
                float some[NB];
                auto powers = [&](int b) {
                    const float off = ref[b] - (float)H::SHIFT;
                    if (biased) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const loss_f4 bs = *(const loss_f4 *)(sd + j * 8);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                pr[b][j * 4 + e] = __builtin_amdgcn_exp2f(fmaf(z[b][j * 4 + e], c[b], bs[e] - off));
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            pr[b][i] = __builtin_amdgcn_exp2f(fmaf(z[b][i], c[b], -off));
                    }
                    some[b] = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        some[b] += pr[b][i];
                };
                bool over = false;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    powers(b);
                    over = over || !(some[b] < H::MOST);
                }
                if (__any(over)) { // a held row's reference (both halves of its lanes) moves to the maximum of its scores so far
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        const bool moves = !(fmaxf(some[b], __shfl_xor(some[b], 32, 64)) < H::MOST) || some[b] != some[b];
                        float to = ref[b];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const loss_f4 bs = *(const loss_f4 *)(sd + j * 8);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                to = fmaxf(to, fmaf(z[b][j * 4 + e], c[b], bs[e]));
                        }
                        const float pair = fmaxf(to, __shfl_xor(to, 32, 64));
                        to = moves ? pair : ref[b];
                        const float f = __builtin_amdgcn_exp2f(ref[b] - to);
                        ref[b] = to;
                        sum[b] *= f;
                        rounded[b] *= f;
                        if (HAS_O) {
#pragma unroll
                            for (int d = 0; d < DS; ++d)
#pragma unroll
                                for (int i = 0; i < 16; ++i)
                                    o[b][d][i] *= f;
                        }
                        powers(b);
                    }
                }
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    sum[b] += some[b];
            }
            if (HAS_O) {
                // Eight streamed rows of a lane are the eight of an operand: rows 16 t + 4 half + {0..3, 8..11}.  P enters O as one number of the types of 16
                // bits, off by up to half a step of itself; a second one for all would double O's matrix instructions.  But what a row leaves to its target
                // is most of a class's gradient, and a target is in few blocks: these enter the gradient's O once more, with what the rounding has taken.
                // gw of 16 384 x 100 003 x 64 bf16 is then 1.66e-3 off its definition in norm, as if rounded once (2.4e-3 without), 3001 x 40 009 x 100
                // fp16 2.1e-4 (2.8e-4), for 1 % of these steps and 1 to 5 % where every block has a target (16 384 x 512 to 16 384 x 64).
                v8 pb[NB][2][P];
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        float v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            v[e] = pr[b][t * 8 + e];
                        loss_split<HOW, MOVES>(v, pb[b][t], up[b]);
                    }
                // P loses up to half a step of its type here: O is then divided by the sum of what P has become, so that what all rows have in common
                // stays (dot products with ones: 30 us of the 1130 of a step of 16 384 x 100 003 x 64 bf16).
                if constexpr (ROUNDED) {
                    if (share == 0) {
#pragma unroll
                        for (int b = 0; b < NB; ++b)
                            rounded[b] += loss_add(pb[b][1][0], loss_add(pb[b][0][0], 0.f));
                    }
                }
                auto products = [&]() {
#pragma unroll
                    for (int d = 0; d < DS; ++d) {
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            v8 x[P];
#pragma unroll
                            for (int p = 0; p < P; ++p) {
                                s4 w[2];
#pragma unroll
                                for (int u = 0; u < 2; ++u)
                                    w[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                        (LOSS_LDS(s4) *)(lds + (o_at[d][u] + buf * TILE) + (p * PLANE + (sb * 32 + t * 16) * DP * 2)));
                                x[p] = __builtin_shufflevector(__builtin_bit_cast(v4, w[0]), __builtin_bit_cast(v4, w[1]), 0, 1, 2, 3, 4, 5, 6, 7);
                            }
#pragma unroll
                            for (int b = 0; b < NB; ++b)
#pragma unroll
                                for (int u = 6 - NP; u < 6; ++u)
                                    o[b][d] = loss_mfma(x[LOSS_PA[u]], pb[b][t][LOSS_PB[u]], o[b][d]);
                        }
                    }
                };
                products();
                if constexpr (MODE == LOSS_GRAD && P == 1) {
                    if (again) {
#pragma unroll
                        for (int b = 0; b < NB; ++b)
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                pb[b][i / 8][0][i % 8] = (E)(pr[b][i] - (float)pb[b][i / 8][0][i % 8]);
                        products();
                    }
                }
            }
        }
        if (more)
            place(buf ^ 1);
        __syncthreads();
    }

#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int n = first + b * 32 + ln;
        const float all = sum[b] + __shfl_xor(sum[b], 32, 64), all_rounded = ROUNDED ? rounded[b] + __shfl_xor(rounded[b], 32, 64) : 0.f;
        const int64_t at = (int64_t)(MODE != LOSS_GRAD && a.spread ? split * LOSS_WAVES + wave : split) * a.n_own + n;
        const bool direct = MODE == LOSS_GRAD && a.n_split == 1;
        if (n < a.n_own && half == 0 && share == 0) {
            if (MODE != LOSS_GRAD) {
                a.stat[at * 2] = ref[b] - (float)H::SHIFT;
                a.stat[at * 2 + 1] = all;
                if (ROUNDED)
                    a.psum[at] = all_rounded;
            } else if (!direct && a.psum)
                a.psum[at] = MOVES ? all : all / g_scale;
            else if (direct && a.out_sum)
                a.out_sum[n] = MOVES ? all : all / g_scale;
        }
        if (HAS_O && n < a.n_own && (direct ? a.out != nullptr : a.part != nullptr)) {
            const float f = MODE == LOSS_GRAD ? (direct ? a.scale : 1.f) / g_scale : 1.f;
#pragma unroll
            for (int d = 0; d < DS; ++d) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int col = (share * DS + d) * 32 + j * 8 + half * 4;
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = MOVES ? __builtin_amdgcn_ldexpf(o[b][d][j * 4 + e] * f, 1 - __builtin_amdgcn_frexp_expf(up[b]) - st_up) : o[b][d][j * 4 + e] * back * f;
                    if (!direct) {
                        if (col < a.pitch)
                            *(loss_f4 *)(a.part + at * a.pitch + col) = loss_f4{v[0], v[1], v[2], v[3]};
                    } else {
                        fae_place<4> p;
                        p.set(col, a.width);
                        fae_store<T, 4, FAE_ANY>((T *)a.out + (int64_t)n * a.out_stride, v, p);
                    }
                }
            }
        }
    }
}

// Few rows (serving, small test batches; sums in fp32 alone, so the target may move the reference here): bound by reading w, so that every wave
// takes a stretch of classes of its own, straight from memory to the matrix instructions' registers with the next 32 on their way, and
// no wave waits for another before the end.  1 x 200 003 x 64 fp32
// 14 to 16 us, 48 x 1 000 003 x 32 47 us, 2.7 TB/s.  When it was built it took 16.8 and 41 (the kernel above: 25 and 106, three of its waves
// without rows; two steps ahead: 17.4 and 43.6; three waves per SIMD, which spill: 20.5 and 46.6).
template <int HOW, int DP, int NB, bool BIAS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(loss_planes_of(HOW) * DP <= 192 ? 2 : 1))) void loss_few_kernel(loss_args a)
{
    typedef loss_type<HOW> H;
    typedef typename H::T T;
    typedef typename loss_vec<typename H::E>::v8 v8;
    constexpr int P = H::PLANES, KS = DP / 16;
    __shared__ float parts[4][2][NB * 32];
    const int lane = fae_lane(), wave = threadIdx.x / 64, ln = lane & 31, half = lane >> 5;
    const uint32_t split = blockIdx.x / a.n_blocks, block = blockIdx.x % a.n_blocks;
    const int64_t strides = (int64_t)a.n_split * 4, mine = (int64_t)split * 4 + wave;
    const int tile0 = (int)(a.tiles * mine / strides), tile1 = (int)(a.tiles * (mine + 1) / strides); // of 32 classes
    const int first = (int)block * 32 * NB;

    loss_raw<T> next[KS];
    loss_f4 next_bias[4];
    bool next_gone = false;
    auto fetch = [&](int tl) {
        const int m = tl * 32 + ln;
#pragma unroll
        for (int k = 0; k < KS; ++k)
            next[k] = loss_load_ends<T>((const T *)a.st + (int64_t)m * a.st_stride, k * 16 + half * 8, a.width, tl < tile1 && m < a.n_st);
        next_gone = BIAS && tl < tile1 && m < a.n_st && a.bias[m] * 1.44269504f == -INFINITY; // such a class may hold anything
        if (BIAS && tl < tile1 && (tl + 1) * 32LL <= a.n_st)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                next_bias[j] = *(const typename fae_vec<float, 4>::loose *)(a.bias + tl * 32 + j * 8 + half * 4);
    };
    fetch(tile0);
    v8 q[NB][KS][P];
    int32_t target[NB];
    float ref[NB], sum[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int n = first + b * 32 + ln;
        const bool there = n < a.n_own;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            loss_raw<T> x = loss_load<T>((const T *)a.own + (int64_t)n * a.own_stride, k * 16 + half * 8, a.width, there);
            if (a.flip) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x.v[e] = -x.v[e];
            }
            loss_planes<HOW>(x, 1.f, q[b][k]);
        }
        target[b] = there ? loss_target(a.targets, a.target_bits, n, a.n_classes, a.status) : -1;
        ref[b] = -3.402823466e38f;
        sum[b] = 0.f;
    }
    for (int tl = tile0; tl < tile1; ++tl) {
        v8 x[KS][P];
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            if (BIAS)
                next[k] = loss_clear(next[k], next_gone);
            loss_planes<HOW>(next[k], 1.f, x[k]);
        }
        float bias[16];
        if ((tl + 1) * 32LL > a.n_st) { // the last 32 are fewer
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int m = tl * 32 + i / 4 * 8 + half * 4 + i % 4;
                bias[i] = m >= a.n_st ? -INFINITY : (BIAS ? a.bias[m] * 1.44269504f : 0.f);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                bias[i] = BIAS ? next_bias[i / 4][i % 4] * 1.44269504f : 0.f;
        }
        fetch(tl + 1);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            loss_f16v z = (loss_f16v)(0.f), less = (loss_f16v)(0.f);
#pragma unroll
            for (int k = 0; k < KS; ++k)
                loss_score<HOW, KS>(x[k], q[b][k], z, less);
            if (loss_apart<HOW, KS>())
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    z[i] += less[i];
            float some;
            auto powers = [&]() {
                some = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    some += __builtin_amdgcn_exp2f(fmaf(z[i], a.c, bias[i] - ref[b]));
            };
            powers();
            if (__any(!(some < loss_type<HOW>::MOST))) { // the reference moves to the maximum of the lane's scores so far
                float to = ref[b];
                const bool moves = !(some < loss_type<HOW>::MOST);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    to = fmaxf(to, fmaf(z[i], a.c, bias[i]));
                to = moves ? to : ref[b];
                sum[b] *= __builtin_amdgcn_exp2f(ref[b] - to);
                ref[b] = to;
                powers();
            }
            const int at = target[b] - tl * 32;
            if (__any((unsigned)at < 32u)) { // the target's score goes out by itself
                some = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float v = fmaf(z[i], a.c, bias[i]);
                    if (8 * (i / 4) + 4 * half + i % 4 == at)
                        a.zt[first + b * 32 + ln] = v;
                    else
                        some += __builtin_amdgcn_exp2f(fmaf(z[i], a.c, bias[i] - ref[b]));
                }
            }
            sum[b] += some;
        }
    }
    // the two halves of a wave, then the four waves, at the largest reference
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const float other = __shfl_xor(ref[b], 32, 64), to = fmaxf(ref[b], other);
        sum[b] *= __builtin_amdgcn_exp2f(ref[b] - to);
        sum[b] += __shfl_xor(sum[b], 32, 64);
        if (half == 0) {
            parts[wave][0][b * 32 + ln] = to;
            parts[wave][1][b * 32 + ln] = sum[b];
        }
    }
    __syncthreads();
    const int n = first + threadIdx.x;
    if (threadIdx.x < NB * 32 && n < a.n_own) {
        float to = parts[0][0][threadIdx.x], all = 0.f;
#pragma unroll
        for (int w = 1; w < 4; ++w)
            to = fmaxf(to, parts[w][0][threadIdx.x]);
#pragma unroll
        for (int w = 0; w < 4; ++w)
            all += parts[w][1][threadIdx.x] * __builtin_amdgcn_exp2f(parts[w][0][threadIdx.x] - to);
        const int64_t at = (int64_t)split * a.n_own + n;
        a.stat[at * 2] = to;
        a.stat[at * 2 + 1] = all;
    }
}

template <int HOW, int DP, bool BIAS> static void loss_launch_mode(fae_ctx *ctx, int mode, const loss_args &a)
{
    const dim3 grid(a.n_blocks * a.n_split), block(LOSS_WAVES * 64), block_o(LOSS_WAVES * 64 * loss_shares(HOW, DP, LOSS_MEAN));
    if constexpr (HOW != LOSS_F32_WIDE) {
        if (mode == LOSS_FEW) {
            if (a.n_own <= 32 || loss_few_blocks(HOW, DP) == 1)
                FAE_LAUNCH(ctx, (loss_few_kernel<HOW, DP, 1, BIAS>), grid, block, 0, ctx->stream, a);
            else
                FAE_LAUNCH(ctx, (loss_few_kernel<HOW, DP, loss_few_blocks(HOW, DP), BIAS>), grid, block, 0, ctx->stream, a);
            return;
        }
    }
    if constexpr (HOW != LOSS_F32 || DP <= LOSS_F32_WIDTH) {
        if (mode == LOSS_STATS)
            FAE_LAUNCH(ctx, (loss_kernel<HOW, DP, LOSS_STATS, BIAS>), grid, block, 0, ctx->stream, a);
        else if (mode == LOSS_MEAN)
            FAE_LAUNCH(ctx, (loss_kernel<HOW, DP, LOSS_MEAN, BIAS>), grid, block_o, 0, ctx->stream, a);
        else if constexpr (HOW != LOSS_F32)
            FAE_LAUNCH(ctx, (loss_kernel<HOW, DP, LOSS_GRAD, BIAS>), grid, block_o, 0, ctx->stream, a);
    }
}
template <int HOW, int DP> static void loss_launch_bias(fae_ctx *ctx, int mode, const loss_args &a)
{
    if (a.bias)
        loss_launch_mode<HOW, DP, true>(ctx, mode, a);
    else
        loss_launch_mode<HOW, DP, false>(ctx, mode, a);
}
template <int HOW> static void loss_launch(fae_ctx *ctx, int mode, const loss_args &a)
{
    switch (loss_padded(a.width)) {
    case 32: return loss_launch_bias<HOW, 32>(ctx, mode, a);
    case 64: return loss_launch_bias<HOW, 64>(ctx, mode, a);
    case 96: return loss_launch_bias<HOW, 96>(ctx, mode, a);
    case 128: return loss_launch_bias<HOW, 128>(ctx, mode, a);
    case 192: return loss_launch_bias<HOW, 192>(ctx, mode, a);
    default: return loss_launch_bias<HOW, 256>(ctx, mode, a);
    }
}

#endif // LOSS_KERNELS
