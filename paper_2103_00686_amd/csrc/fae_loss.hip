// Softmax cross entropy over the rows of a table: checks, workspaces, and the kernels over single rows.
#include <math.h>

#include "fae_loss.h"

#define LOSS_ROUNDS 4   // workgroups of a launch that is shared out, in rounds of as many as the chip holds, at most
#define LOSS_SLOTS 512  // workgroups that the chip holds with two waves per SIMD
#define LOSS_MOST 0x7fff0000LL
#define LOSS_MOST_SHARED ((1LL << 30) - 127) // of held rows whose columns two waves share: 512 threads for 128 of them, fewer than 2^32 in all
#define LOSS_GRID (1 << 20) // workgroups of a kernel over rows at most: a grid holds fewer than 2^32 threads
#define LOSS_WIDE_ROWS 128
#define LOSS_WIDE_SCORES (1LL << 24)

// ---------------------------------------------------------------------------------
// kernels
// ---------------------------------------------------------------------------------
struct LossJoin {
    const float *stat, *zt, *part, *psum; // psum: NULL where it is what stat has
    const void *targets, *w;
    int64_t w_stride;
    int32_t type;
    float *loss, *lse, *mean;
    int32_t target_bits, n_classes, width, pitch;
    int64_t n_rows;
    uint32_t n_split, lanes; // lanes: of a part's row, a power of two
    uint32_t *status;
};

__device__ __forceinline__ float loss_value(const void *p, int32_t type, int64_t i)
{
    return type == FAE_F32 ? ((const float *)p)[i] : type == FAE_BF16 ? (float)((const fae_bf16 *)p)[i] : (float)((const fae_f16 *)p)[i];
}

// W waves per row: the parts' sums at one reference, loss and lse, and the weighted sum of the parts' means.  One wave is a chain of as many
// loads as there are parts: the small kernels of a step of 12 x 100 000 x 64 bf16 take 191 us together with one, 22 with 16.
template <int W> __global__ __launch_bounds__(W == 1 ? 256 : W * 64) void loss_join_kernel(LossJoin a)
{
    __shared__ float part[W][64 * 4];
    const int lane = fae_lane(), wave = W == 1 ? 0 : threadIdx.x / 64;
    auto over_waves = [&](float v, bool most) {
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const float o = __shfl_xor(v, d, 64);
            v = most ? fmaxf(v, o) : v + o;
        }
        if (W > 1) {
            __syncthreads();
            if (lane == 0)
                part[wave][0] = v;
            __syncthreads();
            v = part[0][0];
            for (int w = 1; w < W; ++w)
                v = most ? fmaxf(v, part[w][0]) : v + part[w][0];
        }
        return v;
    };
    for (int64_t r = W == 1 ? (int64_t)blockIdx.x * 4 + threadIdx.x / 64 : blockIdx.x; r < a.n_rows; r += (int64_t)gridDim.x * (W == 1 ? 4 : 1)) {
        float most = -INFINITY;
        for (uint32_t i = wave * 64 + lane; i < a.n_split; i += W * 64)
            most = fmaxf(most, a.stat[(i * a.n_rows + r) * 2]);
        most = over_waves(most, true);
        const int32_t t = loss_target(a.targets, a.target_bits, r, a.n_classes, a.status);
        const float zt = t < 0 ? -INFINITY : a.zt[r];
        most = fmaxf(most, zt); // the parts' references are the other classes'
        float sum = 0.f;
        for (uint32_t i = wave * 64 + lane; i < a.n_split; i += W * 64)
            sum += a.stat[(i * a.n_rows + r) * 2 + 1] * __builtin_amdgcn_exp2f(a.stat[(i * a.n_rows + r) * 2] - most);
        sum = over_waves(sum, false);
        // All classes but the target are in sum: what a confident row leaves to them keeps its digits.
        const float pt = t < 0 ? 0.f : __builtin_amdgcn_exp2f(zt - most), all = sum + pt;
        const float l2 = most + __log2f(all);
        if (lane == 0 && wave == 0) {
            if (a.lse)
                a.lse[r] = l2 * 0.693147181f;
            if (a.loss)
                a.loss[r] = t < 0 || all == 0.f ? 0.f : sum < pt ? log1pf(sum / pt) : (l2 - zt) * 0.693147181f;
        }
        if (!a.mean)
            continue;
        // The parts' means over the sum of the same rounded powers are the other classes' mean row, and what all rows have in common is in it once,
        // however the powers were rounded: their errors count by how far a row is from that mean.
        float even = 1.f;
        if (a.psum) {
            float rest = 0.f;
            for (uint32_t i = wave * 64 + lane; i < a.n_split; i += W * 64)
                rest += a.psum[i * a.n_rows + r] * __builtin_amdgcn_exp2f(a.stat[(i * a.n_rows + r) * 2] - most);
            rest = over_waves(rest, false);
            even = rest > 0.f ? sum / rest : 1.f;
        }
        const int col = (lane % a.lanes) * 4;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (col < a.pitch)
            for (uint32_t i = lane / a.lanes + wave * (64 / a.lanes); i < a.n_split; i += 64 / a.lanes * W) {
                const float f = __builtin_amdgcn_exp2f(a.stat[(i * a.n_rows + r) * 2] - most);
                const float4 p = *(const float4 *)(a.part + (i * a.n_rows + r) * a.pitch + col);
                v[0] += f * p.x;
                v[1] += f * p.y;
                v[2] += f * p.z;
                v[3] += f * p.w;
            }
        for (uint32_t d = a.lanes; d < 64; d <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] += __shfl_xor(v[e], d, 64);
        if (W > 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 4; ++e)
                part[wave][lane * 4 + e] = v[e];
            __syncthreads();
            for (int w = 1; w < W; ++w)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = (w == 1 ? part[0][lane * 4 + e] : v[e]) + part[w][lane * 4 + e];
        }
        if (lane < (int)a.lanes && wave == 0)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < a.width) {
                    const float wt = t < 0 || sum == 0.f ? 0.f : loss_value(a.w, a.type, t * a.w_stride + col + e);
                    a.mean[r * a.width + col + e] = all == 0.f ? 0.f : (v[e] * even - sum * wt) / all;
                }
    }
}

struct LossRows {
    const void *x, *targets;
    void *gx;
    int64_t x_stride, gx_stride, n_rows;
    const float *lse, *loss, *mean, *gloss, *bias; // loss: NULL if the caller has not kept it
    const void *w;
    int64_t w_stride;
    float *nlse, *gt; // NULL: gx alone
    int32_t *t;
    float *g_most, *x_most; // a value for every workgroup
    int32_t target_bits, n_classes, width;
    float scale;
    uint32_t *status;
};

#define LOSS_MOSTS 2048 // workgroups that look for a largest value, and slots for what they find

// the workgroup's largest value into its slot
__device__ __forceinline__ void loss_most_of(float v, float *slot)
{
    __shared__ float part[4];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1)
        v = fmaxf(v, __shfl_xor(v, d, 64));
    __syncthreads();
    if (fae_lane() == 0)
        part[threadIdx.x / 64] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        *slot = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}
// (of finite values)
__device__ __forceinline__ float loss_most(float most, float v)
{
    v = fabsf(v);
    return v < INFINITY ? fmaxf(most, v) : most;
}

// The largest value of all rows of fp32 (of classes that are offered).  Bound by memory.
__global__ __launch_bounds__(256) void loss_most_kernel(const float *w, int64_t stride, int64_t n, int32_t width, const float *bias, float *slots)
{
    float most = 0.f;
    const uint32_t per = ((uint32_t)width + 3) / 4, lanes = per <= 1 ? 1 : 1u << (32 - __clz(per - 1)); // lanes of a row, 4 values each
    const uint32_t rows = 256 / lanes;
    fae_place<4> at;
    at.set((threadIdx.x % lanes) * 4, width);
    for (int64_t r = (int64_t)blockIdx.x * rows + threadIdx.x / lanes; r < n; r += (int64_t)gridDim.x * rows) {
        if (bias && bias[r] * 1.44269504f == -INFINITY)
            continue;
        const float *row = w + r * stride;
        if (width >= 4) {
            const auto v = *(const typename fae_vec<float, 4>::loose *)(row + at.from);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                most = loss_most(most, v[e]);
        } else
            for (int e = 0; e < width; ++e)
                most = loss_most(most, row[e]);
    }
    loss_most_of(most, slots + blockIdx.x);
}

// A wave per row: gx from what the forward has kept, and what the classes' gradient reads of every row.
template <typename T> __global__ __launch_bounds__(256) void loss_rows_kernel(LossRows a)
{
    const int lane = fae_lane();
    float g_most = 0.f, x_most = 0.f;
    for (int64_t r = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; r < a.n_rows; r += (int64_t)gridDim.x * 4) {
        int32_t t = loss_target(a.targets, a.target_bits, r, a.n_classes, a.status);
        const float lse = a.lse[r];
        if (lse == -INFINITY) // no class is offered
            t = -1;
        const float g = t < 0 ? 0.f : a.gloss[r];
        g_most = loss_most(g_most, g);
        if (a.gt) {
            // 1 - p of the target is 1 - exp(-loss); without the loss, from lse and the target's score, whose digits end at lse's
            float loss = 0.f;
            if (t >= 0) {
                if (a.loss)
                    loss = a.loss[r];
                else {
                    float z = 0.f;
                    for (int c = lane; c < a.width; c += 64)
                        z = fmaf((float)((const T *)a.x)[r * a.x_stride + c], (float)((const T *)a.w)[t * a.w_stride + c], z);
#pragma unroll
                    for (int d = 32; d > 0; d >>= 1)
                        z += __shfl_xor(z, d, 64);
                    loss = lse - (a.scale * z + (a.bias ? a.bias[t] : 0.f));
                    loss = loss < 0.f ? 0.f : loss;
                }
            }
            if (lane == 0) {
                a.nlse[r] = t < 0 ? -INFINITY : __log2f(fabsf(g)) - lse * 1.44269504f;
                a.gt[r] = t < 0 ? -0.f : copysignf(g * expm1f(-loss), -g); // (expm1f loses the sign of 0)
                a.t[r] = t;
            }
        }
        for (int c = lane; c < a.width; c += 64) {
            if (a.x_most && t >= 0)
                x_most = loss_most(x_most, (float)((const T *)a.x)[r * a.x_stride + c]);
            if (a.gx)
                ((T *)a.gx)[r * a.gx_stride + c] = (T)(t < 0 ? 0.f : a.scale * g * a.mean[r * a.width + c]);
        }
    }
    if (a.g_most)
        loss_most_of(g_most, a.g_most + blockIdx.x);
    if (a.x_most)
        loss_most_of(x_most, a.x_most + blockIdx.x);
}

struct LossClasses {
    const float *part, *psum;
    void *gw;
    float *gbias;
    int64_t gw_stride, n_classes;
    uint32_t n_split;
    int32_t width, pitch;
    float scale;
};

// G threads per four values of a class, each with every G-th part: the sum of the parts.  One thread is a chain of as many loads as there are
// parts: the small kernels of a step of 12 000 x 300 x 64 bf16 take 66 us together with one, 22 with 16.
template <typename T, int G> __global__ __launch_bounds__(256) void loss_classes_kernel(LossClasses a)
{
    constexpr int OUT = 256 / G;
    __shared__ float some[G][OUT][5];
    const int per = a.pitch / 4, out = threadIdx.x % OUT, group = threadIdx.x / OUT;
    const int64_t i = (int64_t)blockIdx.x * OUT + out, n = i / per;
    const int col = (int)(i - n * per) * 4;
    float v[5] = {0.f, 0.f, 0.f, 0.f, 0.f}; // four values, and the bias's sum with the first of a class
    if (n < a.n_classes) {
        if (a.gw)
#pragma unroll 4
            for (uint32_t s = group; s < a.n_split; s += G) {
                const float4 p = *(const float4 *)(a.part + (s * a.n_classes + n) * a.pitch + col);
                v[0] += p.x;
                v[1] += p.y;
                v[2] += p.z;
                v[3] += p.w;
            }
        if (a.gbias && col == 0)
            for (uint32_t s = group; s < a.n_split; s += G)
                v[4] += a.psum[s * a.n_classes + n];
    }
    if (G > 1) {
#pragma unroll
        for (int e = 0; e < 5; ++e)
            some[group][out][e] = v[e];
        __syncthreads();
        if (group != 0)
            return;
        for (int g = 1; g < G; ++g)
#pragma unroll
            for (int e = 0; e < 5; ++e)
                v[e] += some[g][out][e];
    }
    if (n >= a.n_classes)
        return;
    if (a.gw) {
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            o[e] = v[e] * a.scale;
        fae_place<4> p;
        p.set(col, a.width);
        fae_store<T, 4, FAE_ANY>((T *)a.gw + n * a.gw_stride, o, p);
    }
    if (a.gbias && col == 0)
        a.gbias[n] = v[4];
}
template <typename T> static void loss_classes(fae_ctx *ctx, const LossClasses &c)
{
    const int64_t n = c.n_classes * (c.pitch / 4);
    if (c.n_split >= 32)
        FAE_LAUNCH(ctx, (loss_classes_kernel<T, 16>), dim3((uint32_t)((n + 15) / 16)), dim3(256), 0, ctx->stream, c);
    else
        FAE_LAUNCH(ctx, (loss_classes_kernel<T, 1>), dim3((uint32_t)((n + 255) / 256)), dim3(256), 0, ctx->stream, c);
}

// ---------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------
static bool loss_sizes_fit(const fae_softmax_loss *l)
{
    return l && l->n_rows >= 0 && l->n_rows < LOSS_MOST && l->n_classes >= 1 && l->n_classes < LOSS_MOST && l->width >= 1 &&
           l->width <= FAE_LOSS_MAX_WIDTH && l->type >= FAE_F32 && l->type <= FAE_F16;
}

// fp32 as two fp16 numbers or three bf16: the first take half the matrix instructions and fewer registers, and a look at all streamed rows
// before (5 us and reading them), which few rows or scores of narrow rows do not pay for.  Steps in us, two fp16 numbers and three bf16:
// 40 x 300 000 x 100 216 and 269, 1 x 1 000 000 x 32 equal, 300 x 5003 x 16 41 and 39, 2048 x 1 000 000 x 32 1730 and 2860.
static int loss_how(const fae_softmax_loss *l, int mode)
{
    if (l->type != FAE_F32)
        return l->type == FAE_BF16 ? LOSS_BF16 : LOSS_F16;
    if (mode == LOSS_FEW)
        return LOSS_F32;
    const bool pays = l->width > LOSS_F32_WIDTH || (l->n_rows >= LOSS_WIDE_ROWS && l->n_rows * l->n_classes >= LOSS_WIDE_SCORES);
    return mode == LOSS_GRAD || pays ? LOSS_F32_WIDE : LOSS_F32;
}

// n_own held rows in workgroups of some, n_st streamed rows shared out among as many of them as fill the chip
struct LossShape {
    int how;
    int64_t blocks, tiles, splits;
    int32_t pitch, held;
};
static LossShape loss_shape(const fae_softmax_loss *l, int mode)
{
    LossShape s;
    const int64_t n_own = mode == LOSS_GRAD ? l->n_classes : l->n_rows, n_st = mode == LOSS_GRAD ? l->n_rows : l->n_classes;
    s.how = loss_how(l, mode);
    const int dp = loss_padded(l->width);
    const int tile = mode == LOSS_FEW ? 32 : loss_tile(s.how, dp);
    const int held = mode != LOSS_FEW ? loss_held(s.how, dp, mode) : n_own <= 32 ? 32 : 32 * loss_few_blocks(s.how, dp);
    s.held = held;
    s.blocks = (n_own + held - 1) / held;
    s.tiles = (n_st + tile - 1) / tile;
    s.splits = 1;
    if (mode == LOSS_FEW) {
        s.splits = s.blocks ? LOSS_FEW_GROUPS / s.blocks : 1;
        s.splits = s.splits > s.tiles ? s.tiles : s.splits;
    } else if (s.blocks > 0) {
        // The parts that leave the fewest places empty in the last round, less what putting them together takes: reading and writing a part's
        // row, at 4 TB/s, beside a score's 0.1 + 0.007 dp ps (both as measured).  24 blocks in 16 parts leave a quarter of the chip empty,
        // in 40 6 %: 3001 x 40 009 x 100 fp16 forward 137 and 116 us; 391 blocks in one part the same, in five 5 %: the gradient
        // of 16 384 x 100 003 x 64 bf16 666 and 577 us.
        const double slots = LOSS_SLOTS / 2 * loss_waves(s.how, dp, mode) / loss_shares(s.how, dp, mode);
        double best = 0.0;
        for (int64_t p = 1; p <= s.tiles && (p == 1 || s.blocks * p <= LOSS_ROUNDS * LOSS_SLOTS); p += p >= 8 ? 8 : 1) { // (8: loss_kernel)
            const double rounds = s.blocks * p / slots, most = ceil(rounds);
            const double join = mode == LOSS_GRAD && p == 1 ? 0.0 : 2.0 * p * l->width / (n_st * (0.1 + 0.007 * dp));
            const double good = rounds / most / (1.0 + join);
            if (good > best * 1.001) {
                best = good;
                s.splits = p;
            }
        }
    }
    s.pitch = (l->width + 3) / 4 * 4;
    return s;
}

// held rows of a workgroup at most
static int loss_held_most(int32_t width) { return width <= 128 ? 2 * LOSS_WAVES * 32 : LOSS_WAVES * 32; }
// rows of partial results that any call up to this size would need: in a launch that is shared out, a workgroup's held rows for each workgroup
static int64_t loss_part_rows(const fae_softmax_loss *l, int mode)
{
    const int64_t n_own = mode == LOSS_GRAD ? l->n_classes : l->n_rows, n_st = mode == LOSS_GRAD ? l->n_rows : l->n_classes;
    const int64_t most = (int64_t)LOSS_ROUNDS * LOSS_SLOTS * loss_held_most(l->width);
    const int64_t tiles = (n_st + 31) / 32 * (mode == LOSS_GRAD ? 1 : LOSS_WAVES); // (forward: also a part for each wave)
    const int64_t shared = tiles == 0 ? 0 : n_own > most / tiles ? most : n_own * tiles;
    return mode == LOSS_GRAD || shared > n_own ? shared : n_own; // (the gradient in one part needs none)
}
// what the forward takes: the largest values, per part and row reference and two sums, per row the target's score, and the parts' means
static size_t loss_fwd_bytes(const fae_softmax_loss *l)
{
    const int64_t rows = loss_part_rows(l, LOSS_MEAN), pitch = (l->width + 3) / 4 * 4;
    return fae_align_up(LOSS_MOSTS * 4, 256) + fae_align_up(rows * 8, 256) + fae_align_up(rows * 4, 256) + fae_align_up(l->n_rows * 4, 256) + fae_align_up(rows * pitch * 4, 256);
}
static size_t loss_grad_bytes(const fae_softmax_loss *l)
{
    const int64_t rows = loss_part_rows(l, LOSS_GRAD), pitch = (l->width + 3) / 4 * 4;
    return fae_align_up(rows * 4, 256) + fae_align_up(rows * pitch * 4, 256);
}

extern "C" size_t fae_softmax_loss_fwd_workspace_bytes(const fae_softmax_loss *what)
{
    return loss_sizes_fit(what) ? 256 + loss_fwd_bytes(what) : 0;
}

extern "C" size_t fae_softmax_loss_bwd_workspace_bytes(const fae_softmax_loss *what)
{
    if (!loss_sizes_fit(what))
        return 0;
    const size_t f = loss_fwd_bytes(what), g = loss_grad_bytes(what);
    return 512 + 2 * fae_align_up(LOSS_MOSTS * 4, 256) + 3 * fae_align_up(what->n_rows * 4, 256) + fae_align_up(what->n_rows * what->width * 4, 256) + (f > g ? f : g);
}

// bytes that rows take up
struct LossSpan {
    const char *what;
    uintptr_t p;
    int64_t stride, row, n; // in bytes; rows
};
static LossSpan loss_span(const char *what, const void *p, int64_t stride, int64_t row, int64_t n, int size)
{
    return {what, (uintptr_t)p, stride * size, row * size, p ? n : 0};
}
static bool loss_share(const LossSpan &a, const LossSpan &b)
{
    if (!a.n || !b.n)
        return false;
    const uintptr_t a1 = a.p + (a.n - 1) * a.stride + a.row, b1 = b.p + (b.n - 1) * b.stride + b.row;
    if (a1 <= b.p || b1 <= a.p)
        return false;
    if (a.n > 1 && b.n > 1 && a.stride == b.stride) { // side by side in rows of one buffer
        const int64_t d = (int64_t)(b.p > a.p ? (b.p - a.p) % a.stride : (a.stride - (int64_t)((a.p - b.p) % a.stride)) % a.stride);
        return !(d >= a.row && d + b.row <= a.stride);
    }
    return true;
}

static int32_t loss_check(fae_ctx *ctx, const char *who, const fae_softmax_loss *l, const void *x, int64_t x_stride, const void *w, int64_t w_stride)
{
    if (!ctx)
        return FAE_EINVAL;
    if (!l)
        return fae_fail(ctx, FAE_EINVAL, "%s: null description", who);
    if (!loss_sizes_fit(l))
        return fae_fail(ctx, FAE_EINVAL, "%s: n_rows=%lld n_classes=%lld width=%d type=%d out of range", who, (long long)l->n_rows,
                        (long long)l->n_classes, l->width, l->type);
    if (!isfinite(l->scale))
        return fae_fail(ctx, FAE_EINVAL, "%s: scale=%g is not finite", who, l->scale);
    if (l->target_bits != 32 && l->target_bits != 64)
        return fae_fail(ctx, FAE_EINVAL, "%s: target_bits=%d is neither 32 nor 64", who, l->target_bits);
    if ((uintptr_t)l->bias % 4 != 0 || (uintptr_t)l->targets % (l->target_bits / 8) != 0)
        return fae_fail(ctx, FAE_EINVAL, "%s: bias or targets are not aligned to their values", who);
    if (l->n_rows > 0 && !l->targets)
        return fae_fail(ctx, FAE_EINVAL, "%s: null targets", who);
    int32_t rc = l->n_rows > 0 ? fae_check_rows(ctx, who, "x", {x, l->type, x_stride}, l->n_rows, l->width) : FAE_OK;
    if (rc == FAE_OK)
        rc = fae_check_rows(ctx, who, "w", {w, l->type, w_stride}, l->n_classes, l->width);
    return rc;
}

// no output on an input or another output
static int32_t loss_check_outputs(fae_ctx *ctx, const char *who, const LossSpan *out, int n_out, const LossSpan *in, int n_in)
{
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (loss_share(out[i], in[j]))
                return fae_fail(ctx, FAE_EINVAL, "%s: %s and %s overlap", who, out[i].what, in[j].what);
        for (int j = 0; j < i; ++j)
            if (loss_share(out[i], out[j]))
                return fae_fail(ctx, FAE_EINVAL, "%s: %s and %s overlap", who, out[i].what, out[j].what);
    }
    return FAE_OK;
}

static int32_t loss_check_ws(fae_ctx *ctx, const char *who, const void *ws, size_t bytes, size_t need)
{
    if ((uintptr_t)ws % 16 != 0)
        return fae_fail(ctx, FAE_EINVAL, "%s: the workspace is not on 16 bytes", who);
    if (!ws || bytes < need)
        return fae_fail(ctx, FAE_ENOSPC, "%s: workspace of %zu bytes, %zu needed", who, ws ? bytes : 0, need);
    return FAE_OK;
}

// a launch that sums O over columns shared by two waves (width above 128) holds half as many rows
static int32_t loss_check_held(fae_ctx *ctx, const char *who, const char *what, int64_t n, int32_t width)
{
    return width > 128 && n >= LOSS_MOST_SHARED ? fae_fail(ctx, FAE_EINVAL, "%s: %s=%lld of width %d", who, what, (long long)n, width) : FAE_OK;
}

static void loss_run(fae_ctx *ctx, int how, int mode, const loss_args &a)
{
    if (how == LOSS_F32)
        loss_launch_f32(ctx, mode, a);
    else if (how == LOSS_BF16)
        loss_launch_bf16(ctx, mode, a);
    else if (how == LOSS_F16)
        loss_launch_f16(ctx, mode, a);
    else
        loss_launch_f32_wide(ctx, mode, a);
}

static void loss_common(fae_ctx *ctx, const fae_softmax_loss *l, const LossShape &s, loss_args *a)
{
    memset(a, 0, sizeof(*a));
    a->width = l->width;
    a->flip = l->scale < 0.f;
    a->c = fabsf(l->scale) * 1.44269504f;
    a->scale = l->scale;
    a->bias = l->bias;
    a->targets = l->targets;
    a->target_bits = l->target_bits;
    a->n_classes = (int32_t)l->n_classes;
    a->status = ctx->d_block;
    a->pitch = s.pitch;
    a->tiles = (int32_t)s.tiles;
    a->n_blocks = (uint32_t)s.blocks;
    a->n_split = (uint32_t)s.splits;
}

static int32_t loss_forward(fae_ctx *ctx, const fae_softmax_loss *l, const void *x, int64_t x_stride, const void *w, int64_t w_stride, float *loss,
                            float *lse, float *mean, void *ws, size_t ws_bytes)
{
    const int mode = mean ? LOSS_MEAN : l->n_rows <= LOSS_FEW_ROWS ? LOSS_FEW : LOSS_STATS;
    const LossShape s = loss_shape(l, mode);
    fae_carver cv(ws, ws_bytes);
    loss_args a;
    loss_common(ctx, l, s, &a);
    a.st = w;
    a.own = x;
    a.st_stride = w_stride;
    a.own_stride = x_stride;
    a.n_st = (int32_t)l->n_classes;
    a.n_own = (int32_t)l->n_rows;
    float *most = cv.take<float>(LOSS_MOSTS);
    // one wave's rows: the four share the streamed rows out among themselves, and leave a part each
    a.spread = mode == LOSS_MEAN && l->n_rows <= s.held / LOSS_WAVES;
    const int64_t parts = a.spread ? s.splits * LOSS_WAVES : s.splits;
    a.stat = cv.take<float>(parts * l->n_rows * 2);
    a.zt = cv.take<float>(l->n_rows);
    a.part = mean ? cv.take<float>(parts * l->n_rows * s.pitch) : nullptr;
    a.psum = mean && loss_planes_of(s.how) == 1 ? cv.take<float>(parts * l->n_rows) : nullptr;
    if (!cv.ok)
        return fae_fail(ctx, FAE_ENOSPC, "softmax loss: workspace too small");
    if (s.how == LOSS_F32_WIDE) {
        fae_ktimer kt(ctx, FAE_K_LOSS_JOIN);
        const int64_t groups = (l->n_classes + 63) / 64;
        a.st_most = most;
        a.n_most = (int32_t)(groups < LOSS_MOSTS ? groups : LOSS_MOSTS);
        FAE_LAUNCH(ctx, loss_most_kernel, dim3(a.n_most), dim3(256), 0, ctx->stream, (const float *)w, w_stride, l->n_classes, l->width, l->bias, most);
        FAE_LAUNCH_CHECK(ctx);
    }
    {
        fae_ktimer kt(ctx, FAE_K_LOSS);
        loss_run(ctx, s.how, mode, a);
        FAE_LAUNCH_CHECK(ctx);
    }
    LossJoin j;
    memset(&j, 0, sizeof(j));
    j.stat = a.stat;
    j.zt = a.zt;
    j.w = w;
    j.w_stride = w_stride;
    j.type = l->type;
    j.part = a.part;
    j.psum = a.psum;
    j.targets = l->targets;
    j.loss = loss;
    j.lse = lse;
    j.mean = mean;
    j.target_bits = l->target_bits;
    j.n_classes = (int32_t)l->n_classes;
    j.width = l->width;
    j.pitch = s.pitch;
    j.n_rows = l->n_rows;
    j.n_split = (uint32_t)parts;
    j.lanes = 1;
    while ((int)j.lanes * 4 < s.pitch)
        j.lanes *= 2;
    j.status = ctx->d_block;
    fae_ktimer kt(ctx, FAE_K_LOSS_JOIN);
    if (parts >= 256 && l->n_rows <= 2048)
        FAE_LAUNCH(ctx, (loss_join_kernel<16>), dim3((uint32_t)l->n_rows), dim3(1024), 0, ctx->stream, j);
    else if (parts >= 16 && l->n_rows <= 8192)
        FAE_LAUNCH(ctx, (loss_join_kernel<4>), dim3((uint32_t)l->n_rows), dim3(256), 0, ctx->stream, j);
    else
        FAE_LAUNCH(ctx, (loss_join_kernel<1>), dim3((uint32_t)((l->n_rows + 3) / 4 < LOSS_GRID ? (l->n_rows + 3) / 4 : LOSS_GRID)), dim3(256), 0, ctx->stream, j);
    FAE_LAUNCH_CHECK(ctx);
    return FAE_OK;
}

extern "C" int32_t fae_softmax_loss_fwd(fae_ctx *ctx, const fae_softmax_loss *what, const void *x, int64_t x_row_stride, const void *w,
                                        int64_t w_row_stride, float *loss, float *lse, float *mean, void *ws, size_t ws_bytes)
{
    const char *who = "fae_softmax_loss_fwd";
    int32_t rc = loss_check(ctx, who, what, x, x_row_stride, w, w_row_stride);
    if (rc != FAE_OK)
        return rc;
    const int64_t n = what->n_rows, v = what->n_classes, d = what->width;
    const int size = fae_type_size(what->type);
    if (((uintptr_t)loss | (uintptr_t)lse | (uintptr_t)mean) % 4 != 0)
        return fae_fail(ctx, FAE_EINVAL, "%s: outputs are not aligned to their values", who);
    const LossSpan out[] = {loss_span("loss", loss, 1, 1, n, 4), loss_span("lse", lse, 1, 1, n, 4), loss_span("mean", mean, d, d, n, 4),
                            loss_span("workspace", ws, ws_bytes, ws_bytes, 1, 1)};
    const LossSpan in[] = {loss_span("x", x, x_row_stride, d, n, size), loss_span("w", w, w_row_stride, d, v, size), loss_span("bias", what->bias, 1, 1, v, 4),
                           loss_span("targets", what->targets, 1, 1, n, what->target_bits / 8)};
    rc = loss_check_outputs(ctx, who, out, 4, in, 4);
    if (rc == FAE_OK && mean)
        rc = loss_check_held(ctx, who, "n_rows", n, what->width);
    if (rc != FAE_OK || n == 0)
        return rc;
    rc = loss_check_ws(ctx, who, ws, ws_bytes, fae_softmax_loss_fwd_workspace_bytes(what));
    if (rc != FAE_OK)
        return rc;
    FAE_HIP(ctx, hipSetDevice(ctx->device));
    return loss_forward(ctx, what, x, x_row_stride, w, w_row_stride, loss, lse, mean, ws, ws_bytes);
}

static int32_t loss_backward(fae_ctx *ctx, const char *who, const fae_softmax_loss *what, const void *x, int64_t x_row_stride, const void *w,
                             int64_t w_row_stride, const float *lse, const float *loss, const float *mean, const float *gloss, void *gx,
                             int64_t gx_row_stride, void *gw, int64_t gw_row_stride, float *gbias, void *ws, size_t ws_bytes)
{
    int32_t rc = loss_check(ctx, who, what, x, x_row_stride, w, w_row_stride);
    if (rc != FAE_OK)
        return rc;
    const int64_t n = what->n_rows, v = what->n_classes, d = what->width;
    const int size = fae_type_size(what->type);
    if (((uintptr_t)lse | (uintptr_t)loss | (uintptr_t)mean | (uintptr_t)gloss | (uintptr_t)gbias) % 4 != 0)
        return fae_fail(ctx, FAE_EINVAL, "%s: lse, loss, mean, gloss or gbias are not aligned to their values", who);
    if (n > 0 && (!lse || !gloss))
        return fae_fail(ctx, FAE_EINVAL, "%s: null %s", who, lse ? "gloss" : "lse");
    if (gx && n > 0)
        rc = fae_check_rows(ctx, who, "gx", {gx, what->type, gx_row_stride}, n, d);
    if (rc == FAE_OK && gw)
        rc = fae_check_rows(ctx, who, "gw", {gw, what->type, gw_row_stride}, v, d);
    if (rc != FAE_OK)
        return rc;
    const LossSpan out[] = {loss_span("gx", gx, gx_row_stride, d, n, size), loss_span("gw", gw, gw_row_stride, d, v, size), loss_span("gbias", gbias, 1, 1, v, 4),
                            loss_span("workspace", ws, ws_bytes, ws_bytes, 1, 1)};
    const LossSpan in[] = {loss_span("x", x, x_row_stride, d, n, size), loss_span("w", w, w_row_stride, d, v, size), loss_span("bias", what->bias, 1, 1, v, 4),
                           loss_span("targets", what->targets, 1, 1, n, what->target_bits / 8), loss_span("lse", lse, 1, 1, n, 4),
                           loss_span("mean", mean, d, d, n, 4), loss_span("gloss", gloss, 1, 1, n, 4), loss_span("loss", loss, 1, 1, n, 4)};
    rc = loss_check_outputs(ctx, who, out, 4, in, 8);
    if (rc == FAE_OK && (gw || gbias))
        rc = loss_check_held(ctx, who, "n_classes", v, what->width);
    if (rc == FAE_OK && gx && !mean)
        rc = loss_check_held(ctx, who, "n_rows", n, what->width);
    if (rc == FAE_OK)
        rc = loss_check_ws(ctx, who, ws, ws_bytes, fae_softmax_loss_bwd_workspace_bytes(what));
    if (rc != FAE_OK)
        return rc;
    FAE_HIP(ctx, hipSetDevice(ctx->device));
    fae_carver cv(ws, ws_bytes);
    float *g_most = cv.take<float>(LOSS_MOSTS), *x_most = cv.take<float>(LOSS_MOSTS);
    LossRows r;
    memset(&r, 0, sizeof(r));
    float *nlse = cv.take<float>(n), *gt = cv.take<float>(n);
    r.t = cv.take<int32_t>(n);
    float *own_mean = cv.take<float>(n * d);
    if (!cv.ok)
        return fae_fail(ctx, FAE_ENOSPC, "%s: workspace too small", who);
    void *rest = cv.base + cv.used;
    const size_t rest_bytes = cv.cap - cv.used;
    const int64_t row_groups = (n + 3) / 4;
    const int32_t n_most = (int32_t)(row_groups < LOSS_MOSTS ? row_groups : what->type != FAE_BF16 ? LOSS_MOSTS : row_groups < LOSS_GRID ? row_groups : LOSS_GRID);
    if (n > 0) {
        if (gx && !mean) {
            rc = loss_forward(ctx, what, x, x_row_stride, w, w_row_stride, nullptr, nullptr, own_mean, rest, rest_bytes);
            if (rc != FAE_OK)
                return rc;
            mean = own_mean;
        }
        r.x = x;
        r.targets = what->targets;
        r.gx = gx;
        r.x_stride = x_row_stride;
        r.gx_stride = gx_row_stride;
        r.n_rows = n;
        r.lse = lse;
        r.loss = loss;
        r.mean = mean;
        r.gloss = gloss;
        r.bias = what->bias;
        r.w = w;
        r.w_stride = w_row_stride;
        const bool grads = gw || gbias;
        r.nlse = nlse;
        r.gt = grads ? gt : nullptr;
        r.g_most = grads && what->type == FAE_F16 ? g_most : nullptr;
        r.x_most = grads && what->type == FAE_F32 ? x_most : nullptr;
        r.target_bits = what->target_bits;
        r.n_classes = (int32_t)v;
        r.width = (int32_t)d;
        r.scale = what->scale;
        r.status = ctx->d_block;
        fae_ktimer kt(ctx, FAE_K_LOSS_JOIN);
        const dim3 grid(n_most), block(256);
        if (what->type == FAE_F32)
            FAE_LAUNCH(ctx, loss_rows_kernel<float>, grid, block, 0, ctx->stream, r);
        else if (what->type == FAE_BF16)
            FAE_LAUNCH(ctx, loss_rows_kernel<fae_bf16>, grid, block, 0, ctx->stream, r);
        else
            FAE_LAUNCH(ctx, loss_rows_kernel<fae_f16>, grid, block, 0, ctx->stream, r);
        FAE_LAUNCH_CHECK(ctx);
    }
    if (!gw && !gbias)
        return FAE_OK;
    const LossShape s = loss_shape(what, LOSS_GRAD);
    loss_args a;
    loss_common(ctx, what, s, &a);
    a.st = x;
    a.own = w;
    a.st_stride = x_row_stride;
    a.own_stride = w_row_stride;
    a.n_st = (int32_t)n;
    a.n_own = (int32_t)v;
    a.nlse = nlse;
    a.gt = gt;
    a.t = r.t;
    a.g_most = g_most;
    a.st_most = x_most;
    a.n_most = n_most;
    if (s.splits > 1) {
        fae_carver more(rest, rest_bytes);
        a.psum = gbias ? more.take<float>(s.splits * v) : nullptr;
        a.part = gw ? more.take<float>(s.splits * v * s.pitch) : nullptr;
        if (!more.ok)
            return fae_fail(ctx, FAE_ENOSPC, "%s: workspace too small", who);
    } else {
        a.out = gw;
        a.out_stride = gw_row_stride;
        a.out_sum = gbias;
    }
    {
        fae_ktimer kt(ctx, FAE_K_LOSS_BWD);
        loss_run(ctx, s.how, LOSS_GRAD, a);
        FAE_LAUNCH_CHECK(ctx);
    }
    if (s.splits > 1) {
        LossClasses c;
        memset(&c, 0, sizeof(c));
        c.part = a.part;
        c.psum = a.psum;
        c.gw = gw;
        c.gbias = gbias;
        c.gw_stride = gw_row_stride;
        c.n_classes = v;
        c.n_split = a.n_split;
        c.width = (int32_t)d;
        c.pitch = s.pitch;
        c.scale = what->scale;
        fae_ktimer kt(ctx, FAE_K_LOSS_JOIN);
        if (what->type == FAE_F32)
            loss_classes<float>(ctx, c);
        else if (what->type == FAE_BF16)
            loss_classes<fae_bf16>(ctx, c);
        else
            loss_classes<fae_f16>(ctx, c);
        FAE_LAUNCH_CHECK(ctx);
    }
    return FAE_OK;
}

extern "C" int32_t fae_softmax_loss_bwd(fae_ctx *ctx, const fae_softmax_loss *what, const void *x, int64_t x_row_stride, const void *w,
                                        int64_t w_row_stride, const float *lse, const float *mean, const float *gloss, void *gx,
                                        int64_t gx_row_stride, void *gw, int64_t gw_row_stride, float *gbias, void *ws, size_t ws_bytes)
{
    return loss_backward(ctx, "fae_softmax_loss_bwd", what, x, x_row_stride, w, w_row_stride, lse, nullptr, mean, gloss, gx, gx_row_stride, gw, gw_row_stride, gbias,
                         ws, ws_bytes);
}

extern "C" int32_t fae_softmax_loss_bwd_kept(fae_ctx *ctx, const fae_softmax_loss *what, const void *x, int64_t x_row_stride, const void *w,
                                             int64_t w_row_stride, const float *lse, const float *loss, const float *mean, const float *gloss,
                                             void *gx, int64_t gx_row_stride, void *gw, int64_t gw_row_stride, float *gbias, void *ws,
                                             size_t ws_bytes)
{
    return loss_backward(ctx, "fae_softmax_loss_bwd_kept", what, x, x_row_stride, w, w_row_stride, lse, loss, mean, gloss, gx, gx_row_stride, gw, gw_row_stride,
                         gbias, ws, ws_bytes);
}
