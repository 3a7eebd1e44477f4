// Layer norm over rows in parts, forward and backward, with dropout as its epilogue.
#include <math.h>

#include "fae_rows.h"

struct NormArgs {
    const void *x, *gy;
    void *y; // forward: y, backward: gx
    int64_t x_stride, gy_stride, y_stride;
    const float *gamma, *beta;
    float *dgamma, *dbeta;
    float *mean, *rest, *rstd; // of every row, from the first kernel of the backward to the second
    int64_t n_rows;
    uint32_t n_parts, width;
    float eps, inv_width;
    fae_drop_args drop;
};

__device__ __forceinline__ float norm_wave_sum(float v)
{
#pragma unroll
    for (int m = 1; m < FAE_WAVE; m <<= 1)
        v += __shfl_xor(v, m, FAE_WAVE);
    return v;
}

// A row's mean and 1 / sqrt(variance + eps), by a wave.  Deviations are taken from a first mean, whose own rounding error is
// then their mean, and stays apart (mean + rest): in one number a row far from zero beside its spread would keep that error.
template <typename T> __device__ __forceinline__ void norm_stats(const T *x, uint32_t width, float inv_width, float eps, float *mean, float *rest, float *rstd)
{
    float s = 0.f;
    for (uint32_t c = fae_lane(); c < width; c += FAE_WAVE)
        s += (float)x[c];
    const float m = norm_wave_sum(s) * inv_width;
    float d1 = 0.f, d2 = 0.f;
    for (uint32_t c = fae_lane(); c < width; c += FAE_WAVE) {
        const float d = (float)x[c] - m;
        d1 += d;
        d2 += d * d;
    }
    const float e = norm_wave_sum(d1) * inv_width;
    const float var = norm_wave_sum(d2) * inv_width - e * e;
    *mean = m;
    *rest = e;
    *rstd = 1.0f / sqrtf(fmaxf(var, 0.f) + eps);
}

__device__ __forceinline__ float norm_drop(float v, uint32_t c, uint32_t row, uint64_t offset, const fae_drop_args &d)
{
    return d.below == 0 ? v : fae_drop1(v, fae_philox(c >> 3, row, offset, d.key[0], d.key[1]).number(c & 7), d.below, d.scale);
}

enum { NORM_FWD, NORM_STATS, NORM_BWD };

template <typename TX, typename TY, int MODE> __global__ __launch_bounds__(256) void norm_rows_kernel(NormArgs a)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / FAE_WAVE;
    if (row >= a.n_rows * a.n_parts)
        return;
    const int64_t r = row / a.n_parts;
    const uint32_t at = (uint32_t)(row - r * a.n_parts) * a.width;
    const TX *x = (const TX *)a.x + r * a.x_stride + at;
    const uint64_t offset = a.drop.below ? fae_drop_offset(a.drop) : 0;
    float mean, rest, rstd;
    norm_stats(x, a.width, a.inv_width, a.eps, &mean, &rest, &rstd);
    if constexpr (MODE == NORM_STATS) {
        if (fae_lane() == 0) {
            a.mean[row] = mean;
            a.rest[row] = rest;
            a.rstd[row] = rstd;
        }
    } else if constexpr (MODE == NORM_FWD) {
        TY *y = (TY *)a.y + r * a.y_stride + at;
        for (uint32_t c = fae_lane(); c < a.width; c += FAE_WAVE) {
            const float h = ((float)x[c] - mean - rest) * rstd;
            const float v = h * (a.gamma ? a.gamma[at + c] : 1.f) + (a.beta ? a.beta[at + c] : 0.f);
            y[c] = (TY)norm_drop(v, c, (uint32_t)row, offset, a.drop);
        }
    } else {
        const TY *gy = (const TY *)a.gy + r * a.gy_stride + at;
        TX *gx = (TX *)a.y + r * a.y_stride + at;
        float s1 = 0.f, s2 = 0.f;
        for (uint32_t c = fae_lane(); c < a.width; c += FAE_WAVE) {
            const float g = norm_drop((float)gy[c], c, (uint32_t)row, offset, a.drop) * (a.gamma ? a.gamma[at + c] : 1.f);
            s1 += g;
            s2 += g * (((float)x[c] - mean - rest) * rstd);
        }
        s1 = norm_wave_sum(s1) * a.inv_width;
        s2 = norm_wave_sum(s2) * a.inv_width;
        for (uint32_t c = fae_lane(); c < a.width; c += FAE_WAVE) {
            const float g = norm_drop((float)gy[c], c, (uint32_t)row, offset, a.drop) * (a.gamma ? a.gamma[at + c] : 1.f);
            gx[c] = (TX)(rstd * (g - s1 - ((float)x[c] - mean - rest) * rstd * s2));
        }
    }
}

// dgamma and dbeta: a thread per column, down all rows
template <typename TX, typename TY> __global__ __launch_bounds__(64) void norm_columns_kernel(NormArgs a)
{
    const uint32_t at = blockIdx.x * 64 + threadIdx.x;
    if (at >= a.n_parts * a.width)
        return;
    const uint32_t p = at / a.width, c = at - p * a.width;
    const uint64_t offset = a.drop.below ? fae_drop_offset(a.drop) : 0;
    float s1 = 0.f, c1 = 0.f, s2 = 0.f, c2 = 0.f;
    for (int64_t r = 0; r < a.n_rows; ++r) {
        const int64_t row = r * a.n_parts + p;
        const float h = ((float)((const TX *)a.x + r * a.x_stride)[at] - a.mean[row] - a.rest[row]) * a.rstd[row];
        const float g = norm_drop((float)((const TY *)a.gy + r * a.gy_stride)[at], c, (uint32_t)row, offset, a.drop);
        const float v1 = g * h - c1, t1 = s1 + v1, v2 = g - c2, t2 = s2 + v2; // the rounding error of each sum is carried along
        c1 = (t1 - s1) - v1;
        s1 = t1;
        c2 = (t2 - s2) - v2;
        s2 = t2;
    }
    if (a.dgamma)
        a.dgamma[at] = s1;
    if (a.dbeta)
        a.dbeta[at] = s2;
}

static int32_t norm_check(fae_ctx *ctx, const char *who, const fae_norm *n, const fae_drop *drop, NormArgs *a)
{
    if (!ctx)
        return FAE_EINVAL;
    if (!n)
        return fae_fail(ctx, FAE_EINVAL, "%s: null norm", who);
    if (n->n_parts < 1 || n->n_parts > FAE_MAX_TABLES || n->width < 1 || n->width > FAE_NORM_MAX_WIDTH)
        return fae_fail(ctx, FAE_EINVAL, "%s: n_parts=%d outside [1,%d] or width=%d outside [1,%d]", who, n->n_parts, FAE_MAX_TABLES,
                        n->width, FAE_NORM_MAX_WIDTH);
    if (n->n_rows < 0 || n->n_rows >= 2147483648LL / n->n_parts)
        return fae_fail(ctx, FAE_EINVAL, "%s: n_rows=%lld of %d parts outside [0,2^31)", who, (long long)n->n_rows, n->n_parts);
    if (n->x_type < FAE_F32 || n->x_type > FAE_F16 || n->y_type < FAE_F32 || n->y_type > FAE_F16 ||
        (n->x_type != n->y_type && n->x_type != FAE_F32))
        return fae_fail(ctx, FAE_EINVAL, "%s: types %d and %d do not go together", who, n->x_type, n->y_type);
    if (!(n->eps > 0.f) || !isfinite(n->eps))
        return fae_fail(ctx, FAE_EINVAL, "%s: eps=%g is not above 0", who, (double)n->eps);
    if (((uintptr_t)n->gamma | (uintptr_t)n->beta) % 4 != 0)
        return fae_fail(ctx, FAE_EINVAL, "%s: weights are not aligned to their values", who);
    memset(a, 0, sizeof(*a));
    a->gamma = n->gamma;
    a->beta = n->beta;
    a->n_rows = n->n_rows;
    a->n_parts = n->n_parts;
    a->width = n->width;
    a->eps = n->eps;
    a->inv_width = 1.0f / (float)n->width;
    return fae_check_drop(ctx, who, drop, &a->drop);
}

template <int MODE> static void norm_rows(fae_ctx *ctx, const fae_norm *n, const NormArgs &a)
{
    const dim3 grid((unsigned)((a.n_rows * a.n_parts + 3) / 4)), block(256);
    if (n->y_type == FAE_F32)
        FAE_LAUNCH(ctx, (norm_rows_kernel<float, float, MODE>), grid, block, 0, ctx->stream, a);
    else if (n->y_type == FAE_BF16 && n->x_type == FAE_F32)
        FAE_LAUNCH(ctx, (norm_rows_kernel<float, fae_bf16, MODE>), grid, block, 0, ctx->stream, a);
    else if (n->x_type == FAE_F32)
        FAE_LAUNCH(ctx, (norm_rows_kernel<float, fae_f16, MODE>), grid, block, 0, ctx->stream, a);
    else if (n->x_type == FAE_BF16)
        FAE_LAUNCH(ctx, (norm_rows_kernel<fae_bf16, fae_bf16, MODE>), grid, block, 0, ctx->stream, a);
    else
        FAE_LAUNCH(ctx, (norm_rows_kernel<fae_f16, fae_f16, MODE>), grid, block, 0, ctx->stream, a);
}

static void norm_columns(fae_ctx *ctx, const fae_norm *n, const NormArgs &a)
{
    const dim3 grid((a.n_parts * a.width + 63) / 64), block(64);
    if (n->y_type == FAE_F32)
        FAE_LAUNCH(ctx, (norm_columns_kernel<float, float>), grid, block, 0, ctx->stream, a);
    else if (n->y_type == FAE_BF16 && n->x_type == FAE_F32)
        FAE_LAUNCH(ctx, (norm_columns_kernel<float, fae_bf16>), grid, block, 0, ctx->stream, a);
    else if (n->x_type == FAE_F32)
        FAE_LAUNCH(ctx, (norm_columns_kernel<float, fae_f16>), grid, block, 0, ctx->stream, a);
    else if (n->x_type == FAE_BF16)
        FAE_LAUNCH(ctx, (norm_columns_kernel<fae_bf16, fae_bf16>), grid, block, 0, ctx->stream, a);
    else
        FAE_LAUNCH(ctx, (norm_columns_kernel<fae_f16, fae_f16>), grid, block, 0, ctx->stream, a);
}

extern "C" int32_t fae_layer_norm_fwd(fae_ctx *ctx, const fae_norm *norm, const void *x, int64_t x_row_stride, void *y,
                                      int64_t y_row_stride, const fae_drop *drop)
{
    const char *who = "fae_layer_norm_fwd";
    NormArgs a;
    int32_t rc = norm_check(ctx, who, norm, drop, &a);
    if (rc != FAE_OK || a.n_rows == 0)
        return rc;
    const int64_t row = (int64_t)a.n_parts * a.width;
    const fae_rows bx{x, norm->x_type, x_row_stride}, by{y, norm->y_type, y_row_stride};
    rc = fae_check_rows(ctx, who, "x", bx, a.n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_rows(ctx, who, "y", by, a.n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_overlap(ctx, who, by, bx, a.n_rows, row);
    if (rc != FAE_OK)
        return rc;
    a.x = x;
    a.y = y;
    a.x_stride = x_row_stride;
    a.y_stride = y_row_stride;
    FAE_HIP(ctx, hipSetDevice(ctx->device));
    fae_ktimer kt(ctx, FAE_K_NORM);
    norm_rows<NORM_FWD>(ctx, norm, a);
    FAE_LAUNCH_CHECK(ctx);
    return FAE_OK;
}

extern "C" size_t fae_layer_norm_bwd_workspace_bytes(const fae_norm *norm)
{
    if (!norm || norm->n_rows < 0 || norm->n_parts < 1)
        return 0;
    return 3 * fae_align_up((size_t)norm->n_rows * norm->n_parts * sizeof(float), 256) + 768;
}

extern "C" int32_t fae_layer_norm_bwd(fae_ctx *ctx, const fae_norm *norm, const void *x, int64_t x_row_stride, const void *gy,
                                      int64_t gy_row_stride, void *gx, int64_t gx_row_stride, float *dgamma, float *dbeta,
                                      const fae_drop *drop, void *ws, size_t ws_bytes)
{
    const char *who = "fae_layer_norm_bwd";
    NormArgs a;
    int32_t rc = norm_check(ctx, who, norm, drop, &a);
    if (rc != FAE_OK)
        return rc;
    if (((uintptr_t)dgamma | (uintptr_t)dbeta) % 4 != 0)
        return fae_fail(ctx, FAE_EINVAL, "%s: weights' gradients are not aligned to their values", who);
    const int64_t row = (int64_t)a.n_parts * a.width;
    if (a.n_rows == 0) {
        FAE_HIP(ctx, hipSetDevice(ctx->device));
        rc = dgamma ? fae_fill_u32(ctx, dgamma, row, 0) : FAE_OK;
        return rc == FAE_OK && dbeta ? fae_fill_u32(ctx, dbeta, row, 0) : rc;
    }
    const fae_rows bx{x, norm->x_type, x_row_stride}, bg{gy, norm->y_type, gy_row_stride}, bo{gx, norm->x_type, gx_row_stride};
    rc = fae_check_rows(ctx, who, "x", bx, a.n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_rows(ctx, who, "gy", bg, a.n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_rows(ctx, who, "gx", bo, a.n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_overlap(ctx, who, bo, bx, a.n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_overlap(ctx, who, bo, bg, a.n_rows, row);
    if (rc != FAE_OK)
        return rc;
    if (!ws || ws_bytes < fae_layer_norm_bwd_workspace_bytes(norm))
        return fae_fail(ctx, FAE_ENOSPC, "%s: workspace of %zu bytes, %zu needed", who, ws ? ws_bytes : 0,
                        fae_layer_norm_bwd_workspace_bytes(norm));
    FAE_HIP(ctx, hipSetDevice(ctx->device));
    a.x = x;
    a.gy = gy;
    a.y = gx;
    a.x_stride = x_row_stride;
    a.gy_stride = gy_row_stride;
    a.y_stride = gx_row_stride;
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    fae_carver cv(ws, ws_bytes);
    a.mean = cv.take<float>((size_t)a.n_rows * a.n_parts);
    a.rest = cv.take<float>((size_t)a.n_rows * a.n_parts);
    a.rstd = cv.take<float>((size_t)a.n_rows * a.n_parts);
    if (dgamma || dbeta) { // before gx, which may lie where gy or x is
        {
            fae_ktimer kt(ctx, FAE_K_NORM);
            norm_rows<NORM_STATS>(ctx, norm, a);
        }
        fae_ktimer kt(ctx, FAE_K_NORM_WEIGHTS);
        norm_columns(ctx, norm, a);
    }
    fae_ktimer kt(ctx, FAE_K_NORM);
    norm_rows<NORM_BWD>(ctx, norm, a);
    FAE_LAUNCH_CHECK(ctx);
    return FAE_OK;
}
