// The norm of all gradients together, and clipping by it.
#include <math.h>
#include <stdlib.h>

#include "fae_rows.h"

#define GRADS_LIST FAE_MAX_TABLES // tensors of a launch: their addresses are kernel arguments
#define GRADS_SPAN 8192           // values of a tensor that a workgroup takes at a time
#define GRADS_GROUPS 1024         // workgroups of a launch at most, and partial sums
#define GRADS_MOST (1LL << 37)    // values of a tensor: more than the card holds

struct GradsArgs {
    const void *g[GRADS_LIST];
    void *out[GRADS_LIST];
    int64_t n[GRADS_LIST];
    int32_t start[FAE_MAX_TABLES + 1]; // spans of the tensors before
    uint8_t type[GRADS_LIST];
    int32_t n_list, n_before; // n_before: partial sums of the launches before this one
    double *sums;
    double scale, max_norm;
    float *norm;
    int32_t n_sums;
};

template <typename T> __device__ __forceinline__ double grads_squares(const T *g, int64_t n)
{
    constexpr int E = 16 / sizeof(T), UN = GRADS_SPAN / (256 * E);
    typedef typename fae_vec<T, E>::loose loose;
    double s = 0.0;
    if (n >= GRADS_SPAN) {
        typename fae_vec<T, E>::type v[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u)
            v[u] = *(const loose *)(g + (u * 256 + threadIdx.x) * E);
#pragma unroll
        for (int u = 0; u < UN; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const double d = (double)(float)v[u][e];
                s = fma(d, d, s);
            }
    } else {
        for (int i = threadIdx.x * E; i < n; i += 256 * E)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (i + e < n) {
                    const double d = (double)(float)g[i + e];
                    s = fma(d, d, s);
                }
    }
    return s;
}

__device__ __forceinline__ double grads_block_sum(double s)
{
    __shared__ double part[4];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1)
        s += __shfl_xor(s, d, 64);
    if (fae_lane() == 0)
        part[threadIdx.x / 64] = s;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// A workgroup walks over spans of all tensors of its launch and adds what it finds to its own partial sum.
__global__ __launch_bounds__(256) void grads_squares_kernel(GradsArgs a)
{
    double s = 0.0;
    for (int b = blockIdx.x; b < a.start[a.n_list]; b += gridDim.x) {
        const int z = fae_find_table(a.start, a.n_list, b);
        const int64_t from = (int64_t)(b - a.start[z]) * GRADS_SPAN, n = a.n[z] - from;
        if (a.type[z] == FAE_F32)
            s += grads_squares((const float *)a.g[z] + from, n);
        else if (a.type[z] == FAE_BF16)
            s += grads_squares((const fae_bf16 *)a.g[z] + from, n);
        else
            s += grads_squares((const fae_f16 *)a.g[z] + from, n);
    }
    s = grads_block_sum(s);
    if (threadIdx.x == 0)
        a.sums[blockIdx.x] = ((int)blockIdx.x < a.n_before ? a.sums[blockIdx.x] : 0.0) + s;
}

__device__ __forceinline__ double grads_norm(const double *sums, int n, double scale)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += 256)
        s += sums[i];
    return sqrt(grads_block_sum(s)) * fabs(scale);
}

__global__ __launch_bounds__(256) void grads_norm_kernel(GradsArgs a)
{
    const double norm = grads_norm(a.sums, a.n_sums, a.scale);
    if (threadIdx.x == 0)
        *a.norm = (float)norm;
}

template <typename T> __device__ __forceinline__ void grads_scale(const T *g, T *out, int64_t n, float f0, float f1)
{
    constexpr int E = 16 / sizeof(T), UN = GRADS_SPAN / (256 * E);
    typedef typename fae_vec<T, E>::loose loose;
    if (n >= GRADS_SPAN) {
        typename fae_vec<T, E>::type v[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u)
            v[u] = *(const loose *)(g + (u * 256 + threadIdx.x) * E);
#pragma unroll
        for (int u = 0; u < UN; ++u) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                v[u][e] = (T)((float)v[u][e] * f0 * f1);
            *(loose *)(out + (u * 256 + threadIdx.x) * E) = v[u];
        }
    } else {
        for (int i = threadIdx.x * E; i < n; i += 256 * E)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (i + e < n)
                    out[i + e] = (T)((float)g[i + e] * f0 * f1);
    }
}

// Every workgroup adds up the partial sums by itself, in the same order.
__global__ __launch_bounds__(256) void grads_clip_kernel(GradsArgs a)
{
    const double norm = grads_norm(a.sums, a.n_sums, a.scale);
    if (a.norm && blockIdx.x == 0 && threadIdx.x == 0)
        *a.norm = (float)norm;
    // a factor below fp32's normal range (gradients of 1e38) would lose its digits: it is taken as two then
    const double f = norm <= a.max_norm ? a.scale : a.max_norm / norm * a.scale;
    const bool tiny = fabs(f) < 0x1p-100;
    const float f0 = tiny ? 0x1p-64f : 1.f, f1 = (float)(tiny ? f * 0x1p64 : f);
    for (int b = blockIdx.x; b < a.start[a.n_list]; b += gridDim.x) {
        const int z = fae_find_table(a.start, a.n_list, b);
        const int64_t from = (int64_t)(b - a.start[z]) * GRADS_SPAN, n = a.n[z] - from;
        if (f == 1.0 && a.g[z] == a.out[z])
            continue;
        if (a.type[z] == FAE_F32)
            grads_scale((const float *)a.g[z] + from, (float *)a.out[z] + from, n, f0, f1);
        else if (a.type[z] == FAE_BF16)
            grads_scale((const fae_bf16 *)a.g[z] + from, (fae_bf16 *)a.out[z] + from, n, f0, f1);
        else
            grads_scale((const fae_f16 *)a.g[z] + from, (fae_f16 *)a.out[z] + from, n, f0, f1);
    }
}

// ---------------------------------------------------------------------------------
struct GradsSpan {
    uintptr_t p0, p1;
    int32_t z;
    bool out;
};
static int grads_by_start(const void *a, const void *b)
{
    const GradsSpan *x = (const GradsSpan *)a, *y = (const GradsSpan *)b;
    return x->p0 != y->p0 ? (x->p0 < y->p0 ? -1 : 1) : (x->p1 != y->p1 ? (x->p1 < y->p1 ? -1 : 1) : 0);
}

// no output on another tensor's memory (its own gradient's, whole, is allowed), on the norm or the workspace
static int32_t grads_check_overlap(fae_ctx *ctx, const char *who, int32_t n, const fae_grad *h, const float *norm, const void *ws, size_t ws_bytes)
{
    GradsSpan *s = (GradsSpan *)malloc(sizeof(GradsSpan) * (2 * (size_t)n + 2));
    if (!s)
        return fae_fail(ctx, FAE_ENOSPC, "%s: out of host memory", who);
    int32_t k = 0, rc = FAE_OK;
    if (norm)
        s[k++] = {(uintptr_t)norm, (uintptr_t)norm + 4, -1, true};
    s[k++] = {(uintptr_t)ws, (uintptr_t)ws + ws_bytes, -1, true};
    for (int32_t z = 0; z < n; ++z) {
        const int64_t bytes = h[z].n * fae_type_size(h[z].type);
        if (bytes == 0)
            continue;
        s[k++] = {(uintptr_t)h[z].out, (uintptr_t)h[z].out + bytes, z, true};
        if (h[z].g != h[z].out)
            s[k++] = {(uintptr_t)h[z].g, (uintptr_t)h[z].g + bytes, z, false};
    }
    qsort(s, k, sizeof(*s), grads_by_start);
    int32_t any = -1, out = -1; // of the spans so far, the one that ends last, and the same of outputs
    for (int32_t i = 0; i < k && rc == FAE_OK; ++i) {
        if ((out >= 0 && s[i].p0 < s[out].p1) || (any >= 0 && s[i].out && s[i].p0 < s[any].p1))
            rc = fae_fail(ctx, FAE_EINVAL, "%s: an output overlaps another buffer (tensor %d)", who, s[i].z);
        if (any < 0 || s[i].p1 > s[any].p1)
            any = i;
        if (s[i].out && (out < 0 || s[i].p1 > s[out].p1))
            out = i;
    }
    free(s);
    return rc;
}

static int32_t grads_check(fae_ctx *ctx, const char *who, int32_t n_grads, const fae_grad *h, float scale, const float *norm, const void *ws, size_t ws_bytes, bool clip)
{
    if (!ctx)
        return FAE_EINVAL;
    if (n_grads < 0 || n_grads > FAE_MAX_GRADS || (n_grads > 0 && !h))
        return fae_fail(ctx, FAE_EINVAL, "%s: %d tensors", who, n_grads);
    if (!isfinite(scale))
        return fae_fail(ctx, FAE_EINVAL, "%s: scale=%g is not finite", who, scale);
    if ((!norm && !clip) || (uintptr_t)norm % 4 != 0)
        return fae_fail(ctx, FAE_EINVAL, "%s: norm is null or not aligned to its value", who);
    for (int32_t z = 0; z < n_grads; ++z) {
        if (h[z].type < FAE_F32 || h[z].type > FAE_F16 || h[z].n < 0 || h[z].n >= GRADS_MOST)
            return fae_fail(ctx, FAE_EINVAL, "%s: tensor %d: type %d, %lld values", who, z, h[z].type, (long long)h[z].n);
        if (h[z].n > 0 && (!h[z].g || (uintptr_t)h[z].g % fae_type_size(h[z].type) != 0 || (clip && (!h[z].out || (uintptr_t)h[z].out % fae_type_size(h[z].type) != 0))))
            return fae_fail(ctx, FAE_EINVAL, "%s: tensor %d is null or not aligned to its values", who, z);
    }
    if ((uintptr_t)ws % 16 != 0)
        return fae_fail(ctx, FAE_EINVAL, "%s: the workspace is not on 16 bytes", who);
    const size_t need = fae_grad_workspace_bytes(n_grads, h);
    if (!ws || ws_bytes < need)
        return fae_fail(ctx, FAE_ENOSPC, "%s: workspace of %zu bytes, %zu needed", who, ws ? ws_bytes : 0, need);
    return FAE_OK;
}

// the next launch's tensors from number z on; returns the number behind them
static int32_t grads_list(int32_t n_grads, const fae_grad *h, int32_t z, GradsArgs *a)
{
    int k = 0;
    a->start[0] = 0;
    for (; z < n_grads && k < GRADS_LIST; ++z) {
        if (h[z].n == 0)
            continue;
        a->g[k] = h[z].g;
        a->out[k] = h[z].out;
        a->n[k] = h[z].n;
        a->type[k] = (uint8_t)h[z].type;
        a->start[k + 1] = a->start[k] + (int32_t)((h[z].n + GRADS_SPAN - 1) / GRADS_SPAN);
        ++k;
    }
    a->n_list = k;
    for (int i = k + 1; i <= FAE_MAX_TABLES; ++i)
        a->start[i] = a->start[k];
    return z;
}

extern "C" size_t fae_grad_workspace_bytes(int32_t n_grads, const fae_grad *h_grads)
{
    (void)h_grads;
    return n_grads < 0 || n_grads > FAE_MAX_GRADS ? 0 : GRADS_GROUPS * sizeof(double);
}

static uint32_t grads_groups(const GradsArgs &a)
{
    const int32_t spans = a.start[a.n_list];
    return spans < GRADS_GROUPS ? (spans > 0 ? spans : 1) : GRADS_GROUPS;
}

static int32_t grads_sums(fae_ctx *ctx, int32_t n_grads, const fae_grad *h, GradsArgs *a)
{
    a->n_before = 0;
    int32_t z = 0;
    do {
        z = grads_list(n_grads, h, z, a);
        const uint32_t groups = grads_groups(*a);
        FAE_LAUNCH(ctx, grads_squares_kernel, dim3(groups), dim3(256), 0, ctx->stream, *a);
        FAE_LAUNCH_CHECK(ctx);
        a->n_before = (int32_t)groups > a->n_before ? (int32_t)groups : a->n_before;
    } while (z < n_grads);
    a->n_sums = a->n_before;
    return FAE_OK;
}

extern "C" int32_t fae_grad_norm(fae_ctx *ctx, int32_t n_grads, const fae_grad *h_grads, float scale, float *norm, void *ws, size_t ws_bytes)
{
    int32_t rc = grads_check(ctx, "fae_grad_norm", n_grads, h_grads, scale, norm, ws, ws_bytes, false);
    if (rc != FAE_OK)
        return rc;
    FAE_HIP(ctx, hipSetDevice(ctx->device));
    fae_ktimer kt(ctx, FAE_K_GRADS);
    GradsArgs a;
    memset(&a, 0, sizeof(a));
    a.sums = (double *)ws;
    a.scale = scale;
    a.norm = norm;
    rc = grads_sums(ctx, n_grads, h_grads, &a);
    if (rc != FAE_OK)
        return rc;
    FAE_LAUNCH(ctx, grads_norm_kernel, dim3(1), dim3(256), 0, ctx->stream, a);
    FAE_LAUNCH_CHECK(ctx);
    return FAE_OK;
}

extern "C" int32_t fae_grad_clip(fae_ctx *ctx, int32_t n_grads, const fae_grad *h_grads, float scale, float max_norm, float *norm, void *ws,
                                 size_t ws_bytes)
{
    const char *who = "fae_grad_clip";
    int32_t rc = grads_check(ctx, who, n_grads, h_grads, scale, norm, ws, ws_bytes, true);
    if (rc != FAE_OK)
        return rc;
    if (!(max_norm >= 0.f))
        return fae_fail(ctx, FAE_EINVAL, "%s: max_norm=%g", who, max_norm);
    rc = grads_check_overlap(ctx, who, n_grads, h_grads, norm, ws, fae_grad_workspace_bytes(n_grads, h_grads));
    if (rc != FAE_OK)
        return rc;
    FAE_HIP(ctx, hipSetDevice(ctx->device));
    fae_ktimer kt(ctx, FAE_K_GRADS);
    GradsArgs a;
    memset(&a, 0, sizeof(a));
    a.sums = (double *)ws;
    a.scale = scale;
    a.max_norm = max_norm;
    a.norm = norm;
    rc = grads_sums(ctx, n_grads, h_grads, &a);
    if (rc != FAE_OK)
        return rc;
    int32_t z = 0;
    do {
        z = grads_list(n_grads, h_grads, z, &a);
        FAE_LAUNCH(ctx, grads_clip_kernel, dim3(grads_groups(a)), dim3(256), 0, ctx->stream, a);
        FAE_LAUNCH_CHECK(ctx);
        a.norm = nullptr;
    } while (z < n_grads);
    return FAE_OK;
}
