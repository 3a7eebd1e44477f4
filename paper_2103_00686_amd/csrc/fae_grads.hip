// The norm of all gradients together, and clipping by it.
#include <math.h>
#include <stdlib.h>

#include "fae_rows.h"

// What bounds both kernels: memory.  188 M bf16 values: squares 67 us (5.6 TB/s), clipping 137 us (5.5 TB/s); the list is read twice, as a
// factor is known only after the last square.  Spans of 8 KiB with the next one in flight; 16 KiB 70 and 151 us, 4 KiB 76 and 141.
// Reading goes in stretches, without the caches' help (with it 97 us: the lines that it leaves there serve clipping a little, 127 instead
// of 137, and cost more); stores go a grid's width apart (in stretches 152 us).
#define GRADS_BYTES 8192      // of a tensor that a workgroup takes at a time: a span
#define GRADS_GROUPS 2048     // workgroups of a launch at most, and partial sums
#define GRADS_CHAINS 4
#define GRADS_LIST 128        // tensors of a launch: their addresses are kernel arguments, of which there are 4 KiB
#define GRADS_MOST (1LL << 36) // values of a tensor: more than the card holds

__host__ __device__ static inline int grads_span(int type) { return type == FAE_F32 ? GRADS_BYTES / 4 : GRADS_BYTES / 2; }

struct GradsArgs {
    const void *g[GRADS_LIST];
    void *out[GRADS_LIST];
    int64_t n[GRADS_LIST];
    int32_t start[GRADS_LIST + 1]; // spans of the tensors before
    uint8_t type[GRADS_LIST];
    int32_t spans, n_before; // n_before: partial sums of the launches before this one
    double *sums;
    double scale, max_norm;
    float *norm;
    int32_t n_sums;
};

static_assert(sizeof(GradsArgs) <= 4096, "kernel arguments");

// the tensor of a span: how many start at or before it, less one; counted in two rounds of independent loads
__device__ __forceinline__ int grads_find(const GradsArgs &a, int span)
{
    int v[15], base = 0, more = 0;
#pragma unroll
    for (int i = 1; i < GRADS_LIST / 16; ++i)
        v[i] = a.start[i * 16];
#pragma unroll
    for (int i = 1; i < GRADS_LIST / 16; ++i)
        base += v[i] <= span ? 16 : 0;
#pragma unroll
    for (int i = 1; i < 16; ++i)
        v[i - 1] = a.start[base + i];
#pragma unroll
    for (int i = 1; i < 16; ++i)
        more += v[i - 1] <= span ? 1 : 0;
    return base + more;
}

// A workgroup's spans: where it is, and the 16-byte pieces of a whole span in flight.
struct GradsWalk {
    int b, end, step, z, type, next_start;
    const char *g;
    int64_t left; // bytes from the span's start to the tensor's end
    __device__ __forceinline__ void tensor(const GradsArgs &a)
    {
        type = a.type[z];
        next_start = a.start[z + 1];
        const int64_t from = (int64_t)(b - a.start[z]) * GRADS_BYTES;
        g = (const char *)a.g[z] + from;
        left = a.n[z] * (type == FAE_F32 ? 4 : 2) - from;
    }
    // spans one after the other (for reading alone), or a grid's width apart (where there are stores)
    __device__ __forceinline__ void begin(const GradsArgs &a, bool apart)
    {
        step = apart ? gridDim.x : 1;
        b = apart ? blockIdx.x : (int)((int64_t)a.spans * blockIdx.x / gridDim.x);
        end = apart ? a.spans : (int)((int64_t)a.spans * (blockIdx.x + 1) / gridDim.x);
        if (b < end) {
            z = grads_find(a, b);
            tensor(a);
        }
    }
    __device__ __forceinline__ void next(const GradsArgs &a)
    {
        b += step;
        g += (int64_t)step * GRADS_BYTES;
        left -= (int64_t)step * GRADS_BYTES;
        if (b < end && b >= next_start) {
            z = grads_find(a, b);
            tensor(a);
        }
    }
    __device__ __forceinline__ bool whole() const { return b < end && left >= GRADS_BYTES; }
};
typedef uint32_t grads_raw __attribute__((ext_vector_type(4)));
typedef grads_raw grads_loose __attribute__((aligned(2)));
#define GRADS_UN (GRADS_BYTES / 4096)
__device__ __forceinline__ void grads_load(const GradsWalk &w, grads_raw (&v)[GRADS_UN])
{
    if (w.whole()) {
#pragma unroll
        for (int u = 0; u < GRADS_UN; ++u)
            v[u] = __builtin_nontemporal_load((const grads_loose *)(w.g + (u * 256 + threadIdx.x) * 16));
    }
}

template <typename T> __device__ __forceinline__ void grads_squares(const GradsWalk &w, const grads_raw (&v)[GRADS_UN], double (&s)[GRADS_CHAINS])
{
    constexpr int E = 16 / sizeof(T);
    if (w.whole()) {
#pragma unroll
        for (int u = 0; u < GRADS_UN; ++u) {
            const auto t = __builtin_bit_cast(typename fae_vec<T, E>::type, v[u]);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const double d = (double)(float)t[e];
                s[e % GRADS_CHAINS] = fma(d, d, s[e % GRADS_CHAINS]);
            }
        }
    } else {
        for (int i = threadIdx.x; i < w.left / (int)sizeof(T); i += 256) {
            const double d = (double)(float)((const T *)w.g)[i];
            s[0] = fma(d, d, s[0]);
        }
    }
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

// A workgroup walks over its stretch of the launch's spans, the next one on its way while one is squared, and adds what it finds to its own
// partial sum.
__global__ __launch_bounds__(256) void grads_squares_kernel(GradsArgs a)
{
    double some[GRADS_CHAINS] = {0.0, 0.0, 0.0, 0.0};
    GradsWalk w, n;
    grads_raw v[GRADS_UN], nv[GRADS_UN];
    w.begin(a, false);
    grads_load(w, v);
    while (w.b < w.end) {
        n = w;
        n.next(a);
        grads_load(n, nv);
        if (w.type == FAE_F32)
            grads_squares<float>(w, v, some);
        else if (w.type == FAE_BF16)
            grads_squares<fae_bf16>(w, v, some);
        else
            grads_squares<fae_f16>(w, v, some);
        w = n;
#pragma unroll
        for (int u = 0; u < GRADS_UN; ++u)
            v[u] = nv[u];
    }
    const double s = grads_block_sum((some[0] + some[1]) + (some[2] + some[3]));
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

template <typename T> __device__ __forceinline__ void grads_scale(const GradsWalk &w, const grads_raw (&v)[GRADS_UN], char *out, float f0, float f1)
{
    constexpr int E = 16 / sizeof(T);
    if (w.whole()) {
#pragma unroll
        for (int u = 0; u < GRADS_UN; ++u) {
            auto t = __builtin_bit_cast(typename fae_vec<T, E>::type, v[u]);
#pragma unroll
            for (int e = 0; e < E; ++e)
                t[e] = (T)((float)t[e] * f0 * f1);
            __builtin_nontemporal_store(__builtin_bit_cast(grads_raw, t), (grads_loose *)(out + (u * 256 + threadIdx.x) * 16));
        }
    } else {
        for (int i = threadIdx.x; i < w.left / (int)sizeof(T); i += 256)
            ((T *)out)[i] = (T)((float)((const T *)w.g)[i] * f0 * f1);
    }
}

// Every workgroup adds up the partial sums by itself, in the same order.
__global__ __launch_bounds__(256) void grads_clip_kernel(GradsArgs a)
{
    const double norm = grads_norm(a.sums, a.n_sums, a.scale);
    if (a.norm && blockIdx.x == 0 && threadIdx.x == 0)
        *a.norm = (float)norm;
    // a factor below fp32's normal range (gradients of 1e38) would lose its digits: it is taken as two then
    // (an infinite norm is not below an infinite limit: 0, as under any other)
    const double f = norm < INFINITY && norm <= a.max_norm ? a.scale : (norm == INFINITY ? 0.0 : a.max_norm / norm) * a.scale;
    const bool tiny = fabs(f) < 0x1p-100;
    const float f0 = tiny ? 0x1p-64f : 1.f, f1 = (float)(tiny ? f * 0x1p64 : f);
    GradsWalk w, n;
    grads_raw v[GRADS_UN], nv[GRADS_UN];
    w.begin(a, true);
    grads_load(w, v);
    while (w.b < w.end) {
        n = w;
        n.next(a);
        grads_load(n, nv);
        char *out = (char *)a.out[w.z] + (w.g - (const char *)a.g[w.z]);
        if (f != 1.0 || out != w.g) {
            if (w.type == FAE_F32)
                grads_scale<float>(w, v, out, f0, f1);
            else if (w.type == FAE_BF16)
                grads_scale<fae_bf16>(w, v, out, f0, f1);
            else
                grads_scale<fae_f16>(w, v, out, f0, f1);
        }
        w = n;
#pragma unroll
        for (int u = 0; u < GRADS_UN; ++u)
            v[u] = nv[u];
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
static int32_t grads_check_overlap(fae_ctx *ctx, const char *who, int32_t n, const fae_grad *h, bool clip, const float *norm, const void *ws, size_t ws_bytes)
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
        if (clip)
            s[k++] = {(uintptr_t)h[z].out, (uintptr_t)h[z].out + bytes, z, true};
        if (!clip || h[z].g != h[z].out)
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
        const int64_t spans = (h[z].n + grads_span(h[z].type) - 1) / grads_span(h[z].type);
        if (a->start[k] + spans >= 1LL << 30)
            break;
        a->g[k] = h[z].g;
        a->out[k] = h[z].out;
        a->n[k] = h[z].n;
        a->type[k] = (uint8_t)h[z].type;
        a->start[k + 1] = a->start[k] + (int32_t)spans;
        ++k;
    }
    a->spans = a->start[k];
    for (int i = k + 1; i <= GRADS_LIST; ++i)
        a->start[i] = INT32_MAX;
    return z;
}

extern "C" size_t fae_grad_workspace_bytes(int32_t n_grads, const fae_grad *h_grads)
{
    (void)h_grads;
    return n_grads < 0 || n_grads > FAE_MAX_GRADS ? 0 : GRADS_GROUPS * sizeof(double);
}

static uint32_t grads_groups(const GradsArgs &a)
{
    const int32_t spans = a.spans;
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
    const char *who = "fae_grad_norm";
    int32_t rc = grads_check(ctx, who, n_grads, h_grads, scale, norm, ws, ws_bytes, false);
    if (rc == FAE_OK)
        rc = grads_check_overlap(ctx, who, n_grads, h_grads, false, norm, ws, fae_grad_workspace_bytes(n_grads, h_grads));
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
    rc = grads_check_overlap(ctx, who, n_grads, h_grads, true, norm, ws, fae_grad_workspace_bytes(n_grads, h_grads));
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
