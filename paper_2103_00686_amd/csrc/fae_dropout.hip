// Dropout, forward and backward, and the checks that it shares with layer norm.
#include <math.h>

#include "fae_rows.h"

int32_t fae_check_rows(fae_ctx *ctx, const char *who, const char *what, const fae_rows &b, int64_t n_rows, int64_t row)
{
    const int size = fae_type_size(b.type);
    if (!b.p)
        return fae_fail(ctx, FAE_EINVAL, "%s: null %s", who, what);
    if ((uintptr_t)b.p % size != 0)
        return fae_fail(ctx, FAE_EINVAL, "%s: %s is not aligned to its values", who, what);
    int64_t span;
    if (b.stride < row || __builtin_mul_overflow(n_rows - 1, b.stride, &span) || span > (1LL << 56))
        return fae_fail(ctx, FAE_EINVAL, "%s: row stride %lld of %s is below %lld or out of range", who, (long long)b.stride, what,
                        (long long)row);
    return FAE_OK;
}

int32_t fae_check_overlap(fae_ctx *ctx, const char *who, const fae_rows &out, const fae_rows &in, int64_t n_rows, int64_t row)
{
    if (out.p == in.p && out.type == in.type && (out.stride == in.stride || n_rows == 1))
        return FAE_OK; // in place
    const int64_t so = fae_type_size(out.type), si = fae_type_size(in.type);
    const uintptr_t o0 = (uintptr_t)out.p, i0 = (uintptr_t)in.p;
    const uintptr_t o1 = o0 + ((n_rows - 1) * out.stride + row) * so, i1 = i0 + ((n_rows - 1) * in.stride + row) * si;
    if (o1 <= i0 || i1 <= o0)
        return FAE_OK;
    if (n_rows > 1 && out.stride * so == in.stride * si) { // side by side in rows of one buffer
        const int64_t step = out.stride * so;
        const int64_t d = (int64_t)(i0 > o0 ? (i0 - o0) % step : (step - (int64_t)((o0 - i0) % step)) % step); // from a row of out to the next of in
        if (d >= row * so && d + row * si <= step)
            return FAE_OK;
    }
    return fae_fail(ctx, FAE_EINVAL, "%s: input and output overlap", who);
}

int32_t fae_check_drop(fae_ctx *ctx, const char *who, const fae_drop *drop, fae_drop_args *out)
{
    memset(out, 0, sizeof(*out));
    out->scale = 1.0f;
    if (!drop)
        return FAE_OK;
    if (!(drop->p >= 0.0 && drop->p <= 1.0))
        return fae_fail(ctx, FAE_EINVAL, "%s: p=%g outside [0,1]", who, drop->p);
    if ((uintptr_t)drop->d_offset % 8 != 0)
        return fae_fail(ctx, FAE_EINVAL, "%s: d_offset is not aligned to its value", who);
    const double t = nearbyint(drop->p * 65536.0);
    if ((t == 0.0 && drop->p > 0.0) || (t == 65536.0 && drop->p < 1.0))
        return fae_fail(ctx, FAE_EINVAL, "%s: p=%g is kept to 2^-17 and would round to %d", who, drop->p, t == 0.0 ? 0 : 1);
    out->below = (uint32_t)t;
    out->scale = t < 65536.0 ? (float)(65536.0 / (65536.0 - t)) : 0.0f;
    out->key[0] = (uint32_t)drop->seed;
    out->key[1] = (uint32_t)(drop->seed >> 32);
    out->offset = drop->offset;
    out->d_offset = drop->d_offset;
    return FAE_OK;
}

struct DropArgs {
    const void *x;
    void *y;
    int64_t x_stride, y_stride;
    uint32_t row0;        // the launch's first row (of all parts)
    uint32_t n_groups;    // groups of eight values in its rows
    uint32_t per_row;     // of them in a row
    uint32_t per_row_inv; // 2^18 / per_row, rounded up (for rows of fewer than DROP_TILE groups)
    uint32_t n_parts, width;
    int32_t ends; // how the rows end, in chunks of 16 bytes of x
    fae_drop_args drop;
};

#define DROP_TILE 256
#define DROP_LAUNCH (1LL << 31) // groups of one launch at most, a thread each: a grid holds fewer than 2^32 threads

// A thread takes a group of eight values, a workgroup DROP_TILE consecutive groups: one division per workgroup finds its first row,
// and a group's row is a small number of rows on: none or one where rows are as long as the tile, else a product with
// per_row's inverse, exact as q < 2^9 times the inverse's excess, below per_row < 2^8, stays under 2^17.
// What bounds it: memory.  50 001 x 1664 fp32 to bf16 82 us, 6.1 TB/s (a copy of that size reaches 6.0); 65 536 x 1024 fp16 44 us,
// 6.1 TB/s.  Two and four groups per thread took longer (84 and 85 us, 49 and 46), as did non-temporal
// accesses (100 us, the f32 one of 16 384 x 1664 60 against 40): lines of which a store writes half go out twice.
// ENDS: FAE_WHOLE where every row is a multiple of eight values.
template <typename TX, typename TY, int ENDS> __global__ __launch_bounds__(DROP_TILE) void dropout_kernel(DropArgs a)
{
    constexpr int E = sizeof(TX) == 2 ? 8 : 4; // values in 16 bytes
    const uint32_t base = blockIdx.x * DROP_TILE;
    if (base + threadIdx.x >= a.n_groups)
        return;
    const uint32_t row0 = base / a.per_row;
    const uint32_t q = base - row0 * a.per_row + threadIdx.x;
    const uint32_t on = a.per_row >= DROP_TILE ? (q >= a.per_row ? 1 : 0) : (q * a.per_row_inv) >> 18;
    const uint32_t group = q - on * a.per_row, row = row0 + on;
    uint32_t r = row, part = 0;
    if (a.n_parts > 1) {
        r = row / a.n_parts;
        part = row - r * a.n_parts;
    }
    const TX *x = (const TX *)a.x + r * a.x_stride + (int64_t)part * a.width;
    TY *y = (TY *)a.y + r * a.y_stride + (int64_t)part * a.width;
    fae_place<E> at[8 / E];
    typename fae_vec<TX, E>::type v[8 / E];
#pragma unroll
    for (int h = 0; h < 8 / E; ++h) {
        at[h].set(group * 8 + h * E, a.width);
        v[h] = fae_load<TX, E, ENDS>(x, at[h], a.ends);
    }
    const fae_mask8 m = fae_philox(group, a.row0 + row, fae_drop_offset(a.drop), a.drop.key[0], a.drop.key[1]);
#pragma unroll
    for (int h = 0; h < 8 / E; ++h) {
        float o[E];
        fae_settle<TX, E, ENDS>(v[h], at[h], a.ends, o);
#pragma unroll
        for (int e = 0; e < E; ++e)
            o[e] = fae_drop1(o[e], m.number(h * E + e), a.drop.below, a.drop.scale);
        fae_store<TY, E, ENDS>(y, o, at[h]);
    }
}

static int32_t dropout_impl(fae_ctx *ctx, const char *who, const fae_drop *drop, int64_t n_rows, int32_t n_parts, int32_t width,
                            const fae_rows &x, const fae_rows &y)
{
    if (!ctx)
        return FAE_EINVAL;
    if (!drop)
        return fae_fail(ctx, FAE_EINVAL, "%s: null dropout", who);
    DropArgs a;
    memset(&a, 0, sizeof(a));
    int32_t rc = fae_check_drop(ctx, who, drop, &a.drop);
    if (rc != FAE_OK)
        return rc;
    if (n_rows < 0 || n_parts < 1 || width < 1 || (int64_t)n_parts * width >= 2147483648LL || n_rows >= 4294967296LL ||
        n_rows * n_parts >= 4294967296LL)
        return fae_fail(ctx, FAE_EINVAL, "%s: %lld rows of %d parts of %d values are out of range", who, (long long)n_rows, n_parts, width);
    if (x.type < FAE_F32 || x.type > FAE_F16 || y.type < FAE_F32 || y.type > FAE_F16 ||
        (x.type != y.type && x.type != FAE_F32 && y.type != FAE_F32))
        return fae_fail(ctx, FAE_EINVAL, "%s: types %d and %d do not go together", who, x.type, y.type);
    if (n_rows == 0)
        return FAE_OK;
    const int64_t row = (int64_t)n_parts * width;
    rc = fae_check_rows(ctx, who, "input", x, n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_rows(ctx, who, "output", y, n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_overlap(ctx, who, y, x, n_rows, row);
    if (rc != FAE_OK)
        return rc;
    a.x_stride = x.stride;
    a.y_stride = y.stride;
    a.per_row = ((uint32_t)width + 7) / 8;
    a.per_row_inv = ((1u << 18) + a.per_row - 1) / a.per_row;
    a.n_parts = n_parts;
    a.width = width;
    a.ends = fae_row_end(width, 16 / fae_type_size(x.type), a.per_row * 8LL);
    if (n_rows * n_parts * (int64_t)a.per_row > (1LL << 39)) // 8 TiB and more: no such buffers
        return fae_fail(ctx, FAE_EINVAL, "%s: too many values", who);
    int64_t samples = n_rows;
    if (x.stride == row && y.stride == row) { // the parts are rows
        samples *= n_parts;
        a.n_parts = 1;
        a.x_stride = a.y_stride = width;
    }
    FAE_HIP(ctx, hipSetDevice(ctx->device));
    fae_ktimer kt(ctx, FAE_K_DROPOUT);
    const dim3 block(DROP_TILE);
    const int64_t groups = (int64_t)a.n_parts * a.per_row, most = DROP_LAUNCH / groups; // of a sample; samples of a launch
    for (int64_t first = 0; first < samples; first += most) {
        a.x = (const char *)x.p + first * a.x_stride * fae_type_size(x.type);
        a.y = (char *)y.p + first * a.y_stride * fae_type_size(y.type);
        a.row0 = (uint32_t)(first * a.n_parts);
        a.n_groups = (uint32_t)((samples - first < most ? samples - first : most) * groups);
        const dim3 grid((a.n_groups + DROP_TILE - 1) / DROP_TILE);
#define DROP_CASE(TX, TX_, TY, TY_)                                                              \
    if (x.type == TX && y.type == TY) {                                                          \
        if (a.ends == FAE_WHOLE)                                                                 \
            FAE_LAUNCH(ctx, (dropout_kernel<TX_, TY_, FAE_WHOLE>), grid, block, 0, ctx->stream, a);   \
        else                                                                                     \
            FAE_LAUNCH(ctx, (dropout_kernel<TX_, TY_, FAE_ANY>), grid, block, 0, ctx->stream, a);  \
    }
        DROP_CASE(FAE_F32, float, FAE_F32, float)
        DROP_CASE(FAE_F32, float, FAE_BF16, fae_bf16)
        DROP_CASE(FAE_F32, float, FAE_F16, fae_f16)
        DROP_CASE(FAE_BF16, fae_bf16, FAE_F32, float)
        DROP_CASE(FAE_F16, fae_f16, FAE_F32, float)
        DROP_CASE(FAE_BF16, fae_bf16, FAE_BF16, fae_bf16)
        DROP_CASE(FAE_F16, fae_f16, FAE_F16, fae_f16)
#undef DROP_CASE
        FAE_LAUNCH_CHECK(ctx);
    }
    return FAE_OK;
}

extern "C" int32_t fae_dropout_fwd(fae_ctx *ctx, const fae_drop *drop, int64_t n_rows, int32_t n_parts, int32_t width, const void *x,
                                   int32_t x_type, int64_t x_row_stride, void *y, int32_t y_type, int64_t y_row_stride)
{
    return dropout_impl(ctx, "fae_dropout_fwd", drop, n_rows, n_parts, width, {x, x_type, x_row_stride}, {y, y_type, y_row_stride});
}

// the mask is what it was in the forward: the same call on the gradient
extern "C" int32_t fae_dropout_bwd(fae_ctx *ctx, const fae_drop *drop, int64_t n_rows, int32_t n_parts, int32_t width, const void *gy,
                                   int32_t y_type, int64_t gy_row_stride, void *gx, int32_t x_type, int64_t gx_row_stride)
{
    return dropout_impl(ctx, "fae_dropout_bwd", drop, n_rows, n_parts, width, {gy, y_type, gy_row_stride}, {gx, x_type, gx_row_stride});
}
