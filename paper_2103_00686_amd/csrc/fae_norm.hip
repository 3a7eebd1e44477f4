// Layer norm over rows in parts: how a launch shares out its rows, checks, and the end of the weights' gradients.
#include <math.h>

#include "fae_norm.h"

// dgamma (z = 0) and dbeta (z = 1) of a part from its rows of sums: L lanes of four columns each, THREADS / L rows of sums
// at a time.
struct NormWeightArgs {
    const float *sums[2];
    float *out[2];
    uint32_t n_parts, width, pitch;
    uint32_t n_sums;  // rows of sums of a part
    uint32_t teams;   // of a workgroup if it left a row per part, 0 if it left one per team
};
// From this many columns on, workgroups of 32 columns are enough for the chip and waste less of a line than those of 16 (us of a whole backward
// with 32 | 16 columns: 4096 x 1664 bf16 17.0 | 18.3, 4096 x 4000 26.9 | 29.7; 4000 x 1024 fp32 16.2 | 15.9, 6007 x 4 x 100 12.5 | 12.1).
#define NORM_WIDE_SUMS 1536
template <int L, int THREADS> __global__ __launch_bounds__(THREADS) void norm_weights_kernel(NormWeightArgs a)
{
    constexpr int ROWS = THREADS / L;
    __shared__ float4 part_sum[ROWS][L];
    const float *sums = a.sums[blockIdx.z];
    const uint32_t p = blockIdx.y, l = threadIdx.x % L, g = threadIdx.x / L, c = (blockIdx.x * L + l) * 4;
    if (!a.out[blockIdx.z])
        return;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < a.pitch) {
#pragma unroll 4
        for (uint32_t t = g; t < a.n_sums; t += ROWS) {
            // workgroup t's first team has part t * teams modulo the parts
            const uint32_t k = a.teams ? (p + a.n_parts - t * a.teams % a.n_parts) % a.n_parts : p;
            const float4 v = *(const float4 *)(sums + ((int64_t)t * a.n_parts + k) * a.pitch + c);
            s.x += v.x;
            s.y += v.y;
            s.z += v.z;
            s.w += v.w;
        }
    }
    part_sum[g][l] = s;
    for (int half = ROWS / 2; half > 0; half >>= 1) {
        __syncthreads();
        if ((int)g < half) {
            const float4 v = part_sum[g + half][l];
            s.x += v.x;
            s.y += v.y;
            s.z += v.z;
            s.w += v.w;
            part_sum[g][l] = s;
        }
    }
    if (g == 0) {
        float *out = a.out[blockIdx.z] + (int64_t)p * a.width;
        const float v[4] = {s.x, s.y, s.z, s.w};
        for (int e = 0; e < 4; ++e)
            if (c + e < a.width)
                out[c + e] = v[e];
    }
}

static uint32_t norm_gcd(uint32_t a, uint32_t b) { return b ? norm_gcd(b, a % b) : a; }

// Rows of a team that one launch takes: eight, four where a team is whole waves, six for workgroups of 512 lanes (fp32, us in one launch of
// 512 lanes | in two: 768 x 16 6.0 | 6.4, 192 x 64 5.6 | 6.1, 48 x 256 6.1 | 6.1; 48 x 512 7.4 | 7.1; eight rows: 60 x 256 6.7 | 6.1).
static int norm_few_rows(int lanes, uint32_t threads) { return lanes > 64 ? 4 : threads == 512 ? 6 : 8; }

// Workgroups of 512 lanes or 256 for teams of up to a wave, in the backward.  Where a workgroup adds up its teams' sums in LDS (more teams
// than parts) 512 leave half as many rows of sums, which pays once the launch is as large as it gets (us with 512 | 256: 6007 x 4 x 100 fp32
// 11.1 | 12.3, 2403 x 13 x 64 11.1 | 12.8, 4096 x 256 8.2 | 8.8, 65 536 x 512 76.4 | 78.7; below, 4096 x 64 7.2 | 6.9; and where teams'
// sums go out as they are 1201 x 26 x 64 11.8 | 9.0), or where one launch is then enough (520 x 16 5.4 | 6.4, 717 x 16 6.0 | 6.4,
// 130 x 4 x 16 4.7 | 6.1, 60 x 3 x 64 5.4 | 6.0).
static bool norm_wide_workgroup(int64_t rows, uint32_t parts, int lanes)
{
    const uint32_t teams = 256 / lanes;
    if (teams <= parts)
        return false;
    const int64_t few = teams / parts * parts, few_wide = 2 * teams / parts * parts;
    return rows >= 2LL * 512 * teams || (rows > few * norm_few_rows(lanes, 256) && rows <= few_wide * norm_few_rows(lanes, 512));
}

// Rows of a team at least, backward: fewer where a workgroup adds up its teams' sums before it writes them (2 and 4, us: 717 x 16
// 6.5 and 7.0; 8 instead of 4 where it does not: 4096 x 1664 bf16 27.9 against 22.3, 512 x 8192 bf16 22.0 against 17.2).
static int64_t norm_bwd_rows(uint32_t teams, uint32_t parts) { return teams > parts ? 2 : 4; }

// The backward's workgroups walk on, up to 512 lanes of them to a compute unit (or one workgroup that is larger): with twice as many the rows in flight lie further apart
// and more sums go out (16 384 x 26 x 64 fp32 62 us | 67, 16 384 x 4096 147 | 156), with half as many too little is in flight (91, 154).
// The same number for every compute unit: 341 workgroups of six waves took as long as 512 (16 384 x 6000 bf16 128 us | 180).
static int64_t norm_bwd_most_blocks(uint32_t threads) { return threads > 256 ? 256 : 256 * (512 / threads); }

// workgroups whose teams are a multiple of the parts
static uint32_t norm_whole_blocks(uint32_t teams, uint32_t parts) { return parts / norm_gcd(parts, teams); }

static NormShape norm_shape(const fae_norm *n, bool bwd)
{
    NormShape s;
    memset(&s, 0, sizeof(s));
    s.chunk = fae_type_size(n->x_type) == 2 ? 8 : 4;
    const int chunks = (n->width + s.chunk - 1) / s.chunk, most = norm_chunks(bwd, s.chunk);
    s.nv = 1;
    s.lanes = 2;
    while (s.lanes < 64 && s.lanes < chunks)
        s.lanes *= 2;
    while (s.nv < most && s.nv * 64 < chunks)
        s.nv *= 2;
    if (s.nv * 1024 < chunks) // a workgroup of 1024 holds the row
        s.nv *= 2;
    if (s.nv * 64 < chunks)
        s.lanes = 64 * ((chunks + 64 * s.nv - 1) / (64 * s.nv));
    const int64_t rows = n->n_rows * n->n_parts;
    const uint32_t parts = n->n_parts;
    s.threads = s.lanes > 64 ? s.lanes : bwd && norm_wide_workgroup(rows, parts, s.lanes) ? 512 : 256;
    s.teams = s.threads / s.lanes;
    const uint32_t whole = norm_whole_blocks(s.teams, parts);
    s.pitch = (n->width + 3) / 4 * 4;
    s.part_rows = s.teams > parts ? parts : s.teams;
    const int64_t per_team = bwd ? norm_bwd_rows(s.teams, parts) : norm_fwd_rows(s.nv);
    int64_t blocks = (rows + per_team * s.teams - 1) / (per_team * s.teams);
    const int64_t most_blocks = bwd ? norm_bwd_most_blocks(s.threads) : blocks;
    // Few rows: as many teams as one workgroup holds (or one per part) take them all, and their sums are the gradients, which saves a
    // launch (us with one launch | two: 128 x 64 fp32 5.5 | 6.3, 256 x 64 with 16 rows each 8.2 | 6.4, 16 x 256 4.2 | 6.1,
    // 4 x 26 x 64 3.4 | 6.1, 8 x 8192 bf16 with eight rows each 16.2 | 12.3).
    const uint32_t few = parts * (s.teams > parts ? s.teams / parts : 1);
    if (bwd && rows <= norm_few_rows(s.lanes, s.threads) * (int64_t)few) {
        s.direct = true;
        s.step = few;
        s.blocks = (s.step + s.teams - 1) / s.teams;
        s.n_sums = 1;
        return s;
    }
    if (blocks > most_blocks)
        blocks = most_blocks >= whole ? most_blocks / whole * whole : whole;
    else
        blocks = (blocks + whole - 1) / whole * whole;
    s.blocks = (uint32_t)blocks;
    s.step = s.blocks * s.teams;
    s.n_sums = s.teams > parts ? s.blocks : s.step / parts;
    return s;
}

// Samples of one forward launch: 2^21 workgroups of up to 1024 lanes, as a grid holds fewer than 2^32 threads
static int64_t norm_launch_samples(const fae_norm *n)
{
    fae_norm one = *n;
    one.n_rows = 1;
    const NormShape s = norm_shape(&one, false); // how teams hold a row depends on the row alone
    return ((int64_t)norm_fwd_rows(s.nv) * s.teams << 21) / n->n_parts;
}

static void norm_place_rows(const NormShape &s, NormArgs *a)
{
    const int64_t samples = s.step / a->n_parts;
    a->x_step = samples * a->x_stride;
    a->gy_step = samples * a->gy_stride;
    a->y_step = samples * a->y_stride;
    a->step = s.step;
    a->ends = fae_row_end(a->width, s.chunk, (int64_t)s.lanes * s.nv * s.chunk);
}

// n_rows * n_parts within [0, 2^31), for 1 to FAE_MAX_TABLES parts
static bool norm_rows_fit(const fae_norm *n)
{
    return n->n_rows >= 0 && n->n_rows < 2147483648LL && n->n_rows * n->n_parts < 2147483648LL;
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
    if (!norm_rows_fit(n))
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
    a->n_rows = (uint32_t)(n->n_rows * n->n_parts);
    a->n_parts = n->n_parts;
    a->width = n->width;
    a->eps = n->eps;
    a->inv_width = 1.0f / (float)n->width;
    return fae_check_drop(ctx, who, drop, &a->drop);
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
    rc = fae_check_rows(ctx, who, "x", bx, norm->n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_rows(ctx, who, "y", by, norm->n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_overlap(ctx, who, by, bx, norm->n_rows, row);
    if (rc != FAE_OK)
        return rc;
    a.x_stride = x_row_stride;
    a.y_stride = y_row_stride;
    FAE_HIP(ctx, hipSetDevice(ctx->device));
    fae_ktimer kt(ctx, FAE_K_NORM);
    fae_norm some = *norm; // of as many samples as a launch takes
    const int64_t most = norm_launch_samples(norm);
    for (int64_t first = 0; first < norm->n_rows; first += most) {
        some.n_rows = norm->n_rows - first < most ? norm->n_rows - first : most;
        a.x = (const char *)x + first * x_row_stride * fae_type_size(norm->x_type);
        a.y = (char *)y + first * y_row_stride * fae_type_size(norm->y_type);
        a.row0 = (uint32_t)(first * a.n_parts);
        a.n_rows = (uint32_t)(some.n_rows * a.n_parts);
        const NormShape s = norm_shape(&some, false);
        norm_place_rows(s, &a);
        if (norm->x_type == FAE_F32)
            norm_fwd_by_type(ctx, norm, s, a);
        else
            norm_fwd16_by_type(ctx, norm, s, a);
        FAE_LAUNCH_CHECK(ctx);
    }
    return FAE_OK;
}

// Both sums of every workgroup, a row per team or part; at least 256 bytes.  More rows may take fewer workgroups (a last one's teams rounded
// up to the parts, workgroups of 512 lanes instead of 256): the size is what any number of rows up to these would need, so that it does not fall.
extern "C" size_t fae_layer_norm_bwd_workspace_bytes(const fae_norm *norm)
{
    if (!norm || norm->n_parts < 1 || norm->n_parts > FAE_MAX_TABLES || norm->width < 1 || norm->width > FAE_NORM_MAX_WIDTH ||
        !norm_rows_fit(norm) || norm->x_type < FAE_F32 || norm->x_type > FAE_F16)
        return 0;
    const NormShape s = norm_shape(norm, true);
    if (s.direct)
        return 256;
    const int64_t rows = norm->n_rows * norm->n_parts;
    const uint32_t parts = norm->n_parts;
    int64_t sums = 0; // rows of them, of all parts
    for (uint32_t threads = s.lanes > 64 ? s.threads : 256; threads <= (s.lanes > 64 ? s.threads : 512u); threads += 256) {
        const uint32_t teams = threads / s.lanes, whole = norm_whole_blocks(teams, parts);
        const int64_t per = norm_bwd_rows(teams, parts) * teams, most = norm_bwd_most_blocks(threads);
        int64_t blocks = (rows + per - 1) / per;
        blocks = ((blocks < most ? blocks : most) + whole - 1) / whole * whole;
        const int64_t n = blocks * (teams > parts ? parts : teams);
        sums = n > sums ? n : sums;
    }
    return 2 * fae_align_up((size_t)sums * s.pitch * sizeof(float), 256);
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
    rc = fae_check_rows(ctx, who, "x", bx, norm->n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_rows(ctx, who, "gy", bg, norm->n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_rows(ctx, who, "gx", bo, norm->n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_overlap(ctx, who, bo, bx, norm->n_rows, row);
    if (rc == FAE_OK)
        rc = fae_check_overlap(ctx, who, bo, bg, norm->n_rows, row);
    if (rc != FAE_OK)
        return rc;
    if ((uintptr_t)ws % 16 != 0)
        return fae_fail(ctx, FAE_EINVAL, "%s: the workspace is not on 16 bytes", who);
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
    const NormShape s = norm_shape(norm, true);
    norm_place_rows(s, &a);
    NormWeightArgs w;
    memset(&w, 0, sizeof(w));
    a.part_rows = s.part_rows;
    a.in_regs = s.part_rows == s.teams;
    a.direct = s.direct;
    if (s.direct) {
        a.pgamma = dgamma;
        a.pbeta = dbeta;
        a.pitch = a.width;
    } else if (dgamma || dbeta) {
        fae_carver cv(ws, ws_bytes);
        const size_t n = (size_t)s.n_sums * a.n_parts * s.pitch;
        float *pg = cv.take<float>(n), *pb = cv.take<float>(n);
        a.pgamma = dgamma ? pg : nullptr;
        a.pbeta = dbeta ? pb : nullptr;
        a.pitch = s.pitch;
        w.sums[0] = pg;
        w.sums[1] = pb;
        w.out[0] = dgamma;
        w.out[1] = dbeta;
        w.n_parts = a.n_parts;
        w.width = a.width;
        w.pitch = s.pitch;
        w.n_sums = s.n_sums;
        w.teams = s.teams > a.n_parts ? s.teams : 0;
    }
    {
        fae_ktimer kt(ctx, FAE_K_NORM);
        if (norm->x_type == FAE_F32)
            norm_bwd_by_type(ctx, norm, s, a);
        else
            norm_bwd16_by_type(ctx, norm, s, a);
        FAE_LAUNCH_CHECK(ctx);
    }
    if (!s.direct && (dgamma || dbeta)) {
        fae_ktimer kt(ctx, FAE_K_NORM_WEIGHTS);
        if ((int64_t)a.n_parts * s.pitch >= NORM_WIDE_SUMS)
            FAE_LAUNCH(ctx, (norm_weights_kernel<8, 512>), dim3((s.pitch + 31) / 32, a.n_parts, 2), dim3(512), 0, ctx->stream, w);
        else
            FAE_LAUNCH(ctx, (norm_weights_kernel<4, 256>), dim3((s.pitch + 15) / 16, a.n_parts, 2), dim3(256), 0, ctx->stream, w);
        FAE_LAUNCH_CHECK(ctx);
    }
    return FAE_OK;
}
