// Layer norm over rows in parts, forward and backward, with dropout as its epilogue.
#include <math.h>

#include "fae_rows.h"

// A row is held by a team: LANES lanes of a wave (several teams to a wave) or whole waves, each lane with NV chunks of E
// values in registers, so that x (and gy) are read once whatever the statistics need.  Team q of a launch takes the rows
// q, q + step, q + 2 step, ...; step is a multiple of the parts, so a team stays with one part, holds its weights in registers,
// and can add up their gradient over all its rows.
struct NormArgs {
    const void *x, *gy;
    void *y; // forward: y, backward: gx
    int64_t x_stride, gy_stride, y_stride;
    int64_t x_step, gy_step, y_step; // from one of a team's rows to its next
    const float *gamma, *beta;
    float *pgamma, *pbeta; // backward: sums of the launch's workgroups, or the gradients themselves
    int64_t n_rows;        // rows of all parts
    uint32_t step;         // teams that take rows
    uint32_t n_parts, width;
    uint32_t pitch;   // of a row of sums
    uint32_t part_rows; // rows of sums that a workgroup leaves: its teams, or the parts if these are fewer
    int32_t direct;   // the sums are the gradients
    int32_t ragged;   // some lane's chunks are not all whole
    int32_t in_regs;  // a team's sums go out as they are
    float eps, inv_width;
    fae_drop_args drop;
};

// ---------------------------------------------------------------------------------
// sums over a team, the same bits in every lane
// ---------------------------------------------------------------------------------
template <int CTRL> __device__ __forceinline__ float norm_dpp_add(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int LANES> __device__ __forceinline__ float norm_lane_sum(float v)
{
    if constexpr (LANES >= 2)
        v = norm_dpp_add<0xB1>(v); // the neighbour
    if constexpr (LANES >= 4)
        v = norm_dpp_add<0x4E>(v); // the other pair of four lanes
    if constexpr (LANES >= 8)
        v = norm_dpp_add<0x141>(v); // eight lanes mirrored: the other four
    if constexpr (LANES >= 16)
        v = norm_dpp_add<0x140>(v); // sixteen lanes mirrored: the other eight
    if constexpr (LANES >= 32) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false); // rows 0, 0, 2, 2 and 1, 1, 3, 3 of sixteen lanes
        const uint32_t lo = r[0], hi = r[1];
        v = __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
    }
    if constexpr (LANES >= 64) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false); // the lower half twice and the upper half twice
        const uint32_t lo = r[0], hi = r[1];
        v = __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
    }
    return v;
}

// Two sums at once.  Teams of several waves (a workgroup of their own) join them in LDS, in two buffers taken in turn: one barrier per
// call, as whoever writes a buffer again has passed the barrier behind everyone's reads of it.
template <int LANES, bool WAVES> struct norm_team {
    float2 (*red)[16];
    int turn = 0;
    __device__ __forceinline__ void sum2(float &a, float &b)
    {
        a = norm_lane_sum<LANES>(a);
        b = norm_lane_sum<LANES>(b);
        if constexpr (WAVES) {
            const int lane = fae_lane(), w = threadIdx.x / FAE_WAVE, n = blockDim.x / FAE_WAVE;
            if (lane == 0)
                red[turn][w] = make_float2(a, b);
            __syncthreads();
            const float2 t = (lane & 15) < n ? red[turn][lane & 15] : make_float2(0.f, 0.f);
            a = norm_lane_sum<16>(t.x);
            b = norm_lane_sum<16>(t.y);
            turn ^= 1;
        }
    }
};

// dropout of a chunk that starts at column c
template <int E> __device__ __forceinline__ void norm_drop(float (&v)[E], uint32_t c, uint32_t row, uint64_t offset, const fae_drop_args &d)
{
    static_assert(E == 4 || E == 8, "half a group of eight or a whole one");
    const fae_mask8 m = fae_philox(c >> 3, row, offset, d.key[0], d.key[1]);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const uint32_t w = E == 8 ? m.w[e >> 1] : (c & 4 ? m.w[2 + (e >> 1)] : m.w[e >> 1]);
        v[e] = fae_drop1(v[e], e & 1 ? w >> 16 : w & 0xffffu, d.below, d.scale);
    }
}

template <typename TX> constexpr int norm_chunk() { return sizeof(TX) == 2 ? 8 : 4; } // values in 16 bytes of x

// where a thread stands
template <int LANES, bool WAVES, int NV, int E> struct norm_place {
    uint32_t q;      // team of the launch
    int l;           // lane of the team
    int lanes;       // lanes of the team
    uint32_t col[NV];
    int there[NV];   // values of the chunk that exist
    __device__ __forceinline__ norm_place(uint32_t width)
    {
        if constexpr (WAVES) {
            q = blockIdx.x;
            l = threadIdx.x;
            lanes = blockDim.x;
        } else {
            q = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
            l = threadIdx.x % LANES;
            lanes = LANES;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            col[j] = (uint32_t)(j * lanes + l) * E;
            const int left = (int)width - (int)col[j];
            there[j] = left < 0 ? 0 : (left < E ? left : E);
        }
    }
};

// Deviations from the mean in v's place and 1 / sqrt(variance + eps).  They are taken from a first mean, whose own rounding error
// is then their mean and goes off them too: with one number for the mean, a row far from zero beside its spread
// would keep that error.  Columns that do not exist get the mean: nothing in either sum.
template <int LANES, bool WAVES, int NV, int E>
__device__ __forceinline__ float norm_center(float (&v)[NV][E], const int (&there)[NV], const NormArgs &a, norm_team<LANES, WAVES> &team)
{
    float s = 0.f, none = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e)
            s += v[j][e];
    team.sum2(s, none);
    const float m = s * a.inv_width;
    if (a.ragged) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e)
                v[j][e] = e < there[j] ? v[j][e] : m;
    }
    float d1 = 0.f, d2 = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            v[j][e] -= m;
            d1 += v[j][e];
            d2 += v[j][e] * v[j][e];
        }
    team.sum2(d1, d2);
    const float rest = d1 * a.inv_width;
    const float var = d2 * a.inv_width - rest * rest;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e)
            v[j][e] -= rest;
    return 1.0f / sqrtf(fmaxf(var, 0.f) + a.eps);
}

template <typename TX, typename TY, int LANES, bool WAVES, int NV>
__global__ __launch_bounds__(WAVES ? 1024 : 256) void norm_fwd_kernel(NormArgs a)
{
    constexpr int E = norm_chunk<TX>();
    __shared__ float2 red[2][16];
    norm_team<LANES, WAVES> team{red};
    const norm_place<LANES, WAVES, NV, E> at(a.width);
    if (at.q >= a.step)
        return;
    const uint32_t s0 = at.q / a.n_parts, part = at.q - s0 * a.n_parts;
    const uint64_t offset = a.drop.below ? fae_drop_offset(a.drop) : 0;
    const TX *x = (const TX *)a.x + s0 * a.x_stride + part * a.width;
    TY *y = (TY *)a.y + s0 * a.y_stride + part * a.width;
    float gamma[NV][E], beta[NV][E];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const auto g = a.gamma ? fae_load<float, E>(a.gamma + part * a.width + at.col[j], at.there[j]) : typename fae_vec<float, E>::type(1.f);
        const auto b = a.beta ? fae_load<float, E>(a.beta + part * a.width + at.col[j], at.there[j]) : typename fae_vec<float, E>::type(0.f);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            gamma[j][e] = g[e];
            beta[j][e] = b[e];
        }
    }
    for (int64_t row = at.q; row < a.n_rows; row += a.step, x += a.x_step, y += a.y_step) {
        float v[NV][E];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const auto raw = fae_load<TX, E>(x + at.col[j], at.there[j]);
#pragma unroll
            for (int e = 0; e < E; ++e)
                v[j][e] = (float)raw[e];
        }
        const float rstd = norm_center<LANES, WAVES, NV, E>(v, at.there, a, team);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                v[j][e] = v[j][e] * rstd * gamma[j][e] + beta[j][e];
            if (a.drop.below)
                norm_drop<E>(v[j], at.col[j], (uint32_t)row, offset, a.drop);
            fae_store<TY, E>(y + at.col[j], v[j], at.there[j]);
        }
    }
}

// The rows' gradient, and the team's sums of the weights' gradients in registers over all its rows.
template <typename TX, typename TY, int LANES, bool WAVES, int NV>
__global__ __launch_bounds__(WAVES ? 1024 : 256) void norm_bwd_kernel(NormArgs a)
{
    constexpr int E = norm_chunk<TX>();
    __shared__ float2 red[2][16];
    norm_team<LANES, WAVES> team{red};
    const norm_place<LANES, WAVES, NV, E> at(a.width);
    const uint32_t s0 = at.q / a.n_parts, part = at.q - s0 * a.n_parts;
    const uint64_t offset = a.drop.below ? fae_drop_offset(a.drop) : 0;
    const TX *x = (const TX *)a.x + s0 * a.x_stride + part * a.width;
    const TY *gy = (const TY *)a.gy + s0 * a.gy_stride + part * a.width;
    TX *gx = (TX *)a.y + s0 * a.y_stride + part * a.width;
    float gamma[NV][E], dgamma[NV][E], dbeta[NV][E];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const auto g = a.gamma && at.q < a.step ? fae_load<float, E>(a.gamma + part * a.width + at.col[j], at.there[j]) : typename fae_vec<float, E>::type(1.f);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            gamma[j][e] = g[e];
            dgamma[j][e] = dbeta[j][e] = 0.f;
        }
    }
    for (int64_t row = at.q < a.step ? (int64_t)at.q : a.n_rows; row < a.n_rows; row += a.step, x += a.x_step, gy += a.gy_step, gx += a.y_step) {
        float v[NV][E], g[NV][E];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const auto rx = fae_load<TX, E>(x + at.col[j], at.there[j]);
            const auto rg = fae_load<TY, E>(gy + at.col[j], at.there[j]);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                v[j][e] = (float)rx[e];
                g[j][e] = (float)rg[e];
            }
        }
        const float rstd = norm_center<LANES, WAVES, NV, E>(v, at.there, a, team);
        float c1 = 0.f, c2 = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (a.drop.below)
                norm_drop<E>(g[j], at.col[j], (uint32_t)row, offset, a.drop);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                v[j][e] *= rstd; // h
                dbeta[j][e] += g[j][e];
                dgamma[j][e] += g[j][e] * v[j][e];
                g[j][e] *= gamma[j][e]; // a
                c1 += g[j][e];
                c2 += g[j][e] * v[j][e];
            }
        }
        team.sum2(c1, c2);
        c1 *= a.inv_width;
        c2 *= a.inv_width;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                g[j][e] = rstd * (g[j][e] - c1 - v[j][e] * c2);
            fae_store<TX, E>(gx + at.col[j], g[j], at.there[j]);
        }
    }
    if (!a.pgamma && !a.pbeta)
        return;
    // The sums go out a row per team, or where a workgroup has more teams than there are parts a row per part, the teams of a part
    // added up in LDS.
    if (a.in_regs) {
        const uint32_t r = a.direct ? part : at.q;
        if (a.direct && at.q >= a.step)
            return;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (a.pgamma)
                fae_store<float, E>(a.pgamma + (int64_t)r * a.pitch + at.col[j], dgamma[j], at.there[j]);
            if (a.pbeta)
                fae_store<float, E>(a.pbeta + (int64_t)r * a.pitch + at.col[j], dbeta[j], at.there[j]);
        }
        return;
    }
    if constexpr (!WAVES) {
        constexpr int TEAMS = 256 / LANES, ROW = LANES * NV * E;
        __shared__ float sums[TEAMS * ROW];
        for (int which = 0; which < 2; ++which) {
            float *out = which ? a.pbeta : a.pgamma;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    sums[threadIdx.x / LANES * ROW + at.col[j] + e] = which ? dbeta[j][e] : dgamma[j][e];
            __syncthreads();
            if (!out)
                continue;
            const uint32_t n = a.part_rows * a.width;
            for (uint32_t i = threadIdx.x; i < n; i += 256) {
                const uint32_t k = i / a.width, c = i - k * a.width;
                float s = 0.f;
                for (uint32_t t = k; t < TEAMS; t += a.n_parts)
                    s += sums[t * ROW + c];
                out[(int64_t)(blockIdx.x * a.part_rows + k) * a.pitch + c] = s;
            }
        }
    }
}

// dgamma (z = 0) and dbeta (z = 1) of a part from its rows of sums: sixteen lanes of four columns, 64 rows at a time.
struct NormWeightArgs {
    const float *sums[2];
    float *out[2];
    uint32_t n_parts, width, pitch;
    uint32_t n_sums;  // rows of sums of a part
    uint32_t teams;   // of a workgroup if it left a row per part, 0 if it left one per team
};
__global__ __launch_bounds__(1024) void norm_weights_kernel(NormWeightArgs a)
{
    __shared__ float4 part_sum[64][16];
    const float *sums = a.sums[blockIdx.z];
    const uint32_t p = blockIdx.y, l = threadIdx.x % 16, g = threadIdx.x / 16, c = blockIdx.x * 64 + l * 4;
    if (!a.out[blockIdx.z])
        return;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < a.pitch) {
#pragma unroll 4
        for (uint32_t t = g; t < a.n_sums; t += 64) {
            // workgroup t's first team has part t * teams modulo the parts
            const uint32_t k = a.teams ? (p + a.n_parts - (uint32_t)((uint64_t)t * a.teams % a.n_parts)) % a.n_parts : p;
            const float4 v = *(const float4 *)(sums + ((int64_t)t * a.n_parts + k) * a.pitch + c);
            s.x += v.x;
            s.y += v.y;
            s.z += v.z;
            s.w += v.w;
        }
    }
    part_sum[g][l] = s;
    for (int half = 32; half > 0; half >>= 1) {
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

// ---------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------
// how a launch shares out the rows
struct NormShape {
    int chunk;      // values per chunk
    int lanes;      // per team: 1 .. 64, or 64 times the waves
    int nv;         // chunks per lane
    uint32_t teams; // per workgroup
    uint32_t threads;
    uint32_t blocks, step;
    bool direct;        // backward: the only rows of sums are the gradients
    uint32_t part_rows; // backward: rows of sums per workgroup
    uint32_t n_sums;    // backward: rows of sums per part
    uint32_t pitch;
};

static uint32_t norm_gcd(uint32_t a, uint32_t b) { return b ? norm_gcd(b, a % b) : a; }

static NormShape norm_shape(const fae_norm *n, bool bwd)
{
    NormShape s;
    memset(&s, 0, sizeof(s));
    s.chunk = fae_type_size(n->x_type) == 2 ? 8 : 4;
    const int chunks = (n->width + s.chunk - 1) / s.chunk, most = 16 / s.chunk; // 16 values per lane at most
    s.nv = 1;
    s.lanes = 1;
    while (s.lanes < 64 && s.lanes < chunks)
        s.lanes *= 2;
    while (s.nv < most && s.nv * 64 < chunks)
        ++s.nv;
    if (s.nv * 64 < chunks)
        s.lanes = 64 * ((chunks + 64 * s.nv - 1) / (64 * s.nv));
    s.threads = s.lanes > 64 ? s.lanes : 256;
    s.teams = s.threads / s.lanes;
    const int64_t rows = n->n_rows * n->n_parts;
    const uint32_t parts = n->n_parts, whole = parts / norm_gcd(parts, s.teams); // workgroups whose teams are a multiple of the parts
    s.pitch = (n->width + 3) / 4 * 4;
    const int64_t per_team = bwd ? 8 : 2;
    int64_t blocks = (rows + per_team * s.teams - 1) / (per_team * s.teams);
    if (bwd) {
        const int64_t most_blocks = 256 * 1024 / s.threads;
        if (blocks > most_blocks)
            blocks = most_blocks;
        s.direct = blocks * s.teams <= parts || blocks == 1;
    }
    if (s.direct) {
        s.step = parts * (s.teams > parts ? s.teams / parts : 1);
        s.blocks = (s.step + s.teams - 1) / s.teams;
        s.part_rows = s.teams > parts ? parts : s.teams;
        s.n_sums = 1;
        return s;
    }
    if (bwd) {
        s.blocks = (uint32_t)((blocks + whole - 1) / whole * whole);
        s.step = s.blocks * s.teams;
        s.part_rows = s.teams > parts ? parts : s.teams;
        s.n_sums = s.teams > parts ? s.blocks : s.step / parts;
        return s;
    }
    const int64_t step = (blocks * s.teams + parts - 1) / parts * parts;
    s.step = (uint32_t)step;
    s.blocks = (uint32_t)((step + s.teams - 1) / s.teams);
    return s;
}

static void norm_place_rows(const NormShape &s, NormArgs *a)
{
    const int64_t samples = s.step / a->n_parts;
    a->x_step = samples * a->x_stride;
    a->gy_step = samples * a->gy_stride;
    a->y_step = samples * a->y_stride;
    a->step = s.step;
    a->ragged = a->width != (uint32_t)(s.lanes * s.nv * s.chunk);
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
    a->n_rows = n->n_rows * n->n_parts;
    a->n_parts = n->n_parts;
    a->width = n->width;
    a->eps = n->eps;
    a->inv_width = 1.0f / (float)n->width;
    return fae_check_drop(ctx, who, drop, &a->drop);
}

template <bool BWD, typename TX, typename TY, int LANES, bool WAVES, int NV> static void norm_run(fae_ctx *ctx, const NormShape &s, const NormArgs &a)
{
    if constexpr (BWD)
        FAE_LAUNCH(ctx, (norm_bwd_kernel<TX, TY, LANES, WAVES, NV>), dim3(s.blocks), dim3(s.threads), 0, ctx->stream, a);
    else
        FAE_LAUNCH(ctx, (norm_fwd_kernel<TX, TY, LANES, WAVES, NV>), dim3(s.blocks), dim3(s.threads), 0, ctx->stream, a);
}

template <bool BWD, typename TX, typename TY> static void norm_by_width(fae_ctx *ctx, const NormShape &s, const NormArgs &a)
{
    constexpr int MOST = 16 / norm_chunk<TX>();
    switch (s.lanes) {
    case 1: norm_run<BWD, TX, TY, 1, false, 1>(ctx, s, a); return;
    case 2: norm_run<BWD, TX, TY, 2, false, 1>(ctx, s, a); return;
    case 4: norm_run<BWD, TX, TY, 4, false, 1>(ctx, s, a); return;
    case 8: norm_run<BWD, TX, TY, 8, false, 1>(ctx, s, a); return;
    case 16: norm_run<BWD, TX, TY, 16, false, 1>(ctx, s, a); return;
    case 32: norm_run<BWD, TX, TY, 32, false, 1>(ctx, s, a); return;
    case 64: break;
    default: norm_run<BWD, TX, TY, 64, true, MOST>(ctx, s, a); return;
    }
    if (s.nv == 1)
        norm_run<BWD, TX, TY, 64, false, 1>(ctx, s, a);
    else if (s.nv == 2)
        norm_run<BWD, TX, TY, 64, false, 2>(ctx, s, a);
    if constexpr (MOST == 4) {
        if (s.nv == 3)
            norm_run<BWD, TX, TY, 64, false, 3>(ctx, s, a);
        else if (s.nv == 4)
            norm_run<BWD, TX, TY, 64, false, 4>(ctx, s, a);
    }
}

template <bool BWD> static void norm_by_type(fae_ctx *ctx, const fae_norm *n, const NormShape &s, const NormArgs &a)
{
    if (n->y_type == FAE_F32)
        norm_by_width<BWD, float, float>(ctx, s, a);
    else if (n->y_type == FAE_BF16 && n->x_type == FAE_F32)
        norm_by_width<BWD, float, fae_bf16>(ctx, s, a);
    else if (n->x_type == FAE_F32)
        norm_by_width<BWD, float, fae_f16>(ctx, s, a);
    else if (n->x_type == FAE_BF16)
        norm_by_width<BWD, fae_bf16, fae_bf16>(ctx, s, a);
    else
        norm_by_width<BWD, fae_f16, fae_f16>(ctx, s, a);
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
    a.x = x;
    a.y = y;
    a.x_stride = x_row_stride;
    a.y_stride = y_row_stride;
    FAE_HIP(ctx, hipSetDevice(ctx->device));
    fae_ktimer kt(ctx, FAE_K_NORM);
    const NormShape s = norm_shape(norm, false);
    norm_place_rows(s, &a);
    norm_by_type<false>(ctx, norm, s, a);
    FAE_LAUNCH_CHECK(ctx);
    return FAE_OK;
}

// Both sums of every workgroup, a row per team or part; at least 256 bytes
extern "C" size_t fae_layer_norm_bwd_workspace_bytes(const fae_norm *norm)
{
    if (!norm || norm->n_rows < 0 || norm->n_parts < 1 || norm->n_parts > FAE_MAX_TABLES || norm->width < 1 ||
        norm->width > FAE_NORM_MAX_WIDTH || norm->n_rows >= 2147483648LL / norm->n_parts || norm->x_type < FAE_F32 || norm->x_type > FAE_F16)
        return 0;
    const NormShape s = norm_shape(norm, true);
    return s.direct ? 256 : 2 * fae_align_up((size_t)s.n_sums * norm->n_parts * s.pitch * sizeof(float), 256);
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
        norm_by_type<true>(ctx, norm, s, a);
        FAE_LAUNCH_CHECK(ctx);
    }
    if (!s.direct && (dgamma || dbeta)) {
        fae_ktimer kt(ctx, FAE_K_NORM_WEIGHTS);
        FAE_LAUNCH(ctx, norm_weights_kernel, dim3((s.pitch + 63) / 64, a.n_parts, 2), dim3(1024), 0, ctx->stream, w);
        FAE_LAUNCH_CHECK(ctx);
    }
    return FAE_OK;
}
