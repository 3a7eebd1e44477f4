// Layer norm over rows in parts, forward and backward, with dropout as its epilogue: kernels (gfx950).
#pragma once

#include "fae_rows.h"

// A row is held by a team: LANES lanes of a wave (several teams to a wave) or whole waves, each lane with NV chunks of E
// values in registers, so that x (and gy) are read once whatever the statistics need.  Team q of a launch takes the rows q, q + step,
// q + 2 step, ... (the forward one batch of them); step, the number of teams, is a multiple of the parts, so a team stays with one part, holds its weights in
// registers, and can add up their gradient over all its rows.
//
// What bounds it: memory where there are many rows of whole chunks (the forward of 16 384 x 26 x 64 fp32 takes 40 us, 5.4 TB/s, where
// copying such a buffer takes 39; the backward 61 us, 5.4 TB/s, where adding two of them up into a third takes 56), the chain of a row's three
// reductions where there are few (about half a microsecond a row, one where a team is several waves).  Rows that end inside a chunk, above
// all of two-byte values, are bound by the vector units' work on that chunk (bf16 rows of 100 values 3.6 TB/s forward, 3.8 backward; fp32
// 5.2 and 5.0), rows just above what a wave holds by their empty lanes (1030 values: fp32 4.1 and 4.0, bf16 3.1 and 2.9).
struct NormArgs {
    const void *x, *gy;
    void *y; // forward: y, backward: gx
    int64_t x_stride, gy_stride, y_stride;
    int64_t x_step, gy_step, y_step; // from one of a team's rows to its next
    const float *gamma, *beta;
    float *pgamma, *pbeta; // backward: sums of the launch's workgroups, or the gradients themselves
    uint32_t row0;    // forward: the launch's first row
    uint32_t n_rows;  // rows of all parts, below 2^31 (forward: the launch's)
    uint32_t step;    // teams
    uint32_t n_parts, width;
    uint32_t pitch;   // of a row of sums
    uint32_t part_rows; // rows of sums that a workgroup leaves: its teams, or the parts if these are fewer
    int32_t direct;   // the sums are the gradients
    int32_t in_regs;  // a team's sums go out as they are
    int32_t ends;     // how the rows end: FAE_WHOLE ..
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

// Teams of several waves (a workgroup of their own) join their sums in LDS, in two buffers taken in turn: one barrier per
// call, as whoever writes a buffer again has passed the barrier behind everyone's reads of it.
template <int LANES, bool WAVES> struct norm_team {
    float2 (*red)[16];
    int turn = 0;
    __device__ __forceinline__ float sum(float a)
    {
        a = norm_lane_sum<LANES>(a);
        if constexpr (WAVES) {
            const int lane = fae_lane(), w = threadIdx.x / FAE_WAVE, n = blockDim.x / FAE_WAVE;
            if (lane == 0)
                red[turn][w].x = a;
            __syncthreads();
            a = norm_lane_sum<16>((lane & 15) < n ? red[turn][lane & 15].x : 0.f);
            turn ^= 1;
        }
        return a;
    }
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

// The numbers of a chunk's E values, two to a word
template <int E> struct norm_mask {
    uint32_t w[E / 2];
    // dropped values to zero, whatever they were; what the others are multiplied by is in the weights
    __device__ __forceinline__ void drop(float (&v)[E], const fae_drop_args &d) const
    {
#pragma unroll
        for (int e = 0; e < E; ++e)
            v[e] = (e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu) < d.below ? 0.f : v[e];
    }
};
// Two chunks' numbers (chunks of four or eight that start at columns ca and cb).  A chunk of four is half a group of eight, whose
// other half a neighbouring lane has: each of the two makes one of the two groups whole and hands over what it does
// not need itself (50 001 x 26 x 64 with dropout, forward 105 -> 98 us, backward 181 -> 173).
template <int E>
__device__ __forceinline__ void norm_masks(norm_mask<E> &a, norm_mask<E> &b, uint32_t ca, uint32_t ra, uint32_t cb, uint32_t rb, uint64_t offset,
                                           const fae_drop_args &d)
{
    if constexpr (E == 8) {
        const fae_mask8 ma = fae_philox(ca >> 3, ra, offset, d.key[0], d.key[1]), mb = fae_philox(cb >> 3, rb, offset, d.key[0], d.key[1]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a.w[i] = ma.w[i];
            b.w[i] = mb.w[i];
        }
    } else {
        static_assert(E == 4, "half a group of eight or a whole one");
        const bool odd = threadIdx.x & 1; // a team's lanes are even in number: the neighbour is of the same team
        const fae_mask8 m = fae_philox((odd ? cb : ca) >> 3, odd ? rb : ra, offset, d.key[0], d.key[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t give = odd ? m.w[i] : m.w[2 + i];
            const uint32_t got = __builtin_amdgcn_update_dpp(0, give, 0xB1, 0xf, 0xf, true);
            a.w[i] = odd ? got : m.w[i];
            b.w[i] = odd ? m.w[2 + i] : got;
        }
    }
}
// all chunks of a row where a lane has two and more
template <int E, int NV>
__device__ __forceinline__ void norm_row_masks(norm_mask<E> (&m)[NV], const fae_place<E> (&at)[NV], uint32_t row, uint64_t offset, const fae_drop_args &d)
{
#pragma unroll
    for (int j = 0; j + 1 < NV; j += 2)
        norm_masks<E>(m[j], m[j + 1], at[j].col, row, at[j + 1].col, row, offset, d);
}

// The first half of a lane's chunks exist and are whole, as a lane is only given two and more where its team has more than half of them.
// (Teams of 64 lanes with NV chunks hold more than NV / 2 x 64; teams of w waves, w > 1, more than NV x 64 (w - 1).)
template <int NV> constexpr bool norm_sure(int j) { return j < NV / 2; }

template <typename TX> constexpr int norm_chunk() { return sizeof(TX) == 2 ? 8 : 4; } // values in 16 bytes of x

// where a thread stands
template <int LANES, int THREADS, bool WAVES, int NV, int E> struct norm_place {
    uint32_t q;      // team of the launch
    int l;           // lane of the team
    int lanes;       // lanes of the team
    fae_place<E> at[NV];
    __device__ __forceinline__ norm_place(uint32_t width)
    {
        if constexpr (WAVES) {
            q = blockIdx.x;
            l = threadIdx.x;
            lanes = blockDim.x;
        } else {
            q = blockIdx.x * (THREADS / LANES) + threadIdx.x / LANES;
            l = threadIdx.x % LANES;
            lanes = LANES;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
            at[j].set((uint32_t)(j * lanes + l) * E, width);
    }
};

// Deviations from the mean in v's place and 1 / sqrt(variance + eps).  They are taken from a first mean, whose own rounding error
// is then their mean and goes off them too: with one number for the mean, a row far from zero beside its spread
// would keep that error.  Columns that do not exist add nothing to either sum.
template <int ENDS, int LANES, bool WAVES, int NV, int E>
__device__ __forceinline__ float norm_center(float (&v)[NV][E], const fae_place<E> (&at)[NV], const NormArgs &a, norm_team<LANES, WAVES> &team)
{
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e)
            s += v[j][e];
    float m = team.sum(s) * a.inv_width;
    asm("" : "+v"(m)); // one value: not a product that is rounded for some chunks and fused into the difference for others
    float d1 = 0.f, d2 = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (ENDS == FAE_ANY && !norm_sure<NV>(j))
                v[j][e] = e < at[j].there ? v[j][e] - m : 0.f;
            else
                v[j][e] -= ENDS == FAE_WHOLE || norm_sure<NV>(j) || at[j].there > 0 ? m : 0.f; // an absent chunk's values are zeros
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
    return rsqrtf(fmaxf(var, 0.f) + a.eps); // to a unit of the last place; a root and a quotient would be a third of a short row's work
}

// a part's gamma or beta (ones or zeros if there are none) times dropout's factor
template <int ENDS, bool DROP, int E, int NV>
__device__ __forceinline__ void norm_weights(const float *w, float none, const NormArgs &a, uint32_t part, const fae_place<E> (&at)[NV],
                                             float (&out)[NV][E])
{
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (!w) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                out[j][e] = none;
        } else if constexpr (ENDS != FAE_ANY) {
            const auto v = fae_load<float, E, ENDS>(w + part * a.width, at[j], a.ends);
#pragma unroll
            for (int e = 0; e < E; ++e)
                out[j][e] = v[e];
        } else { // four at a time, as rows that end anywhere
            const int ends = a.width < 4 ? FAE_SHORT : FAE_CROOKED;
#pragma unroll
            for (int h = 0; h < E; h += 4) {
                fae_place<4> p;
                p.set(at[j].col + h, a.width);
                float v[4];
                fae_settle<float, 4, FAE_ANY>(fae_load<float, 4, FAE_ANY>(w + part * a.width, p, ends), p, ends, v);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    out[j][h + e] = v[e];
            }
        }
        if constexpr (DROP) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                out[j][e] *= a.drop.scale;
        }
    }
}

// A batch of U rows of a team, asked for together; rows past the end are the first one again, so that no load is behind a branch
// (behind one that some lanes do not take, every load waited for the one before: 6007 x 4 x 100 backward 28 -> 16 us)
template <typename T, int E, int NV, int U, int ENDS, bool MAY_SHORT> struct norm_batch {
    typename fae_vec<T, E>::type raw[U][NV];
    __device__ __forceinline__ void load(const T *p, int64_t step, uint32_t row, uint32_t end, const NormArgs &a, const fae_place<E> (&at)[NV])
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const T *r = U == 1 || row + u * a.step < end ? p + u * step : p;
#pragma unroll
            for (int j = 0; j < NV; ++j)
                raw[u][j] = fae_load<T, E, ENDS, MAY_SHORT>(r, at[j], a.ends);
        }
    }
    __device__ __forceinline__ void get(int u, const NormArgs &a, const fae_place<E> (&at)[NV], float (&v)[NV][E]) const
    {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            fae_settle<T, E, ENDS>(raw[u][j], at[j], a.ends, v[j], norm_sure<NV>(j));
    }
};

// A team takes one batch of U rows and the next workgroup the next ones: teams that walked on would hold addresses and steps in registers
// that wide rows need (4000 x 9001 fp32 68 us | 86, bf16 8000 x 9001 95 | 117, 30 000 x 1030 fp32 55 | 64; most others alike).
template <typename TX, typename TY, int LANES, int THREADS, bool WAVES, int NV, int U, int ENDS, bool DROP>
__global__ __launch_bounds__(THREADS) void norm_fwd_kernel(NormArgs a)
{
    constexpr int E = norm_chunk<TX>();
    __shared__ float2 red[2][16];
    norm_team<LANES, WAVES> team{red};
    const norm_place<LANES, THREADS, WAVES, NV, E> at(a.width);
    if (at.q >= a.step || at.q >= a.n_rows)
        return;
    const uint32_t s0 = at.q / a.n_parts, part = at.q - s0 * a.n_parts;
    const uint32_t end = a.n_rows, row = at.q;
    const TX *x = (const TX *)a.x + s0 * a.x_stride + part * a.width;
    TY *y = (TY *)a.y + s0 * a.y_stride + part * a.width;
    norm_batch<TX, E, NV, U, ENDS, LANES == 2> in;
    in.load(x, a.x_step, row, end, a, at.at);
    const uint64_t offset = DROP ? fae_drop_offset(a.drop) : 0;
    float gamma[NV][E], beta[NV][E];
    norm_weights<ENDS, DROP, E, NV>(a.gamma, 1.f, a, part, at.at, gamma);
    norm_weights<ENDS, DROP, E, NV>(a.beta, 0.f, a, part, at.at, beta);
    norm_mask<E> mask[2][NV]; // of two rows where a lane has one chunk
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (U > 1 && row + u * a.step >= end)
            break;
        if constexpr (DROP) {
            const uint32_t r = a.row0 + row + u * a.step;
            if constexpr (NV > 1)
                norm_row_masks<E, NV>(mask[u & 1], at.at, r, offset, a.drop);
            else if (u % 2 == 0)
                norm_masks<E>(mask[0][0], mask[1][0], at.at[0].col, r, at.at[0].col, r + a.step, offset, a.drop);
        }
        float v[NV][E];
        in.get(u, a, at.at, v);
        const float rstd = norm_center<ENDS, LANES, WAVES, NV, E>(v, at.at, a, team);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                v[j][e] = v[j][e] * rstd * gamma[j][e] + beta[j][e];
            if constexpr (DROP)
                mask[u & 1][j].drop(v[j], a.drop);
            fae_store<TY, E, ENDS>(y + u * a.y_step, v[j], at.at[j], norm_sure<NV>(j));
        }
    }
}

// The rows' gradient, and the team's sums of the weights' gradients in registers over all its rows.  DEPTH rows of a team are held: the
// loads of the next DEPTH - 1 go out before the present one's sums are taken (into registers of their own, with no copies between them,
// which would wait for the loads).  EARLY: a row's own registers are loaded again as soon as its values are taken.  All teams walk with
// one stride: rows in flight then lie side by side (16 384 x 26 x 64 73 -> 67 us against a stretch of rows for every few workgroups).
template <typename TX, typename TY, int LANES, int THREADS, bool WAVES, int NV, int DEPTH, bool EARLY, int ENDS, bool DROP>
__global__ __launch_bounds__(THREADS) void norm_bwd_kernel(NormArgs a)
{
    constexpr int E = norm_chunk<TX>();
    __shared__ float2 red[2][16];
    norm_team<LANES, WAVES> team{red};
    const norm_place<LANES, THREADS, WAVES, NV, E> at(a.width);
    const uint32_t s0 = at.q / a.n_parts, part = at.q - s0 * a.n_parts;
    const uint32_t end = a.n_rows;
    uint32_t row = at.q < a.step ? at.q : end;
    const TX *x = (const TX *)a.x + s0 * a.x_stride + part * a.width;
    const TY *gy = (const TY *)a.gy + s0 * a.gy_stride + part * a.width;
    TX *gx = (TX *)a.y + s0 * a.y_stride + part * a.width;
    norm_batch<TX, E, NV, 1, ENDS, LANES == 2> inx[DEPTH];
    norm_batch<TY, E, NV, 1, ENDS, LANES == 2> ing[DEPTH];
    // row `ahead` from the present one, or that one again if the team has no such row
    auto load = [&](int k, int ahead) {
        const int64_t n = row + ahead * a.step < end ? ahead : 0;
        inx[k].load(x + n * a.x_step, 0, row, end, a, at.at);
        ing[k].load(gy + n * a.gy_step, 0, row, end, a, at.at);
    };
    if (row < end) {
#pragma unroll
        for (int k = 0; k < (EARLY ? DEPTH : DEPTH - 1); ++k)
            load(k, k);
    }
    const uint64_t offset = DROP ? fae_drop_offset(a.drop) : 0;
    float gamma[NV][E], dgamma[NV][E], dbeta[NV][E];
    norm_weights<ENDS, DROP, E, NV>(a.gamma, 1.f, a, part, at.at, gamma);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e)
            dgamma[j][e] = dbeta[j][e] = 0.f;
    static_assert(NV > 1 || DEPTH % 2 == 0, "rows whose masks are made together");
    norm_mask<E> mask[2][NV]; // of two rows where a lane has one chunk
    while (row < end) {
#pragma unroll
        for (int k = 0; k < DEPTH; ++k) {
            if constexpr (!EARLY)
                load((k + DEPTH - 1) % DEPTH, DEPTH - 1);
            if constexpr (DROP) {
                if constexpr (NV > 1)
                    norm_row_masks<E, NV>(mask[k & 1], at.at, row, offset, a.drop);
                else if (k % 2 == 0)
                    norm_masks<E>(mask[0][0], mask[1][0], at.at[0].col, row, at.at[0].col, row + a.step, offset, a.drop);
            }
            float v[NV][E], g[NV][E];
            inx[k].get(0, a, at.at, v);
            ing[k].get(0, a, at.at, g);
            if constexpr (EARLY)
                load(k, DEPTH);
            const float rstd = norm_center<ENDS, LANES, WAVES, NV, E>(v, at.at, a, team);
            float c1 = 0.f, c2 = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if constexpr (DROP)
                    mask[k & 1][j].drop(g[j], a.drop);
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
                fae_store<TX, E, ENDS>(gx, g[j], at.at[j], norm_sure<NV>(j));
            }
            row += a.step;
            if (row >= end)
                break;
            x += a.x_step;
            gy += a.gy_step;
            gx += a.y_step;
        }
    }
    if (!a.pgamma && !a.pbeta)
        return;
    if constexpr (DROP) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                dgamma[j][e] *= a.drop.scale;
                dbeta[j][e] *= a.drop.scale;
            }
    }
    // The sums go out a row per team, or where a workgroup has more teams than there are parts a row per part, the teams of a part
    // added up in LDS.
    if (a.in_regs) {
        const uint32_t r = a.direct ? part : at.q;
        if (a.direct && at.q >= a.step)
            return;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (a.pgamma)
                fae_store<float, E, ENDS>(a.pgamma + (int64_t)r * a.pitch, dgamma[j], at.at[j]);
            if (a.pbeta)
                fae_store<float, E, ENDS>(a.pbeta + (int64_t)r * a.pitch, dbeta[j], at.at[j]);
        }
        return;
    }
    if constexpr (!WAVES) {
        constexpr int TEAMS = THREADS / LANES, ROW = LANES * NV * E;
        __shared__ float sums[TEAMS * ROW], pieces[THREADS];
        for (int which = 0; which < 2; ++which) {
            float *out = which ? a.pbeta : a.pgamma;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    sums[threadIdx.x / LANES * ROW + at.at[j].col + e] = which ? dbeta[j][e] : dgamma[j][e];
            __syncthreads();
            if (!out)
                continue;
            // several threads to an output where there are fewer of these than threads
            const uint32_t n = a.part_rows * a.width, split = n < THREADS ? THREADS / n : 1;
            for (uint32_t i = threadIdx.x; i < n * split; i += THREADS) {
                const uint32_t piece = i / n, o = i - piece * n, k = o / a.width, c = o - k * a.width;
                float s = 0.f;
                for (uint32_t t = k + piece * a.n_parts; t < TEAMS; t += split * a.n_parts)
                    s += sums[t * ROW + c];
                if (split == 1)
                    out[(int64_t)(blockIdx.x * a.part_rows + k) * a.pitch + c] = s;
                else
                    pieces[i] = s;
            }
            if (split == 1)
                continue;
            __syncthreads();
            if (threadIdx.x < n) {
                float s = pieces[threadIdx.x];
                for (uint32_t q = 1; q < split; ++q)
                    s += pieces[threadIdx.x + q * n];
                const uint32_t k = threadIdx.x / a.width;
                out[(int64_t)(blockIdx.x * a.part_rows + k) * a.pitch + threadIdx.x - k * a.width] = s;
            }
        }
    }
}

// ---------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------
// rows of a team whose loads go out together: up to 64 bytes of a lane
constexpr int norm_fwd_rows(int nv) { return nv == 1 ? 4 : nv == 2 ? 2 : 1; }
// How the backward's loads run ahead.  Two rows held (four: 16 384 x 26 x 64 62 -> 65 us, 50 001 x 26 x 64 with dropout 152 -> 160); fp32 rows of
// several waves with one row's registers, filled again as soon as its values are taken (16 384 x 4096 150 -> 140 us, 40 000 x 2048 with
// dropout 171 -> 158; 16-bit rows, with twice the values per lane, 133 -> 139 for 65 536 x 1664); one row and nothing ahead where a
// workgroup of 1024 lanes, with 128 registers each, holds 16 values in a lane (4096 x 16 384 bf16 148 -> 97 us, with one filled early 136).
// Those 16 values take up to eight registers each (x, g, their raw words, gamma, the two sums), and do not all fit: fp32 rows above 8192
// values keep 6 to 40 registers' worth in scratch, 28 to 164 bytes a lane, 16-bit ones with dropout on rows that do not fill
// the lanes 6 to 17 (2441 x 16 384 fp32 112 us, 4.3 TB/s; bf16 67 us, 3.6).
constexpr bool norm_bwd_early(int nv, int chunk, int threads, bool waves) { return waves && threads == 512 && nv * chunk <= 8; }
constexpr int norm_bwd_depth(int nv, int chunk, int threads, bool waves)
{
    return norm_bwd_early(nv, chunk, threads, waves) || (threads == 1024 && nv * chunk > 8) ? 1 : 2;
}

// Chunks per lane at most, as long as a workgroup of 1024 then holds the row: 16 values in the forward; two in the backward, where a value
// takes eight registers (16 384 x 4096 fp32 with two and four 147 and 160 us; with one, bf16, 16 384 x 1664 53 instead of 48).
constexpr int norm_chunks(bool bwd, int chunk) { return bwd ? 2 : 16 / chunk; }

// how a launch shares out the rows
struct NormShape {
    int chunk;      // values per chunk
    int lanes;      // per team: 2 .. 64, or 64 times the waves
    int nv;         // chunks per lane
    uint32_t teams; // per workgroup
    uint32_t threads;
    uint32_t blocks, step;
    bool direct;        // backward: the only rows of sums are the gradients
    uint32_t part_rows; // backward: rows of sums per workgroup
    uint32_t n_sums;    // backward: rows of sums per part
    uint32_t pitch;
};

template <bool BWD, typename TX, typename TY, int LANES, int THREADS, bool WAVES, int NV, int ENDS, bool DROP>
static void norm_launch(fae_ctx *ctx, const NormShape &s, const NormArgs &a)
{
    if constexpr (BWD)
        FAE_LAUNCH(ctx, (norm_bwd_kernel<TX, TY, LANES, THREADS, WAVES, NV, norm_bwd_depth(NV, norm_chunk<TX>(), THREADS, WAVES), norm_bwd_early(NV, norm_chunk<TX>(), THREADS, WAVES), ENDS, DROP>), dim3(s.blocks), dim3(s.threads), 0,
                   ctx->stream, a);
    else
        FAE_LAUNCH(ctx, (norm_fwd_kernel<TX, TY, LANES, THREADS, WAVES, NV, norm_fwd_rows(NV), ENDS, DROP>), dim3(s.blocks), dim3(s.threads), 0, ctx->stream, a);
}

template <bool BWD, typename TX, typename TY, int LANES, int THREADS, bool WAVES, int NV, bool DROP>
static void norm_by_end(fae_ctx *ctx, const NormShape &s, const NormArgs &a)
{
    if (a.ends == FAE_WHOLE)
        norm_launch<BWD, TX, TY, LANES, THREADS, WAVES, NV, FAE_WHOLE, DROP>(ctx, s, a);
    else if (a.ends == FAE_CHUNKS)
        norm_launch<BWD, TX, TY, LANES, THREADS, WAVES, NV, FAE_CHUNKS, DROP>(ctx, s, a);
    else
        norm_launch<BWD, TX, TY, LANES, THREADS, WAVES, NV, FAE_ANY, DROP>(ctx, s, a);
}

template <bool BWD, typename TX, typename TY, int LANES, int THREADS, bool WAVES, int NV> static void norm_run(fae_ctx *ctx, const NormShape &s, const NormArgs &a)
{
    if (a.drop.below)
        norm_by_end<BWD, TX, TY, LANES, THREADS, WAVES, NV, true>(ctx, s, a);
    else
        norm_by_end<BWD, TX, TY, LANES, THREADS, WAVES, NV, false>(ctx, s, a);
}

template <bool BWD, typename TX, typename TY, int THREADS> static void norm_teams(fae_ctx *ctx, const NormShape &s, const NormArgs &a)
{
    switch (s.lanes) {
    case 2: norm_run<BWD, TX, TY, 2, THREADS, false, 1>(ctx, s, a); return;
    case 4: norm_run<BWD, TX, TY, 4, THREADS, false, 1>(ctx, s, a); return;
    case 8: norm_run<BWD, TX, TY, 8, THREADS, false, 1>(ctx, s, a); return;
    case 16: norm_run<BWD, TX, TY, 16, THREADS, false, 1>(ctx, s, a); return;
    case 32: norm_run<BWD, TX, TY, 32, THREADS, false, 1>(ctx, s, a); return;
    }
    if (s.nv == 1)
        norm_run<BWD, TX, TY, 64, THREADS, false, 1>(ctx, s, a);
    else if (s.nv == 2)
        norm_run<BWD, TX, TY, 64, THREADS, false, 2>(ctx, s, a);
    else if constexpr (norm_chunks(BWD, norm_chunk<TX>()) >= 4)
        norm_run<BWD, TX, TY, 64, THREADS, false, 4>(ctx, s, a);
}

template <bool BWD, typename TX, typename TY> static void norm_by_width(fae_ctx *ctx, const NormShape &s, const NormArgs &a)
{
    constexpr int MOST = norm_chunks(BWD, norm_chunk<TX>()), ALL = FAE_NORM_MAX_WIDTH / norm_chunk<TX>() / 1024; // per lane
    if (s.lanes <= 64) {
        if constexpr (BWD) {
            if (s.threads == 512) {
                norm_teams<BWD, TX, TY, 512>(ctx, s, a);
                return;
            }
        }
        norm_teams<BWD, TX, TY, 256>(ctx, s, a);
    } else if (s.lanes <= 512)
        norm_run<BWD, TX, TY, 64, 512, true, MOST>(ctx, s, a);
    else if (s.nv == MOST)
        norm_run<BWD, TX, TY, 64, 1024, true, MOST>(ctx, s, a);
    else if constexpr (ALL > MOST)
        norm_run<BWD, TX, TY, 64, 1024, true, ALL>(ctx, s, a);
}

// a file each, so that they are compiled beside each other
void norm_fwd_by_type(fae_ctx *ctx, const fae_norm *n, const NormShape &s, const NormArgs &a);
void norm_bwd_by_type(fae_ctx *ctx, const fae_norm *n, const NormShape &s, const NormArgs &a);
void norm_bwd16_by_type(fae_ctx *ctx, const fae_norm *n, const NormShape &s, const NormArgs &a);
void norm_fwd16_by_type(fae_ctx *ctx, const fae_norm *n, const NormShape &s, const NormArgs &a);
