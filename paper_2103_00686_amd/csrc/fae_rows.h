// What layer norm and dropout share: rows of fp32, bf16 or fp16 values in parts, their host checks, and the
// generator of the dropout mask (gfx950).
#pragma once

#include "fae_internal.h"

typedef __bf16 fae_bf16;
typedef _Float16 fae_f16;

// ---------------------------------------------------------------------------------
// host checks
// ---------------------------------------------------------------------------------
static inline int fae_type_size(int32_t type) { return type == FAE_F32 ? 4 : 2; }

// one side of a call: n_rows samples of `row` values, `stride` values apart
struct fae_rows {
    const void *p;
    int32_t type;
    int64_t stride;
};

// the checks of one buffer (n_rows > 0): there, aligned to its values, no row over the next, addressable
int32_t fae_check_rows(fae_ctx *ctx, const char *who, const char *what, const fae_rows &b, int64_t n_rows, int64_t row);
// an output beside an input of the same shape: the same rows or none in common
int32_t fae_check_overlap(fae_ctx *ctx, const char *who, const fae_rows &out, const fae_rows &in, int64_t n_rows, int64_t row);

// the dropout of a launch, as the kernels take it
struct fae_drop_args {
    uint32_t below;  // numbers below this one are dropped (0 .. 65536); 0: no dropout at all
    float scale;     // what the others are multiplied by
    uint32_t key[2];
    uint64_t offset;
    const uint64_t *d_offset;
};
int32_t fae_check_drop(fae_ctx *ctx, const char *who, const fae_drop *drop, fae_drop_args *out);

#ifdef __HIPCC__

// ---------------------------------------------------------------------------------
// chunks: E values, loaded and stored at once where all are there (the vector unit's accesses take any alignment of the values)
// ---------------------------------------------------------------------------------
template <typename T, int E> struct fae_vec {
    typedef T type __attribute__((ext_vector_type(E)));
    typedef type loose __attribute__((aligned(sizeof(T))));
};

// Where a lane's chunk of E values lies in a row of `width`.  Loads have no branch per lane or value (a load behind one waits for the
// loads in front of it): a chunk that the row's end cuts is loaded as the E values that end with the row and moved down when they
// are there, and lanes behind the row load that chunk too.  Rows shorter than a chunk are the exception.
template <int E> struct fae_place {
    uint32_t col;  // the chunk's first column
    uint32_t from; // the first column that is loaded
    int there;     // values of the chunk that exist, 0 .. E
    __device__ __forceinline__ void set(uint32_t c, uint32_t width)
    {
        col = c;
        there = c >= width ? 0 : (width - c < (uint32_t)E ? (int)(width - c) : E);
        const uint32_t last = width < (uint32_t)E ? 0 : width - E;
        from = c < last ? c : last;
    }
};
// How a launch's rows end: every lane's chunk whole; whole or absent; one cut by the end; no whole chunk at all.  Kernels are built for
// the first two, and for the others together (FAE_ANY).
enum { FAE_WHOLE, FAE_CHUNKS, FAE_CROOKED, FAE_SHORT };
#define FAE_ANY FAE_CROOKED
static inline int32_t fae_row_end(int64_t width, int chunk, int64_t lanes_width)
{
    return width == lanes_width ? FAE_WHOLE : (width < chunk ? FAE_SHORT : (width % chunk ? FAE_CROOKED : FAE_CHUNKS));
}
// ENDS: FAE_WHOLE, FAE_CHUNKS or FAE_ANY.  MAY_SHORT: a row may be shorter than a chunk (never where it has two).  sure: a chunk that is
// known to be whole whatever the rows' end (a constant where it is true)
template <typename T, int E, int ENDS, bool MAY_SHORT = true>
__device__ __forceinline__ typename fae_vec<T, E>::type fae_load(const T *row, const fae_place<E> &at, int ends)
{
    if (ENDS == FAE_ANY && MAY_SHORT && ends == FAE_SHORT) {
        typename fae_vec<T, E>::type v;
#pragma unroll
        for (int e = 0; e < E; ++e)
            v[e] = e < at.there ? row[e] : (T)0.f;
        return v;
    }
    return *(const typename fae_vec<T, E>::loose *)(row + (ENDS == FAE_WHOLE ? at.col : at.from));
}
// what fae_load brought, as it belongs: zeros where the row has no values (a cut chunk gets them by being moved down)
template <typename T, int E, int ENDS>
__device__ __forceinline__ void fae_settle(typename fae_vec<T, E>::type v, const fae_place<E> &at, int ends, float (&out)[E], bool sure = false)
{
    static_assert(sizeof(v) == 8 || sizeof(v) == 16, "8 or 16 bytes");
    if (ENDS != FAE_WHOLE && !sure) {
        if (ENDS == FAE_ANY && ends == FAE_CROOKED && at.there > 0) {
            const uint32_t sh = (at.col - at.from) * 8 * sizeof(T);
            if constexpr (sizeof(v) == 8) {
                v = __builtin_bit_cast(typename fae_vec<T, E>::type, __builtin_bit_cast(uint64_t, v) >> sh);
            } else {
                typedef uint64_t pair __attribute__((ext_vector_type(2)));
                pair w = __builtin_bit_cast(pair, v);
                const uint64_t lo = w[0], hi = w[1];
                const uint32_t s = sh & 63;
                const uint64_t h = hi >> s, l = (lo >> s) | ((hi << 1) << (63 - s));
                w[0] = sh < 64 ? l : h;
                w[1] = sh < 64 ? h : 0;
                v = __builtin_bit_cast(typename fae_vec<T, E>::type, w);
            }
        }
        typedef uint32_t words __attribute__((ext_vector_type(sizeof(v) / 4)));
        words w = __builtin_bit_cast(words, v);
#pragma unroll
        for (int i = 0; i < (int)sizeof(v) / 4; ++i)
            w[i] = at.there > 0 ? w[i] : 0u;
        v = __builtin_bit_cast(typename fae_vec<T, E>::type, w);
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        out[e] = (float)v[e];
}

template <typename T, int E, int ENDS> __device__ __forceinline__ void fae_store(T *row, const float (&v)[E], const fae_place<E> &at, bool sure = false)
{
    T *p = row + at.col;
    typename fae_vec<T, E>::type o;
#pragma unroll
    for (int e = 0; e < E; ++e)
        o[e] = (T)v[e];
    if (ENDS == FAE_WHOLE || sure || at.there == E) {
        *(typename fae_vec<T, E>::loose *)p = o;
    } else if (ENDS == FAE_ANY) {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < at.there)
                p[e] = o[e];
    }
}

// ---------------------------------------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011).  Its ten rounds are 20 products of 32 by 32 bits and 60 exclusive
// ors and additions, for eight values: 16 bits each decide as well as 32 would (a share of dropped values is kept to
// 2^-17), and half the generator's work is left out.
// ---------------------------------------------------------------------------------
struct fae_mask8 {
    uint32_t w[4]; // number j of the eight: half j & 1 of word j >> 1
    __device__ __forceinline__ uint32_t number(int j) const { return j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xffffu; }
};

__device__ __forceinline__ uint64_t fae_drop_offset(const fae_drop_args &d) { return d.offset + (d.d_offset ? *d.d_offset : 0); }

__device__ __forceinline__ uint32_t fae_xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

__device__ __forceinline__ fae_mask8 fae_philox(uint32_t group, uint32_t row, uint64_t offset, uint32_t k0, uint32_t k1)
{
    uint32_t c0 = group, c1 = row, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = fae_xor3((uint32_t)(b >> 32), c1, k0);
        c1 = (uint32_t)b;
        c2 = fae_xor3((uint32_t)(a >> 32), c3, k1);
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return fae_mask8{{c0, c1, c2, c3}};
}

// A dropped value is zero whatever it was: a choice, not a product.  The product is rounded to fp32 also where fp16 is
// stored: the compiler would multiply and round to fp16 in one instruction, and a result would depend on where it does.
__device__ __forceinline__ float fae_drop1(float v, uint32_t number, uint32_t below, float scale)
{
    float kept = v * scale;
    asm("" : "+v"(kept));
    return number < below ? 0.0f : kept;
}

#endif // __HIPCC__
