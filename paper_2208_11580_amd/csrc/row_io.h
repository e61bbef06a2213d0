// Rows of activations and logits as kernels read and write them: 16 bytes at a time at any element's address, fp32 in
// registers.
#pragma once

#include "product4.h"

// Eight elements of a row as fp32; only the first `left` are touched.
template <int TYPE>
__device__ inline void load8(const void *p, int64_t at, int left, float (&v)[8])
{
    if (TYPE == OBC_F32) {
        const float *q = (const float *)p + at;
        if (left >= 8) {
            const floatx4 a = *(const floatx4_at4 *)q, b = *(const floatx4_at4 *)(q + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) { v[j] = a[j]; v[4 + j] = b[j]; }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < left ? q[j] : 0.f;
        }
    } else {
        const unsigned short *q = (const unsigned short *)p + at;
        unsigned short e[8];
        if (left >= 8) {
            const uintx4 w = *(const uintx4_at2 *)q;
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = (unsigned short)(w[j >> 1] >> (16 * (j & 1)));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = j < left ? q[j] : (unsigned short)0;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = TYPE == OBC_F16 ? (float)__builtin_bit_cast(_Float16, e[j]) : (float)__builtin_bit_cast(__bf16, e[j]);
    }
}

template <int TYPE>
__device__ inline void store8(void *p, int64_t at, int left, const float (&v)[8])
{
    if (left >= 8) {
        if (TYPE == OBC_F32) {
            float *q = (float *)p + at;
            *(floatx4_at4 *)q = floatx4{v[0], v[1], v[2], v[3]};
            *(floatx4_at4 *)(q + 4) = floatx4{v[4], v[5], v[6], v[7]};
        } else {
            uintx4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[j] = TYPE == OBC_F16 ? pair_f16(v[2 * j], v[2 * j + 1]) : pair_bf16(v[2 * j], v[2 * j + 1]);
            *(uintx4_at2 *)((unsigned short *)p + at) = w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < left) store_as<TYPE>(p, at + j, v[j]);
    }
}

// As store8, past the caches where `past` says so: results that are larger than what the dies' caches hold (4 MB each) only push out what
// is still to be read (layer norm of 4096 x 4096 in bf16: 22.7 us instead of 32, lookup of 16384 x 4096: 32 instead of 44).
constexpr int64_t kCaches = 32 << 20;

template <int TYPE>
__device__ inline void put8(void *p, int64_t at, int left, const float (&v)[8], bool past)
{
    if (left < 8 || !past) return store8<TYPE>(p, at, left, v);
    if (TYPE == OBC_F32) {
        __builtin_nontemporal_store(floatx4{v[0], v[1], v[2], v[3]}, (floatx4_at4 *)((float *)p + at));
        __builtin_nontemporal_store(floatx4{v[4], v[5], v[6], v[7]}, (floatx4_at4 *)((float *)p + at + 4));
    } else {
        uintx4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = TYPE == OBC_F16 ? pair_f16(v[2 * j], v[2 * j + 1]) : pair_bf16(v[2 * j], v[2 * j + 1]);
        __builtin_nontemporal_store(w, (uintx4_at2 *)((unsigned short *)p + at));
    }
}

// N words moved to the front by `by` half-words (HALF) or words, `fill` behind them; by a power of two at a time
template <bool HALF, int N>
__device__ inline void move_words(unsigned (&w)[N], int by, unsigned fill)
{
#pragma unroll
    for (int step = N / 2; step > 0; step >>= 1) {
        const bool on = by & (HALF ? 2 * step : step);
#pragma unroll
        for (int j = 0; j < N; ++j) w[j] = on ? (j + step < N ? w[j + step < N ? j + step : j] : fill) : w[j];
    }
    if (HALF) {
        const bool on = by & 1;
#pragma unroll
        for (int j = 0; j < N; ++j) w[j] = on ? w[j] >> 16 | (j + 1 < N ? w[j + 1 < N ? j + 1 : j] : fill) << 16 : w[j];
    }
}

// 16 bytes of a row at column c of d, `fill` beyond its end (in both halves of a word).  At the row's end the last 16 bytes are read and
// moved, for one load instead of several that wait for each other; only a row shorter than that goes element by element.
template <int TYPE>
__device__ inline void load_words(const void *p, int64_t base, int c, int d, unsigned fill, unsigned (&w)[4])
{
    constexpr int E = TYPE == OBC_F32 ? 4 : 8;
    const char *const row = (const char *)p + base * (16 / E);
    if (c + E <= d || (d >= E && c < d)) {
        const char *const at = row + (unsigned)(c + E <= d ? c : d - E) * (16u / E);
        const uintx4 v = TYPE == OBC_F32 ? __builtin_bit_cast(uintx4, (floatx4) * (const floatx4_at4 *)at) : (uintx4) * (const uintx4_at2 *)at;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = v[j];
        if (c + E > d) move_words<TYPE != OBC_F32>(w, c + E - d, fill);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = fill;
    if (c >= d) return;
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (c + j < d) {
            if (TYPE == OBC_F32) w[j & 3] = ((const unsigned *)row)[c + j];
            else w[j >> 1] = j & 1 ? (w[j >> 1] & 0xffffu) | (unsigned)((const unsigned short *)row)[c + j] << 16
                                   : (w[j >> 1] & 0xffff0000u) | ((const unsigned short *)row)[c + j];
        }
}

// Eight elements of a row of d at column c as fp32, zeros beyond its end
template <int TYPE>
__device__ inline void load8_of(const void *p, int64_t base, int c, int d, float (&v)[8])
{
    unsigned w[2][4];
    load_words<TYPE>(p, base, c, d, 0u, w[0]);
    if (TYPE == OBC_F32) load_words<TYPE>(p, base, c + 4, d, 0u, w[1]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const unsigned e = TYPE == OBC_F32 ? w[j >> 2][j & 3] : w[0][j >> 1];
        v[j] = TYPE == OBC_F32 ? __builtin_bit_cast(float, e) : TYPE == OBC_F16 ? (j & 1 ? half_hi(e) : half_lo(e)) : (j & 1 ? bf16_hi(e) : bf16_lo(e));
    }
}

// Eight elements on their way, in their own type
template <int TYPE>
struct Eight {
    uintx4 v[TYPE == OBC_F32 ? 2 : 1];

    __device__ void load(const void *p, int64_t at, int left)
    {
        if (left >= 8) {
            if (TYPE == OBC_F32) {
                v[0] = __builtin_bit_cast(uintx4, (floatx4) * (const floatx4_at4 *)((const float *)p + at));
                v[TYPE == OBC_F32] = __builtin_bit_cast(uintx4, (floatx4) * (const floatx4_at4 *)((const float *)p + at + 4));
            } else {
                v[0] = *(const uintx4_at2 *)((const unsigned short *)p + at);
            }
            return;
        }
        unsigned e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            e[j] = j >= left ? 0u : TYPE == OBC_F32 ? ((const unsigned *)p)[at + j] : ((const unsigned short *)p)[at + j];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[0][j] = TYPE == OBC_F32 ? e[j] : e[2 * j] | e[2 * j + 1] << 16;
            if (TYPE == OBC_F32) v[TYPE == OBC_F32][j] = e[4 + j];
        }
    }
    __device__ void get(float (&f)[8]) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned w = TYPE == OBC_F32 ? v[j >> 2][j & 3] : v[0][j >> 1];
            f[j] = TYPE == OBC_F32 ? __builtin_bit_cast(float, w) : TYPE == OBC_F16 ? (j & 1 ? half_hi(w) : half_lo(w)) : (j & 1 ? bf16_hi(w) : bf16_lo(w));
        }
    }
};

// The larger of two magnitudes; an infinity or a NaN is larger than any number (as their bits are), where fmaxf would drop the NaN.
__device__ inline float larger(float top, float v)
{
    const unsigned a = __builtin_bit_cast(unsigned, top), b = __builtin_bit_cast(unsigned, v) & 0x7fffffffu;
    return __builtin_bit_cast(float, a > b ? a : b);
}

template <int TYPE>
__device__ inline float load_as(const void *p, int64_t at)
{
    return TYPE == OBC_F32 ? ((const float *)p)[at] : TYPE == OBC_F16 ? (float)((const _Float16 *)p)[at] : (float)((const __bf16 *)p)[at];
}

// Logits of a 16-byte piece
template <int TYPE>
struct Piece {
    static constexpr int E = TYPE == OBC_F32 ? 4 : 8;
    uintx4 v;

    // From logit `c` of the row at z on.  (A row's address is the same for all threads, and 32 bits of offset to it take half
    // the registers of an address.)
    __device__ void load(const char *z, int c)
    {
        const char *at = z + (unsigned)c * (16u / E);
        if (TYPE == OBC_F32) v = __builtin_bit_cast(uintx4, (floatx4) * (const floatx4_at4 *)at);
        else v = *(const uintx4_at2 *)at;
    }
    // the same at the end of a row of V: -inf beyond it
    __device__ void load_end(const char *z, int c, int V)
    {
        if (c + E <= V) return load(z, c);
        constexpr unsigned low = TYPE == OBC_F32 ? 0xff800000u : TYPE == OBC_F16 ? 0xfc00u : 0xff80u;
        unsigned e[E];
#pragma unroll
        for (int j = 0; j < E; ++j)
            e[j] = c + j >= V ? low : TYPE == OBC_F32 ? ((const unsigned *)z)[(unsigned)(c + j)] : ((const unsigned short *)z)[(unsigned)(c + j)];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = TYPE == OBC_F32 ? e[j] : e[2 * j % E] | e[(2 * j + 1) % E] << 16;
    }
    __device__ float operator[](int j) const
    {
        if (TYPE == OBC_F32) {
            const unsigned w = v[j & 3];
            return __builtin_bit_cast(float, w);
        }
        const unsigned w = v[j >> 1];
        if (TYPE == OBC_F16) return j & 1 ? half_hi(w) : half_lo(w);
        return __builtin_bit_cast(float, j & 1 ? w & 0xffff0000u : w << 16);
    }
    // keeps the compiler from carrying the piece's fp32 values, twice its registers, from one pass over the row to the next
    __device__ void forget() { asm volatile("" : "+v"(v)); }
    static __device__ void store(char *p, int c, const float (&g)[E])
    {
        char *at = p + (unsigned)c * (16u / E);
        if (TYPE == OBC_F32) {
            *(floatx4_at4 *)at = floatx4{g[0], g[1], g[2], g[3]};
        } else {
            uintx4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[j] = TYPE == OBC_F16 ? pair_f16(g[2 * j % E], g[(2 * j + 1) % E]) : pair_bf16(g[2 * j % E], g[(2 * j + 1) % E]);
            *(uintx4_at2 *)at = w;
        }
    }
    static __device__ void store_end(char *p, int c, int V, const float (&g)[E])
    {
        if (c + E <= V) return store(p, c, g);
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (c + j < V) store_as<TYPE>(p, c + j, g[j]);
    }
};

// A wave's lanes joined by an operation that is the same in either order; every lane gets the same result.  Steps between the lanes of
// 16 and swaps of halves: a few cycles each, where a shuffle goes through LDS.
template <int CONTROL>
__device__ inline unsigned from_lane(unsigned v)
{
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, 0xf, 0xf, true);
}

template <int LANES = 64, typename V, typename OP>
__device__ inline V join_lanes(V v, OP op)
{
    static_assert(sizeof(V) == 4 && (LANES == 32 || LANES == 64), "");
    const auto bits = [](V x) { return __builtin_bit_cast(unsigned, x); };
    const auto value = [](unsigned x) { return __builtin_bit_cast(V, x); };
    v = op(v, value(from_lane<0xb1>(bits(v))));       // lanes 1 0 3 2
    v = op(v, value(from_lane<0x4e>(bits(v))));       // lanes 2 3 0 1
    v = op(v, value(from_lane<0x141>(bits(v))));      // eight lanes turned round
    v = op(v, value(from_lane<0x140>(bits(v))));      // sixteen lanes turned round
    auto pair = __builtin_amdgcn_permlane16_swap(bits(v), bits(v), false, false);
    v = op(value(pair[0]), value(pair[1]));
    if (LANES == 32) return v;
    pair = __builtin_amdgcn_permlane32_swap(bits(v), bits(v), false, false);
    return op(value(pair[0]), value(pair[1]));
}

__device__ inline float sum_lanes(float v)
{
    return join_lanes(v, [](float a, float b) { return a + b; });
}
