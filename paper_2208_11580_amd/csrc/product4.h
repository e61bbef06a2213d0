// What the products with 4-bit weights share: operand types of the matrix instructions, loads of
// activations in their order, codes as numbers.
#pragma once

#include "pack4.h"

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx2 __attribute__((ext_vector_type(2)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
// the same, at any element's address
typedef unsigned uintx4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned uintx2_at1 __attribute__((ext_vector_type(2), aligned(1)));
typedef float floatx4_at4 __attribute__((ext_vector_type(4), aligned(4)));

// A code q as the 16-bit number 16 + q, exactly: the code in the top four bits of the mantissa under the
// exponent of 16.  (A base of 16 costs the sums two or three bits by cancellation, where 128 or 1024, which the
// code's bits at the bottom of the mantissa would give, cost five or eight.)
constexpr float kCodeBase = 16.f;

// dword i of the operand holds the columns 2 i and 2 i + 1.  (Mask and base in registers of either kind: an instruction
// has room for one constant, and with two the and and the or become two instructions.)
__device__ inline uintx4 codes_bf16(unsigned w)
{
    unsigned mask = 0x00780078u, base = 0x41804180u;
    asm("" : "+s"(mask), "+v"(base));
    return uintx4{((w << 3) & mask) | base, ((w >> 1) & mask) | base, ((w >> 5) & mask) | base, ((w >> 9) & mask) | base};
}

__device__ inline uintx4 codes_f16(unsigned w)
{
    unsigned mask = 0x03c003c0u, base = 0x4c004c00u;
    asm("" : "+s"(mask), "+v"(base));
    return uintx4{((w << 6) & mask) | base, ((w << 2) & mask) | base, ((w >> 2) & mask) | base, ((w >> 6) & mask) | base};
}

// A code q as 2 q - 15, exactly, in the same order: the sums have no large common part to take out again.  q >= 8 is 2 k + 1 and q < 8
// its opposite with k = (q & 7) or 7 - q, of which two permutes look up both bytes.
template <bool HALF>
__device__ inline uintx4 codes_centred(unsigned w)
{
    auto four = [](unsigned q, unsigned &first, unsigned &second) {      // a code to a byte
        const unsigned neg = ~q & 0x08080808u, k = (q ^ (neg - (neg >> 3))) & 0x07070707u;
        const unsigned hi = (HALF ? __builtin_amdgcn_perm(0x4b4a4948u, 0x4745423cu, k) : __builtin_amdgcn_perm(0x41414141u, 0x4040403fu, k)) | (neg << 4);
        const unsigned lo = HALF ? __builtin_amdgcn_perm(0x80808080u, 0u, k) : __builtin_amdgcn_perm(0x70503010u, 0xe0a04080u, k);
        first = __builtin_amdgcn_perm(hi, lo, 0x06020400u);
        second = __builtin_amdgcn_perm(hi, lo, 0x07030501u);
    };
    unsigned v0, v1, v2, v3;
    four(w & 0x0f0f0f0fu, v0, v2);
    four((w >> 4) & 0x0f0f0f0fu, v1, v3);
    return uintx4{v0, v1, v2, v3};
}

// Eight codes as bytes, in the order of the columns 0 4 1 5 2 6 3 7; bytes_like_codes brings eight 8-bit
// inputs into the same order.
__device__ inline uintx2 codes_i8(unsigned w) { return uintx2{w & 0x0f0f0f0fu, (w >> 4) & 0x0f0f0f0fu}; }

__device__ inline uintx2 bytes_like_codes(uintx2 x)
{
    return uintx2{__builtin_amdgcn_perm(x.y, x.x, 0x05010400u), __builtin_amdgcn_perm(x.y, x.x, 0x07030602u)};
}

__device__ inline float bf16_lo(unsigned w) { return __builtin_bit_cast(float, w << 16); }
__device__ inline float bf16_hi(unsigned w) { return __builtin_bit_cast(float, w & 0xffff0000u); }

__device__ inline floatx4 mfma_bf16(uintx4 a, uintx4 b, floatx4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ inline floatx4 mfma_f16(uintx4 a, uintx4 b, floatx4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(halfx8, a), __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
}

// 32 columns of 8-bit inputs: half the depth of this type's instruction, so that a group of 32 ends between two
__device__ inline intx4 mfma_i8(uintx2 a, uintx2 b, intx4 c)
{
    return __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, a), __builtin_bit_cast(long, b), c, 0, 0, 0);
}

__device__ inline unsigned pair_bf16(float lo, float hi)
{
    return __builtin_bit_cast(unsigned, bf16x2{(__bf16)lo, (__bf16)hi});
}

__device__ inline unsigned pair_f16(float lo, float hi)
{
    return __builtin_bit_cast(unsigned, halfx2{(_Float16)lo, (_Float16)hi});
}

// x = h + m + l, three bf16 numbers, exact from 2^-110 on; an infinity or a NaN stays in h alone.
__device__ inline void split3(float x, float &h, float &m, float &l)
{
    h = (float)(__bf16)x;
    const float r = x - h;
    const bool finite = fabsf(h) < __builtin_inff();
    m = finite ? (float)(__bf16)r : 0.f;
    l = finite ? (float)(__bf16)(r - m) : 0.f;
}

// (By value: a bit cast of a vector's element in place takes the vector's first.)
__device__ inline halfx2 half_pair(unsigned w) { return __builtin_bit_cast(halfx2, w); }
__device__ inline unsigned bits_of(halfx2 v) { return __builtin_bit_cast(unsigned, v); }
__device__ inline float half_lo(unsigned w) { return (float)__builtin_bit_cast(_Float16, (unsigned short)(w & 0xffffu)); }
__device__ inline float half_hi(unsigned w) { return (float)__builtin_bit_cast(_Float16, (unsigned short)(w >> 16)); }

template <int YT>
__device__ inline void store_as(void *y, int64_t at, float v)
{
    if (YT == OBC_F32) ((float *)y)[at] = v;
    else if (YT == OBC_F16) ((_Float16 *)y)[at] = (_Float16)v;
    else ((__bf16 *)y)[at] = (__bf16)v;
}

typedef __attribute__((address_space(1))) const void *global_ptr;
typedef __attribute__((address_space(3))) void *lds_ptr;

// s_waitcnt vmcnt(n) lgkmcnt(0): all loads but the n newest, and every access to LDS
constexpr int wait_loads(int n) { return 0x0070 | (n & 15) | (n >> 4) << 14; }

// A barrier that waits for nothing itself: __syncthreads (and a fence) would wait for every load on its way, the newest stages'
// among them.  wait_loads goes before it: what a wave has read from LDS has then arrived, and its share of the next stage is there.
__device__ inline void stage_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Consecutive workgroups go to different dies, each with a cache of its own: a die takes a run of tiles.
__device__ inline int tile_of(int id, int tiles)
{
    const int each = tiles >> 3, left = tiles & 7, die = id & 7;
    return die * each + (die < left ? die : left) + (id >> 3);
}

// The sum of an element's slices, n apart, in their order; several loads on their way at a time.
__device__ inline float add_slices(const float *part, int64_t n, int slices)
{
    constexpr int AT = 8;
    float v = 0.f;
    int s = 0;
    for (; s + AT <= slices; s += AT) {
        float x[AT];
#pragma unroll
        for (int i = 0; i < AT; ++i) x[i] = part[(s + i) * n];
#pragma unroll
        for (int i = 0; i < AT; ++i) v += x[i];
    }
    for (; s < slices; ++s) v += part[s * n];
    return v;
}

static inline bool float_type(int type) { return type == OBC_F32 || type == OBC_F16 || type == OBC_BF16; }
static inline size_t size_of_type(int type) { return type == OBC_F32 ? 4 : type == OBC_I8 ? 1 : 2; }
