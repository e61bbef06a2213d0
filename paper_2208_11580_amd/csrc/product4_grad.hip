// obc_product4_grad: dx = dy W, the gradient of the inputs of a product with 4-bit weights.
//
//   dx[t, c] = sum_r dy[t, r] (offset + delta code)[r, c]
// The sum runs over the rows, whose steps differ, so the weights are formed before the product.  16-bit types: each as two
// numbers of half precision, 22 bits of it (rounded to one, its 11 bits changed 10 % of the bf16 results and 40 % of the fp16
// ones); a token's bf16 gradients, scaled by a power of two so that the largest is near 2^14, are half-precision numbers too (what
// that loses lies 2^-39 below the largest).  fp32: weights and gradients as three bf16 terms each, six of the nine
// products (what is left out is below 2^-24).
//
// A first launch lays out the gradients as the matrix instructions' operands want them and turns the codes, so that the
// lanes lie along the columns and a dword holds eight rows: 9 of a large product's 121 us.  The product then is like the
// forward one: gradients and codes through LDS, weights formed in registers once for a wave's tokens.  Few tokens leave too few
// tiles for the chip: the rows are cut into slices, whose sums a third launch adds in order.
//
// Bound by the matrix cores and the forming of weights, neither of which fills the time: 2048 tokens through 4096 x 4096 in bf16 take
// 121 us, 570 TFLOP/s of the product and twice that in the matrix cores, which in the tiles' 112 us are busy 50 % of the time, where the
// vector instructions issue 32 % of it; 77 tokens through 2304 x 1283 in fp32 19.4 us (12 the tiles, 4 the layout, 3 the sum of slices).
#include "product4.h"

namespace {

struct Args {
    const unsigned *codes;      // as packed
    const unsigned *scales;
    const void *dy;
    void *dx;
    int T, R, d, RB, KT, NG, SUB, tpg;
    int RT;                     // tiles of 128 rows
    int64_t lddy, lddx;
    // laid out in the workspace
    uint4 *rows;                // gradients: T x RT * 128, 16 bits, one or three planes
    float *back;                // T: what undoes a token's power of two
    unsigned *turned;           // codes: tile (column block cb, row tile rt) at (cb * RT + rt) * 256, as in pack4.h
    unsigned short *steps;      // NG x 2 x RT * 128: a group's steps, then its offsets
    unsigned char *wide;        // NG x RT * 2: whether a group has a weight beyond half precision among 64 rows
    float *part;                // slices x T x d
    int slices, per;            // slices of the rows, row tiles of a slice
};

// ---- layout -------------------------------------------------------------------------------------------------------
constexpr int kKeep = 4;      // pieces of a token's gradients that a thread keeps between the largest and the rounding

// Workgroups below `turns`: 128 rows x 128 columns of codes, through LDS; then the groups' steps; the others: a token's gradients.
template <int TYPE>
__global__ __launch_bounds__(256) void grad_lay_kernel(Args a, int64_t turns, int64_t scale_blocks)
{
    const int tid = threadIdx.x;
    if ((int64_t)blockIdx.x < turns) {
        __shared__ unsigned codes[2048 + 256];      // a dword of padding behind every eight
        auto at = [](int i) { return i + (i >> 3); };
        const int kt = (int)((int64_t)blockIdx.x / a.RT), rt = (int)((int64_t)blockIdx.x % a.RT);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int e = h * 256 + tid, rb = rt * 8 + (e >> 6);      // 16-byte place of the eight tiles
            uintx4 v = {0u, 0u, 0u, 0u};
            if (rb < a.RB) v = *((const uintx4 *)a.codes + ((int64_t)rb * a.KT + kt) * 64 + (e & 63));
#pragma unroll
            for (int j = 0; j < 4; ++j) codes[at(e * 4 + j)] = v[j];
        }
        __syncthreads();
        // a thread turns an octet of rows x an octet of columns; octets count 4 s + quad
        const int co = tid & 15, ro = tid >> 4;
        unsigned in[8], out[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) in[i] = codes[at((ro >> 1) * 256 + ((co & 3) * 16 + (ro & 1) * 8 + i) * 4 + (co >> 2))];
        // nibble of element e: (e >> 1) + 4 (e & 1)
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            unsigned w = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) w |= ((in[i] >> (4 * ((c >> 1) + 4 * (c & 1)))) & 15u) << (4 * ((i >> 1) + 4 * (i & 1)));
            out[c] = w;
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 8; ++c) codes[at((co >> 1) * 256 + ((ro & 3) * 16 + (co & 1) * 8 + c) * 4 + (ro >> 2))] = out[c];
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int e = h * 256 + tid;
            uintx4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = codes[at(e * 4 + j)];
            *((uintx4 *)a.turned + ((int64_t)(kt * 8 + (e >> 6)) * a.RT + rt) * 64 + (e & 63)) = v;
        }
        return;
    }
    if ((int64_t)blockIdx.x < turns + scale_blocks) {
        const int64_t i = ((int64_t)blockIdx.x - turns) * 256 + tid, len = (int64_t)a.RT * 128;
        if (i >= len * a.NG) return;
        const int g = (int)(i / len);
        const int64_t r = i - g * len;
        unsigned w = 0;
        if (r < a.R)
            w = a.SUB > 1 ? a.scales[(((r >> 4) * a.KT + g / a.SUB) * 16 + (r & 15)) * a.SUB + g % a.SUB] : a.scales[((r >> 4) * a.NG + g) * 16 + (r & 15)];
        a.steps[2 * g * len + r] = (unsigned short)w;
        a.steps[(2 * g + 1) * len + r] = (unsigned short)(w >> 16);
        const float first = half_hi(w), last = fmaf(15.f, half_lo(w), first);
        const bool wide = __any(!(fmaxf(fabsf(first), fabsf(last)) <= 65504.f));      // (a wave's 64 rows belong to one group)
        if ((tid & 63) == 0) a.wide[i >> 6] = wide;
        return;
    }
    const int64_t t = (int64_t)blockIdx.x - turns - scale_blocks;
    const int pieces = a.RT * 16, whole = a.R >> 3;      // pieces of eight elements, of which `whole` lie inside the row
    const int64_t at = t * a.lddy, plane = (int64_t)a.T * pieces;
    auto load = [&](int p, float (&v)[8]) {
        const int r = p * 8;
        if (p < whole) {
            if (TYPE == OBC_F32) {
                const floatx4 lo = *(const floatx4_at4 *)((const float *)a.dy + at + r), hi = *(const floatx4_at4 *)((const float *)a.dy + at + r + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) { v[j] = lo[j]; v[4 + j] = hi[j]; }
            } else {
                const uintx4 w = *(const uintx4_at2 *)((const unsigned short *)a.dy + at + r);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned x = w[j];
                    v[2 * j] = TYPE == OBC_F16 ? half_lo(x) : bf16_lo(x);
                    v[2 * j + 1] = TYPE == OBC_F16 ? half_hi(x) : bf16_hi(x);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (TYPE == OBC_F32) v[j] = r + j < a.R ? ((const float *)a.dy)[at + r + j] : 0.f;
                else if (TYPE == OBC_F16) v[j] = r + j < a.R ? (float)((const _Float16 *)a.dy)[at + r + j] : 0.f;
                else v[j] = r + j < a.R ? (float)((const __bf16 *)a.dy)[at + r + j] : 0.f;
            }
        }
    };
    auto put = [&](int p, const float (&v)[8], float up) {
        uintx4 w[3];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (TYPE == OBC_F32) {
                float h0, m0, l0, h1, m1, l1;
                split3(v[2 * j], h0, m0, l0);
                split3(v[2 * j + 1], h1, m1, l1);
                w[0][j] = pair_bf16(h0, h1);
                w[1][j] = pair_bf16(m0, m1);
                w[2][j] = pair_bf16(l0, l1);
            } else {
                w[0][j] = pair_f16(v[2 * j] * up, v[2 * j + 1] * up);
            }
        }
        uintx4 *const to = (uintx4 *)a.rows + t * pieces + p;
        to[0] = w[0];
        if (TYPE == OBC_F32) {
            to[plane] = w[1];
            to[2 * plane] = w[2];
        }
    };
    if (TYPE != OBC_BF16) {
        for (int p = tid; p < pieces; p += 256) {
            float v[8];
            load(p, v);
            put(p, v, 1.f);
        }
        return;
    }
    __shared__ float tops[4];
    float kept[kKeep][8], top = 0.f;
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
        if (i * 256 + tid < pieces) {
            load(i * 256 + tid, kept[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(kept[i][j]));
        }
    for (int p = kKeep * 256 + tid; p < pieces; p += 256) {
        float v[8];
        load(p, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[j]));
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    // 2^14 / the power of two below the largest; both it and its inverse are normal numbers
    int e;
    (void)frexpf(top, &e);
    const float up = top > 0.f && top < __builtin_inff() ? ldexpf(1.f, e > -111 ? 15 - e : 126) : 1.f;
    if (tid == 0) a.back[t] = 1.f / up;
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
        if (i * 256 + tid < pieces) put(i * 256 + tid, kept[i], up);
    for (int p = kKeep * 256 + tid; p < pieces; p += 256) {
        float v[8];
        load(p, v);
        put(p, v, up);
    }
}

// ---- product ------------------------------------------------------------------------------------------------------
// Eight weights of a lane's column, of the eight rows that `steps` and `offsets` (half precision) belong to, each as two numbers of
// half precision: the first cut off, the second what it leaves, so that a weight is exact below 1 and off by 2^-22 above.  WIDE: a 32nd
// of them, for weights beyond half precision (which end below 2^20).
template <bool WIDE>
__device__ inline void weights_f16(unsigned w, uintx4 steps, uintx4 offsets, uintx4 (&r)[2])
{
    const uintx4 c = codes_f16(w);
    const _Float16 b = (_Float16)-16.f, s = (_Float16)(1.f / 32.f);
    const halfx2 base = {b, b}, part = {s, s};
    // (not known to be -1, or the mixed-precision multiply-add becomes a conversion and a subtraction)
    float minus = -1.f;
    asm("" : "+s"(minus));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        halfx2 q = half_pair(c[j]) + base, step = half_pair(steps[j]), off = half_pair(offsets[j]);
        if (WIDE) {
            q *= part;
            off *= part;
        }
        const float v0 = fmaf((float)step.x, (float)q.x, (float)off.x), v1 = fmaf((float)step.y, (float)q.y, (float)off.y);
        const halfx2 hi = __builtin_bit_cast(halfx2, __builtin_amdgcn_cvt_pkrtz(v0, v1));
        r[0][j] = bits_of(hi);
        r[1][j] = bits_of(halfx2{(_Float16)fmaf(minus, (float)hi.x, v0), (_Float16)fmaf(minus, (float)hi.y, v1)});
    }
}

// The same in three bf16 terms, eight bits of the weight after the other: cut off rather than rounded, which is as exact and half
// the instructions (500 tokens through 4096 x 4096: 186 -> 151 us).  Weights are finite, steps and offsets being so.
__device__ inline void weights_split(unsigned w, uintx4 steps, uintx4 offsets, uintx4 (&r)[3])
{
    const uintx4 c = codes_bf16(w);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float v[2] = {fmaf(half_lo(steps[j]), bf16_lo(c[j]) - kCodeBase, half_lo(offsets[j])),
                      fmaf(half_hi(steps[j]), bf16_hi(c[j]) - kCodeBase, half_hi(offsets[j]))};
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            const unsigned lo = __builtin_bit_cast(unsigned, v[0]), hi = __builtin_bit_cast(unsigned, v[1]);
            r[p][j] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
            v[0] -= bf16_hi(lo);
            v[1] -= bf16_hi(hi);
        }
    }
}

template <bool V>
struct Flag {
    static constexpr bool value = V;
};

template <int TYPE, int BM, int BN>
struct Tile {
    // planes of the gradients, terms of a weight; a wave takes all tokens and 32 columns, so that every weight is formed once
    static constexpr int P = TYPE == OBC_F32 ? 3 : 1, TERMS = TYPE == OBC_F32 ? 3 : 2, WAVES = BN / 32, MF = BM / 16, NF = 2;
    static constexpr int XN = P * BM * 16, CN = BN * 4;      // 16-byte places of a stage: gradients, codes; then steps
    static constexpr int PLACES = XN + CN + WAVES * 32;
    // loads of a wave for a stage: 64 places each, and twice 64 times 4 bytes of steps and offsets, a quarter of a tile's columns
    static constexpr int XL = XN / 64 / WAVES, CL = CN / 64 / WAVES, LOADS = XL + CL + 2;
    static constexpr int STAGES = P == 3 && BM > 32 ? 2 : 3;      // what 160 KB hold
    static_assert(XN % (64 * WAVES) == 0 && CN % (64 * WAVES) == 0, "whole loads");
};

// BM tokens x BN columns to a workgroup: gradients, codes and steps of 128 rows go through two or three stages of LDS
// in turn, as in the forward product.
template <int TYPE, int BM, int BN>
__global__ __launch_bounds__(BN * 2, 2) void grad_tiles_kernel(Args a, int mtiles, int ntiles)
{
    using C = Tile<TYPE, BM, BN>;
    constexpr int P = C::P, TERMS = C::TERMS, MF = C::MF, NF = C::NF, STAGES = C::STAGES;
    __shared__ uintx4 lds0[C::PLACES], lds1[C::PLACES], lds2[STAGES > 2 ? C::PLACES : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, quad = lane >> 4;
    const int tiles = mtiles * ntiles, slice = blockIdx.x / tiles, tile = tile_of(blockIdx.x % tiles, tiles);
    const int t0 = (tile % mtiles) * BM, kt = tile / mtiles * (BN / 128);      // first token, first tile of 128 columns
    const int rt0 = slice * a.per, rt1 = rt0 + a.per < a.RT ? rt0 + a.per : a.RT;
    const int64_t plane = (int64_t)a.T * a.RT * 256;       // bytes
    const int64_t len = (int64_t)a.RT * 128;
    // where this lane's loads come from, at the slice's first tile; piece o of token t at place o ^ (t mod 16) of its row
    const char *xsrc[C::XL], *csrc[C::CL], *ssrc;
#pragma unroll
    for (int i = 0; i < C::XL; ++i) {
        const int first = (i * C::WAVES + wave) * 4;
        const int p = P > 1 ? first / BM : 0, t = first - p * BM + (lane >> 4);
        const int row = t0 + t < a.T ? t0 + t : a.T - 1;
        xsrc[i] = (const char *)a.rows + p * plane + ((int64_t)row * a.RT + rt0) * 256 + ((lane & 15) ^ (t & 15)) * 16;
    }
#pragma unroll
    for (int i = 0; i < C::CL; ++i) {
        int cb = kt * 8 + i * C::WAVES + wave;
        if (cb >= a.KT * 8) cb = a.KT * 8 - 1;      // beyond the last column: not stored
        csrc[i] = (const char *)a.turned + ((int64_t)cb * a.RT + rt0) * 1024 + lane * 16;
    }
    bool beyond = false;      // weights of this wave's columns, in the slice's rows, that half precision does not hold
    {
        const int own = kt + (wave >> 2);      // the tile of this wave's 32 columns
        int g = a.SUB > 1 ? own * a.SUB + (wave & 3) * a.SUB / 4 : own / a.tpg;
        if (g >= a.NG) g = a.NG - 1;
        ssrc = (const char *)(a.steps + 2 * g * len + rt0 * 128) + lane * 4;
        if (TYPE != OBC_F32)
            for (int i = 2 * rt0 + lane; i < 2 * rt1; i += 64) beyond |= a.wide[(int64_t)g * a.RT * 2 + i] != 0;
    }
    auto fetch = [&](int rt, uintx4 *lds) __attribute__((always_inline)) {
        const int64_t k = (rt < rt1 ? rt : rt1 - 1) - rt0;      // (behind the last: its tile again, for the count of loads)
#pragma unroll
        for (int i = 0; i < C::XL; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(xsrc[i] + k * 256), (lds_ptr)(lds + (i * C::WAVES + wave) * 64), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < C::CL; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(csrc[i] + k * 1024), (lds_ptr)(lds + C::XN + (i * C::WAVES + wave) * 64), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(ssrc + i * len * 2 + k * 256), (lds_ptr)(lds + C::XN + C::CN + wave * 32 + i * 16), 4, 0, 0);
    };
    floatx4 acc[MF][NF];
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[m][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    fetch(rt0, lds0);
    if (STAGES > 2) fetch(rt0 + 1, lds1);
    const bool wide = __any(beyond);
    __builtin_amdgcn_s_waitcnt(wait_loads(0));
    stage_barrier();
    auto turn = [&](auto flag, const int rt, const uintx4 *lds, uintx4 *lds_next) __attribute__((always_inline)) {
        fetch(rt + STAGES - 1, lds_next);
        uintx4 w[NF];
#pragma unroll
        for (int j = 0; j < NF; ++j) w[j] = lds[C::XN + (wave * NF + j) * 64 + lane];
        const uintx4 *const steps = lds + C::XN + C::CN + wave * 32;
        // fp32: a sum of its own for these 128 rows, added with an fp32 addition: the matrix cores' sums are not rounded to nearest, and
        // their error grows with the instructions on one sum (500 tokens through 4096 x 2048: 6.4e-7 off in one sum over all rows)
        floatx4 S[MF][NF];
        if constexpr (TYPE == OBC_F32)
#pragma unroll
            for (int m = 0; m < MF; ++m)
#pragma unroll
                for (int j = 0; j < NF; ++j) S[m][j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uintx4 step = steps[4 * k + quad], off = steps[16 + 4 * k + quad];
            uintx4 B[NF][TERMS];
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                if constexpr (TYPE == OBC_F32) weights_split(w[j][k], step, off, B[j]);
                else weights_f16<decltype(flag)::value>(w[j][k], step, off, B[j]);
            }
#pragma unroll
            for (int m = 0; m < MF; ++m) {
                const int t = m * 16 + n;
                if constexpr (TYPE == OBC_F32) {
                    uintx4 A[3];
#pragma unroll
                    for (int p = 0; p < 3; ++p) A[p] = lds[(p * BM + t) * 16 + ((4 * k + quad) ^ n)];
#pragma unroll
                    for (int o = 2; o >= 0; --o)
#pragma unroll
                        for (int p = 0; p <= o; ++p)
#pragma unroll
                            for (int j = 0; j < NF; ++j) S[m][j] = mfma_bf16(A[p], B[j][o - p], S[m][j]);
                } else {
                    const uintx4 A = lds[t * 16 + ((4 * k + quad) ^ n)];
#pragma unroll
                    for (int o = 1; o >= 0; --o)
#pragma unroll
                        for (int j = 0; j < NF; ++j) acc[m][j] = mfma_f16(A, B[j][o], acc[m][j]);
                }
            }
        }
        if constexpr (TYPE == OBC_F32)
#pragma unroll
            for (int m = 0; m < MF; ++m)
#pragma unroll
                for (int j = 0; j < NF; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][j][i] += S[m][j][i];
        __builtin_amdgcn_s_waitcnt(wait_loads(STAGES > 2 ? C::LOADS : 0));      // the next tile is in LDS
        stage_barrier();
    };
    auto all = [&](auto flag) __attribute__((always_inline)) {
        for (int rt = rt0;;) {
            turn(flag, rt, lds0, STAGES > 2 ? lds2 : lds1);
            if (++rt >= rt1) break;
            turn(flag, rt, lds1, lds0);
            if (++rt >= rt1) break;
            if (STAGES > 2) {
                turn(flag, rt, lds2, lds1);
                if (++rt >= rt1) break;
            }
        }
    };
    // (the waves of a workgroup may part here: either way they pass the same number of barriers)
    if (TYPE != OBC_F32 && wide) all(Flag<true>());
    else all(Flag<false>());
    // (loads behind the last tile still write to LDS: they are waited for before it can be another workgroup's)
    __builtin_amdgcn_s_waitcnt(wait_loads(0));
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + m * 16 + 4 * quad + i;
            if (t >= a.T) continue;
            const float back = (TYPE == OBC_BF16 ? a.back[t] : 1.f) * (wide ? 32.f : 1.f);
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                const int c = kt * 128 + (wave * NF + j) * 16 + n;
                if (c >= a.d) continue;
                const float v = acc[m][j][i] * back;
                if (a.slices > 1) a.part[((int64_t)slice * a.T + t) * a.d + c] = v;
                else store_as<TYPE>(a.dx, (int64_t)t * a.lddx + c, v);
            }
        }
}

template <int TYPE>
__global__ __launch_bounds__(256) void grad_add_kernel(Args a)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)a.T * a.d;
    if (i >= n) return;
    const float v = add_slices(a.part + i, n, a.slices);
    const int64_t t = i / a.d;
    store_as<TYPE>(a.dx, t * a.lddx + (i - t * a.d), v);
}

// ---- host ---------------------------------------------------------------------------------------------------------
struct Plan {
    int BM, BN, mtiles, ntiles, slices, per, RT;
    size_t rows, back, turned, steps, wide, part, bytes;
};

Plan plan_of(const pack4_layout &L, int T, int type)
{
    Plan p;
    p.RT = L.R / 128 + (L.R % 128 != 0);
    auto cut = [&](int BM, int BN) {
        p.BM = BM;
        p.BN = BN;
        p.mtiles = T / BM + (T % BM != 0);
        p.ntiles = BN == 256 ? (L.KT + 1) / 2 : L.KT;
        return (int64_t)p.mtiles * p.ntiles;
    };
    int64_t tiles = 0;
    // (fp32 in tiles of 32 and of 64: 77 tokens through 768 x 768 13.7 and 16.3 us, 96 through 700 x 3100 16.7 and 19.3, 77 through
    // 2304 x 1283 19.4 and 19.2, 96 through 4096 x 4096 48 and 40, 500 151 and 114)
    if (T <= 32 || (type == OBC_F32 && T <= 96)) tiles = cut(32, 128);
    else if (type == OBC_F32) tiles = cut(64, 128);
    // 128 x 256 for three quarters of the compute units and more (2048 x 4096 x 4096 in bf16: 121 us, in tiles of 64 x 128 145; 500 x 4096 x
    // 4096: 105 us and 53)
    else if (T <= 64 || (tiles = cut(128, 256)) < 192) tiles = cut(64, 128);
    // few tokens: slices of the rows, two workgroups to a compute unit (fp32, whose planes leave room for one: one), two row tiles
    // at least to a slice (77 x 2304 x 1283 in fp32: 19 us, with one slice 46; 64 x 4096 x 4096 in bf16: 24 and 48)
    int64_t s = p.BM < 128 && tiles > 0 ? (type == OBC_F32 ? 256 : 512) / tiles : 1;
    if (s > p.RT / 2) s = p.RT / 2;
    if (s < 1) s = 1;
    p.per = (int)((p.RT + s - 1) / s);
    p.slices = p.per > 0 ? (p.RT + p.per - 1) / p.per : 1;
    size_t at = 0;
    auto take = [&](size_t n) { const size_t b = at; at += obc_align_up(n, 256); return b; };
    p.rows = take((size_t)T * p.RT * 256 * (type == OBC_F32 ? 3 : 1));
    p.back = take((size_t)T * 4);
    p.turned = take((size_t)L.KT * 8 * p.RT * 1024);
    p.steps = take((size_t)L.NG * p.RT * 512);
    p.wide = take((size_t)L.NG * p.RT * 2);
    p.part = take(p.slices > 1 ? (size_t)p.slices * T * L.d * 4 : 0);
    p.bytes = at;
    return p;
}

template <int TYPE>
int launch(obc_ctx *ctx, Args a, const Plan &p)
{
    const int64_t turns = (int64_t)a.KT * a.RT, scale_blocks = ((int64_t)a.NG * a.RT * 128 + 255) / 256;
    const int64_t lay = turns + scale_blocks + a.T, tiles = (int64_t)p.mtiles * p.ntiles * p.slices, adds = ((int64_t)a.T * a.d + 255) / 256;
    if (!obc_grid_fits(lay, 256) || !obc_grid_fits(tiles, p.BN * 2) || (p.slices > 1 && !obc_grid_fits(adds, 256)))
        return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_product4_grad: too many tiles");
    grad_lay_kernel<TYPE><<<(unsigned)lay, 256, 0, ctx->stream>>>(a, turns, scale_blocks);
    OBC_LAUNCH_CHECK(ctx, "grad_lay_kernel");
    if (p.BM == 32) grad_tiles_kernel<TYPE, 32, 128><<<(unsigned)tiles, 256, 0, ctx->stream>>>(a, p.mtiles, p.ntiles);
    else if (p.BM == 64) grad_tiles_kernel<TYPE, 64, 128><<<(unsigned)tiles, 256, 0, ctx->stream>>>(a, p.mtiles, p.ntiles);
    else if constexpr (TYPE != OBC_F32) grad_tiles_kernel<TYPE, 128, 256><<<(unsigned)tiles, 512, 0, ctx->stream>>>(a, p.mtiles, p.ntiles);
    OBC_LAUNCH_CHECK(ctx, "grad_tiles_kernel");
    if (p.slices > 1) {
        grad_add_kernel<TYPE><<<(unsigned)adds, 256, 0, ctx->stream>>>(a);
        OBC_LAUNCH_CHECK(ctx, "grad_add_kernel");
    }
    return OBC_OK;
}

__global__ __launch_bounds__(256) void grad_zero_kernel(void *dx, int64_t lddx, int T, int d, int size)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)T * d) return;
    const int64_t at = i / d * lddx + i % d;
    if (size == 4) ((float *)dx)[at] = 0.f;
    else ((unsigned short *)dx)[at] = 0;
}

}  // namespace

extern "C" {

int obc_product4_grad_workspace_bytes(int T, int R, int d, int group, int type, size_t *bytes)
{
    pack4_layout L;
    if (!bytes || T < 0 || R < 0 || d <= 0 || !float_type(type) || !pack4_layout_of(R, d, group, &L)) return OBC_ERR_BAD_ARG;
    *bytes = T > 0 && R > 0 ? plan_of(L, T, type).bytes : 0;
    return OBC_OK;
}

int obc_product4_grad(obc_ctx *ctx, const void *packed, int R, int d, int group, const void *dy, int type, int T, int64_t lddy,
                      void *dx, int64_t lddx, void *ws, size_t ws_bytes)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (T < 0 || R < 0 || d <= 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4_grad: bad size");
    if (!float_type(type)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4_grad: type %d is not a floating type", type);
    pack4_layout L;
    if (!pack4_layout_of(R, d, group, &L))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4_grad: group (%d) is not 0, 32, 64 or a multiple of 128", group);
    if (lddy < R || lddx < d) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_product4_grad: leading dimension below the row's length");
    if (T == 0) return OBC_OK;
    if (!dx || (R > 0 && (!packed || !dy))) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4_grad: null argument");
    if (((uintptr_t)packed & 15) != 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4_grad: packed is not aligned to 16 bytes");
    if ((((uintptr_t)dy | (uintptr_t)dx) & (size_of_type(type) - 1)) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4_grad: dy or dx is not aligned to its elements");
    if (R == 0) {
        const int64_t blocks = ((int64_t)T * d + 255) / 256;
        if (!obc_grid_fits(blocks, 256)) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_product4_grad: too many tiles");
        grad_zero_kernel<<<(unsigned)blocks, 256, 0, ctx->stream>>>(dx, lddx, T, d, (int)size_of_type(type));
        OBC_LAUNCH_CHECK(ctx, "grad_zero_kernel");
        return OBC_OK;
    }
    const Plan p = plan_of(L, T, type);
    if (!ws || ((uintptr_t)ws & 15) != 0 || ws_bytes < p.bytes)
        return obc_fail(ctx, OBC_ERR_WORKSPACE, "obc_product4_grad: workspace of %zu bytes needed", p.bytes);
    Args a;
    a.codes = (const unsigned *)packed;
    a.scales = (const unsigned *)((const char *)packed + L.scales);
    a.dy = dy; a.dx = dx;
    a.T = T; a.R = R; a.d = d; a.RB = L.RB; a.KT = L.KT; a.NG = L.NG; a.SUB = L.SUB; a.tpg = L.tpg;
    a.RT = p.RT;
    a.lddy = lddy; a.lddx = lddx;
    char *w = (char *)ws;
    a.rows = (uint4 *)(w + p.rows);
    a.back = (float *)(w + p.back);
    a.turned = (unsigned *)(w + p.turned);
    a.steps = (unsigned short *)(w + p.steps);
    a.wide = (unsigned char *)(w + p.wide);
    a.part = (float *)(w + p.part);
    a.slices = p.slices; a.per = p.per;
    return type == OBC_F32 ? launch<OBC_F32>(ctx, a, p) : type == OBC_F16 ? launch<OBC_F16>(ctx, a, p) : launch<OBC_BF16>(ctx, a, p);
}

}  // extern "C"
