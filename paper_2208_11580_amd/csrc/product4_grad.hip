// obc_product4_grad: dx = dy W, the gradient of the inputs of a product with 4-bit weights.
//
//   dx[t, c] = sum_r dy[t, r] (offset + delta code)[r, c]
// The sum runs over the rows, whose steps differ, so the weights are formed before the product.  16-bit types: in half
// precision, whose packed instructions take two weights at a time and which rounds eight times finer than bf16; a
// token's bf16 gradients, scaled by a power of two so that the largest is near 2^14, are half-precision numbers too (what
// that loses lies 2^-39 below the largest).  fp32: weights and gradients as three bf16 terms each, six of the nine
// products (what is left out is below 2^-24).
//
// A first launch lays out the gradients as the matrix instructions' operands want them and turns the codes, so that the
// lanes lie along the columns and a dword holds eight rows: 1/60 of a large product's time.  The product then is like the
// forward one: gradients through LDS, codes straight from memory, weights formed in registers once for a wave's tokens.
// Few tokens leave too few tiles for the chip: the rows are cut into slices, whose sums a third launch adds in order.
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
    float *part;                // slices x T x d
    int slices, per;            // slices of the rows, row tiles of a slice
};

// ---- layout -------------------------------------------------------------------------------------------------------

// Workgroups below `turns`: 64 rows x 128 columns of codes, a thread an octet of rows x an octet of columns (and a group's
// steps along the way); the others: a token's gradients each.
template <int TYPE>
__global__ __launch_bounds__(256) void grad_lay_kernel(Args a, int64_t turns, int64_t scale_blocks)
{
    const int tid = threadIdx.x;
    if ((int64_t)blockIdx.x < turns) {
        // octets: 16 of columns (a tile's 4 dwords x 4 quads) x 16 of rows of one row tile
        const int kt = (int)((int64_t)blockIdx.x / a.RT), rt = (int)((int64_t)blockIdx.x % a.RT);
        const int co = tid & 15, ro = tid >> 4;      // column octet 4 s + quad, row octet 4 s + quad
        unsigned in[8], out[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = rt * 128 + ro * 8 + i;
            in[i] = row < a.RB * 16 ? a.codes[((int64_t)(row >> 4) * a.KT + kt) * 256 + ((co & 3) * 16 + (row & 15)) * 4 + (co >> 2)] : 0u;
        }
        // nibble of element e: (e >> 1) + 4 (e & 1)
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            unsigned w = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) w |= ((in[i] >> (4 * ((c >> 1) + 4 * (c & 1)))) & 15u) << (4 * ((i >> 1) + 4 * (i & 1)));
            out[c] = w;
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const int col = co * 8 + c;
            a.turned[((int64_t)(kt * 8 + (col >> 4)) * a.RT + rt) * 256 + ((ro & 3) * 16 + (col & 15)) * 4 + (ro >> 2)] = out[c];
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
        return;
    }
    const int64_t t = (int64_t)blockIdx.x - turns - scale_blocks;
    const int pieces = a.RT * 16;
    const int64_t at = t * a.lddy, plane = (int64_t)a.T * pieces;
    auto load = [&](int r, float (&v)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (TYPE == OBC_F32) v[j] = r + j < a.R ? ((const float *)a.dy)[at + r + j] : 0.f;
            else if (TYPE == OBC_F16) v[j] = r + j < a.R ? (float)((const _Float16 *)a.dy)[at + r + j] : 0.f;
            else v[j] = r + j < a.R ? (float)((const __bf16 *)a.dy)[at + r + j] : 0.f;
        }
    };
    float up = 1.f;
    if (TYPE == OBC_BF16) {
        __shared__ float tops[4];
        float top = 0.f;
        for (int p = tid; p < pieces; p += 256) {
            float v[8];
            load(p * 8, v);
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
        up = top > 0.f && top < __builtin_inff() ? ldexpf(1.f, e > -111 ? 15 - e : 126) : 1.f;
        if (tid == 0) a.back[t] = 1.f / up;
    }
    for (int p = tid; p < pieces; p += 256) {
        float v[8];
        load(p * 8, v);
        uint4 w[3];
        unsigned *u = (unsigned *)w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (TYPE == OBC_F32) {
                float h0, m0, l0, h1, m1, l1;
                split3(v[2 * j], h0, m0, l0);
                split3(v[2 * j + 1], h1, m1, l1);
                u[j] = pair_bf16(h0, h1);
                u[4 + j] = pair_bf16(m0, m1);
                u[8 + j] = pair_bf16(l0, l1);
            } else {
                u[j] = pair_f16(v[2 * j] * up, v[2 * j + 1] * up);
            }
        }
        a.rows[t * pieces + p] = w[0];
        if (TYPE == OBC_F32) {
            a.rows[plane + t * pieces + p] = w[1];
            a.rows[2 * plane + t * pieces + p] = w[2];
        }
    }
}

// ---- product ------------------------------------------------------------------------------------------------------
typedef __attribute__((address_space(1))) const void *global_ptr;
typedef __attribute__((address_space(3))) void *lds_ptr;
constexpr int kWaitVm0 = 0x0f70;      // s_waitcnt vmcnt(0)

// Eight weights of a lane's column, of the eight rows that `steps` and `offsets` (half precision) belong to.
__device__ inline uintx4 weights_f16(unsigned w, uintx4 steps, uintx4 offsets)
{
    const uintx4 c = codes_f16(w);
    const halfx2 base = {(_Float16)-16.f, (_Float16)-16.f};
    uintx4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        r[j] = bits_of(__builtin_elementwise_fma(half_pair(steps[j]), half_pair(c[j]) + base, half_pair(offsets[j])));
    return r;
}

__device__ inline void weights_split(unsigned w, uintx4 steps, uintx4 offsets, uintx4 (&r)[3])
{
    const uintx4 c = codes_bf16(w);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float lo = fmaf(half_lo(steps[j]), __builtin_bit_cast(float, c[j] << 16) - 16.f, half_lo(offsets[j]));
        const float hi = fmaf(half_hi(steps[j]), __builtin_bit_cast(float, c[j] & 0xffff0000u) - 16.f, half_hi(offsets[j]));
        float h0, m0, l0, h1, m1, l1;
        split3(lo, h0, m0, l0);
        split3(hi, h1, m1, l1);
        r[0][j] = pair_bf16(h0, h1);
        r[1][j] = pair_bf16(m0, m1);
        r[2][j] = pair_bf16(l0, l1);
    }
}

// BM tokens x 128 columns to a workgroup of WM x (4 / WM) waves.
template <int TYPE, int BM, int WM>
__global__ __launch_bounds__(256, 2) void grad_tiles_kernel(Args a, int mtiles, int ntiles)
{
    constexpr int P = TYPE == OBC_F32 ? 3 : 1, WN = 4 / WM, MF = BM / WM / 16, NF = 8 / WN;
    __shared__ uintx4 even[P * BM * 16], odd[P * BM * 16];
    __shared__ uintx4 even_steps[128], odd_steps[128];       // four groups of 128 rows: steps and offsets
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = lane & 15, quad = lane >> 4;
    const int wm = wave % WM, wn = wave / WM;
    const int tiles = mtiles * ntiles, slice = blockIdx.x / tiles, id = blockIdx.x % tiles;
    const int per = tiles >> 3, left = tiles & 7, die = id & 7;
    const int tile = die * per + (die < left ? die : left) + (id >> 3);
    const int t0 = (tile % mtiles) * BM, kt = tile / mtiles;
    const int rt0 = slice * a.per, rt1 = rt0 + a.per < a.RT ? rt0 + a.per : a.RT;
    const int64_t plane = (int64_t)a.T * a.RT * 256;       // bytes
    const int64_t len = (int64_t)a.RT * 128;
    floatx4 acc[MF][NF];
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[m][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    // piece o of token t at place o ^ (t mod 16) of its row, as in the forward product
    auto fetch = [&](int rt, uintx4 *lds, uintx4 *steps) {
#pragma unroll
        for (int i = 0; i < P * BM / 16; ++i) {
            const int first = (i * 4 + wave) * 4;
            const int p = P > 1 ? first / BM : 0, t = first - p * BM + (lane >> 4);
            const int row = t0 + t < a.T ? t0 + t : a.T - 1;
            const char *src = (const char *)a.rows + p * plane + ((int64_t)row * a.RT + rt) * 256 + ((lane & 15) ^ (t & 15)) * 16;
            __builtin_amdgcn_global_load_lds((global_ptr)src, (lds_ptr)(lds + first * 16), 16, 0, 0);
        }
        if (wave < 2) {
            int g = a.SUB > 1 ? kt * a.SUB + (2 * wave + (lane >> 5)) * a.SUB / 4 : kt / a.tpg;
            if (g >= a.NG) g = a.NG - 1;
            const char *src = (const char *)(a.steps + (2 * g + ((lane >> 4) & 1)) * len + rt * 128) + (lane & 15) * 16;
            __builtin_amdgcn_global_load_lds((global_ptr)src, (lds_ptr)(steps + wave * 64), 16, 0, 0);
        }
    };
    uintx4 codes[NF];
    auto fetch_codes = [&](int rt) {
#pragma unroll
        for (int j = 0; j < NF; ++j) codes[j] = *((const uintx4 *)a.turned + ((int64_t)(kt * 8 + wn * NF + j) * a.RT + rt) * 64 + lane);
    };
    fetch(rt0, even, even_steps);
    fetch_codes(rt0);
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __syncthreads();
    auto turn = [&](const int rt, const uintx4 *lds, const uintx4 *steps, uintx4 *lds_next, uintx4 *steps_next) __attribute__((always_inline)) {
        uintx4 w[NF];
#pragma unroll
        for (int j = 0; j < NF; ++j) w[j] = codes[j];
        const int ahead = rt + 1 < rt1 ? rt + 1 : rt;
        fetch(ahead, lds_next, steps_next);
        fetch_codes(ahead);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uintx4 B[P][NF];
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                const int u = (wn * NF + j) >> 1;      // which of the tile's quarters of 32 columns
                const uintx4 step = steps[u * 32 + 4 * k + quad], off = steps[u * 32 + 16 + 4 * k + quad];
                if constexpr (P == 3) {
                    uintx4 r[3];
                    weights_split(w[j][k], step, off, r);
#pragma unroll
                    for (int p = 0; p < 3; ++p) B[p][j] = r[p];
                } else {
                    B[0][j] = weights_f16(w[j][k], step, off);
                }
            }
#pragma unroll
            for (int m = 0; m < MF; ++m) {
                const int t = (wm * MF + m) * 16 + n;
                if constexpr (P == 3) {
                    uintx4 A[3];
#pragma unroll
                    for (int p = 0; p < 3; ++p) A[p] = lds[(p * BM + t) * 16 + ((4 * k + quad) ^ n)];
#pragma unroll
                    for (int o = 2; o >= 0; --o)
#pragma unroll
                        for (int p = 0; p <= o; ++p)
#pragma unroll
                            for (int j = 0; j < NF; ++j) acc[m][j] = mfma_bf16(A[p], B[o - p][j], acc[m][j]);
                } else {
                    const uintx4 A = lds[t * 16 + ((4 * k + quad) ^ n)];
#pragma unroll
                    for (int j = 0; j < NF; ++j) acc[m][j] = mfma_f16(A, B[0][j], acc[m][j]);
                }
            }
        }
        __builtin_amdgcn_s_waitcnt(kWaitVm0);
        __syncthreads();
    };
    for (int rt = rt0;; rt += 2) {
        turn(rt, even, even_steps, odd, odd_steps);
        if (rt + 1 >= rt1) break;
        turn(rt + 1, odd, odd_steps, even, even_steps);
        if (rt + 2 >= rt1) break;
    }
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + (wm * MF + m) * 16 + 4 * quad + i;
            if (t >= a.T) continue;
            const float back = TYPE == OBC_BF16 ? a.back[t] : 1.f;
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                const int c = kt * 128 + (wn * NF + j) * 16 + n;
                if (c >= a.d) continue;
                const float v = TYPE == OBC_BF16 ? acc[m][j][i] * back : acc[m][j][i];
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
    float v = a.part[i];
    for (int s = 1; s < a.slices; ++s) v += a.part[s * n + i];
    const int64_t t = i / a.d;
    store_as<TYPE>(a.dx, t * a.lddx + (i - t * a.d), v);
}

// ---- host ---------------------------------------------------------------------------------------------------------
struct Plan {
    int BM, mtiles, slices, per, RT;
    size_t rows, back, turned, steps, part, bytes;
};

Plan plan_of(const pack4_layout &L, int T, int type)
{
    Plan p;
    p.RT = L.R / 128 + (L.R % 128 != 0);
    p.BM = T <= 32 ? 32 : type == OBC_F32 ? 64 : 128;
    p.mtiles = T / p.BM + (T % p.BM != 0);
    // two workgroups to a compute unit, two row tiles at least to a slice
    const int64_t tiles = (int64_t)p.mtiles * L.KT;
    int64_t s = tiles > 0 ? 512 / tiles : 1;
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
    p.part = take(p.slices > 1 ? (size_t)p.slices * T * L.d * 4 : 0);
    p.bytes = at;
    return p;
}

template <int TYPE>
int launch(obc_ctx *ctx, Args a, const Plan &p)
{
    const int64_t turns = (int64_t)a.KT * a.RT, scale_blocks = ((int64_t)a.NG * a.RT * 128 + 255) / 256;
    const int64_t lay = turns + scale_blocks + a.T, tiles = (int64_t)p.mtiles * a.KT * p.slices, adds = ((int64_t)a.T * a.d + 255) / 256;
    if (lay > 0x7fffffff || tiles > 0x7fffffff || (p.slices > 1 && adds > 0x7fffffff))
        return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_product4_grad: too many tiles");
    grad_lay_kernel<TYPE><<<(unsigned)lay, 256, 0, ctx->stream>>>(a, turns, scale_blocks);
    OBC_LAUNCH_CHECK(ctx, "grad_lay_kernel");
    if (p.BM == 32) grad_tiles_kernel<TYPE, 32, 1><<<(unsigned)tiles, 256, 0, ctx->stream>>>(a, p.mtiles, a.KT);
    else grad_tiles_kernel<TYPE, TYPE == OBC_F32 ? 64 : 128, 2><<<(unsigned)tiles, 256, 0, ctx->stream>>>(a, p.mtiles, a.KT);
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
        if (blocks > 0x7fffffff) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_product4_grad: too many tiles");
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
    a.part = (float *)(w + p.part);
    a.slices = p.slices; a.per = p.per;
    return type == OBC_F32 ? launch<OBC_F32>(ctx, a, p) : type == OBC_F16 ? launch<OBC_F16>(ctx, a, p) : launch<OBC_BF16>(ctx, a, p);
}

}  // extern "C"
