// obc_product4: y = x W^T with W in 4-bit codes and a step and an offset per row and group of columns.
//
//   y[t, r] = sum_g ( delta[r, g] S - (16 delta[r, g] - offset[r, g]) s ),   S = sum_{c in g} x[t, c] (16 + code[r, c]),
//                                                                           s = sum_{c in g} x[t, c]
// The codes enter the matrix instructions as the 16-bit numbers 16 + code, exactly (8-bit inputs: as bytes, without
// the 16), so their products with 16-bit inputs are exact in fp32 and the only roundings are those of the fp32 sums; a
// group's sums start from zero and are scaled when it ends.  fp32 inputs go in as three bf16 terms.  s comes from one
// more instruction, against ones, in the very lanes that need it.
#include "product4.h"

namespace {

struct Args {
    const uintx4 *codes;
    const unsigned *scales;
    const void *x;
    const float *xs;
    void *y;
    int T, R, d, RB, KT, NG, tpg;
    int64_t ldx, ldy;
};

// One 16x16x32 operand of token rows: the lane's eight columns from `c` on of row `row`, zeros from d on.
template <int XT>
struct Operand;

template <>
struct Operand<OBC_BF16> {
    uintx4 v;
    __device__ void load(const void *x, int64_t at, int left)
    {
        const unsigned short *p = (const unsigned short *)x + at;
        if (left >= 8) {
            v = *(const uintx4_at2 *)p;
        } else {
            unsigned short e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = j < left ? p[j] : (unsigned short)0;
            v = uintx4{e[0] | (unsigned)e[1] << 16, e[2] | (unsigned)e[3] << 16, e[4] | (unsigned)e[5] << 16, e[6] | (unsigned)e[7] << 16};
        }
    }
};

template <>
struct Operand<OBC_F16> : Operand<OBC_BF16> {
};

template <>
struct Operand<OBC_F32> {
    uintx4 v[3];
    __device__ void load(const void *x, int64_t at, int left)
    {
        const float *p = (const float *)x + at;
        float e[8];
        if (left >= 8) {
            const floatx4 a = *(const floatx4_at4 *)p, b = *(const floatx4_at4 *)(p + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) { e[j] = a[j]; e[4 + j] = b[j]; }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = j < left ? p[j] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float h0, m0, l0, h1, m1, l1;
            split3(e[2 * j], h0, m0, l0);
            split3(e[2 * j + 1], h1, m1, l1);
            v[0][j] = pair_bf16(h0, h1);
            v[1][j] = pair_bf16(m0, m1);
            v[2][j] = pair_bf16(l0, l1);
        }
    }
};

template <>
struct Operand<OBC_I8> {
    uintx2 v;
    __device__ void load(const void *x, int64_t at, int left)
    {
        const uint8_t *p = (const uint8_t *)x + at;
        uintx2 r;
        if (left >= 8) {
            r = *(const uintx2_at1 *)p;
        } else {
            unsigned e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = j < left ? p[j] : 0u;
            r = uintx2{e[0] | e[1] << 8 | e[2] << 16 | e[3] << 24, e[4] | e[5] << 8 | e[6] << 16 | e[7] << 24};
        }
        v = bytes_like_codes(r);
    }
};

// Codes of one instruction and ones, as the operand that meets XT's.
template <int XT>
struct Codes {
    uintx4 v;
    __device__ explicit Codes(unsigned w) : v(XT == OBC_F16 ? codes_f16(w) : codes_bf16(w)) {}
    static __device__ Codes ones()
    {
        Codes c(0);
        const unsigned one = XT == OBC_F16 ? 0x3c003c00u : 0x3f803f80u;
        c.v = uintx4{one, one, one, one};
        return c;
    }
};

template <>
struct Codes<OBC_I8> {
    uintx2 v;
    __device__ explicit Codes(unsigned w) : v(codes_i8(w)) {}
    static __device__ Codes ones()
    {
        Codes c(0);
        c.v = uintx2{0x01010101u, 0x01010101u};
        return c;
    }
};

template <int XT>
struct Sum {
    floatx4 s = {0.f, 0.f, 0.f, 0.f};
    __device__ void add(const Operand<XT> &a, const Codes<XT> &b)
    {
        if constexpr (XT == OBC_F32) {
            s = mfma_bf16(a.v[2], b.v, s);
            s = mfma_bf16(a.v[1], b.v, s);
            s = mfma_bf16(a.v[0], b.v, s);
        } else if constexpr (XT == OBC_F16) {
            s = mfma_f16(a.v, b.v, s);
        } else {
            s = mfma_bf16(a.v, b.v, s);
        }
    }
    __device__ float operator[](int i) const { return s[i]; }
};

template <>
struct Sum<OBC_I8> {
    intx4 s = {0, 0, 0, 0};
    __device__ void add(const Operand<OBC_I8> &a, const Codes<OBC_I8> &b) { s = mfma_i8(a.v, b.v, s); }
    __device__ float operator[](int i) const { return (float)s[i]; }
};

// 16 rows of W and 16 MF tokens to a workgroup whose WAVES waves take turns along the columns' tiles and sum in LDS.
template <int XT, int SUB, int MF, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void product4_rows_kernel(Args a, int y_type)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = lane & 15, quad = lane >> 4;
    const int rb = blockIdx.x;
    const int t0 = blockIdx.y * 16 * MF;
    int64_t row_at[MF];
#pragma unroll
    for (int m = 0; m < MF; ++m) {
        const int t = t0 + 16 * m + n;
        row_at[m] = (int64_t)(t < a.T ? t : a.T - 1) * a.ldx;      // rows beyond the last: their sums are not stored
    }
    float acc[MF][4];
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][i] = 0.f;
    constexpr float base = XT == OBC_I8 ? 0.f : kCodeBase;
    const Codes<XT> ones = Codes<XT>::ones();
    for (int kt = wave; kt < a.KT; kt += WAVES) {
        const uintx4 w = a.codes[((int64_t)rb * a.KT + kt) * 64 + lane];
        unsigned sc[SUB];
#pragma unroll
        for (int u = 0; u < SUB; ++u)
            sc[u] = SUB > 1 ? a.scales[(((int64_t)rb * a.KT + kt) * 16 + n) * SUB + u]
                            : a.scales[((int64_t)rb * a.NG + kt / a.tpg) * 16 + n];
#pragma unroll
        for (int m = 0; m < MF; ++m) {
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                Sum<XT> S, s;
#pragma unroll
                for (int k = u * 4 / SUB; k < (u + 1) * 4 / SUB; ++k) {
                    Operand<XT> x;
                    const int c = kt * 128 + 32 * k + 8 * quad;
                    x.load(a.x, row_at[m] + c, a.d - c);
                    S.add(x, Codes<XT>(w[k]));
                    s.add(x, ones);
                }
                const float step = half_lo(sc[u]), off = half_hi(sc[u]) - base * step;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][i] = fmaf(step, S[i], fmaf(off, s[i], acc[m][i]));
            }
        }
    }
    __shared__ float part[WAVES][MF][64][4];
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[wave][m][lane][i] = acc[m][i];
    __syncthreads();
    for (int e = threadIdx.x; e < MF * 256; e += WAVES * 64) {
        const int m = e >> 8, i = (e >> 6) & 3, l = e & 63;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += part[w][m][l][i];
        const int t = t0 + 16 * m + 4 * (l >> 4) + i, r = rb * 16 + (l & 15);
        if (t >= a.T || r >= a.R) continue;
        if (XT == OBC_I8) v *= a.xs[t];
        const int64_t at = (int64_t)t * a.ldy + r;
        if (y_type == OBC_F32) store_as<OBC_F32>(a.y, at, v);
        else if (y_type == OBC_F16) store_as<OBC_F16>(a.y, at, v);
        else store_as<OBC_BF16>(a.y, at, v);
    }
}

template <int XT, int SUB>
int launch(obc_ctx *ctx, const Args &a, int y_type)
{
    if (a.T <= 16) {
        product4_rows_kernel<XT, SUB, 1, 8><<<dim3(a.RB, 1), 512, 0, ctx->stream>>>(a, y_type);
    } else {
        const int per = 64, blocks = (a.T + per - 1) / per;
        for (int b0 = 0; b0 < blocks; b0 += 65535) {
            Args c = a;
            const int64_t t0 = (int64_t)b0 * per;
            c.x = (const char *)a.x + t0 * a.ldx * (int64_t)size_of_type(XT);
            c.y = (char *)a.y + t0 * a.ldy * (int64_t)size_of_type(y_type);
            if (a.xs) c.xs = a.xs + t0;
            c.T = a.T - (int)t0;
            const int nb = blocks - b0 < 65535 ? blocks - b0 : 65535;
            product4_rows_kernel<XT, SUB, 4, 4><<<dim3(a.RB, nb), 256, 0, ctx->stream>>>(c, y_type);
        }
    }
    OBC_LAUNCH_CHECK(ctx, "product4_rows_kernel");
    return OBC_OK;
}

template <int XT>
int launch_sub(obc_ctx *ctx, const Args &a, int sub, int y_type)
{
    return sub == 1 ? launch<XT, 1>(ctx, a, y_type) : sub == 2 ? launch<XT, 2>(ctx, a, y_type) : launch<XT, 4>(ctx, a, y_type);
}

}  // namespace

extern "C" {

int obc_product4_workspace_bytes(int T, int R, int d, int group, int x_type, size_t *bytes)
{
    pack4_layout L;
    if (!bytes || T < 0 || R < 0 || d <= 0 || !(float_type(x_type) || x_type == OBC_I8) || !pack4_layout_of(R, d, group, &L))
        return OBC_ERR_BAD_ARG;
    *bytes = 0;
    return OBC_OK;
}

int obc_product4(obc_ctx *ctx, const void *packed, int R, int d, int group, const void *x, int x_type, const float *x_scale,
                 int T, int64_t ldx, void *y, int y_type, int64_t ldy, void *ws, size_t ws_bytes)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (T < 0 || R < 0 || d <= 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: bad size");
    if (!float_type(x_type) && x_type != OBC_I8) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: unknown x_type %d", x_type);
    if (!float_type(y_type)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: y_type %d is not a floating type", y_type);
    pack4_layout L;
    if (!pack4_layout_of(R, d, group, &L))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: group (%d) is not 0, 32, 64 or a multiple of 128", group);
    if (ldx < d || ldy < R) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_product4: leading dimension below the row's length");
    if (T == 0 || R == 0) return OBC_OK;
    if (!packed || !x || !y) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: null argument");
    if ((x_type == OBC_I8) != (x_scale != nullptr))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: x_scale goes with 8-bit inputs");
    if (((uintptr_t)packed & 15) != 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: packed is not aligned to 16 bytes");
    if (((uintptr_t)x & (size_of_type(x_type) - 1)) != 0 || ((uintptr_t)y & (size_of_type(y_type) - 1)) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: x or y is not aligned to its elements");
    (void)ws;
    (void)ws_bytes;
    Args a;
    a.codes = (const uintx4 *)packed;
    a.scales = (const unsigned *)((const char *)packed + L.scales);
    a.x = x; a.xs = x_scale; a.y = y;
    a.T = T; a.R = R; a.d = d; a.RB = L.RB; a.KT = L.KT; a.NG = L.NG; a.tpg = L.tpg;
    a.ldx = ldx; a.ldy = ldy;
    switch (x_type) {
    case OBC_F32: return launch_sub<OBC_F32>(ctx, a, L.SUB, y_type);
    case OBC_F16: return launch_sub<OBC_F16>(ctx, a, L.SUB, y_type);
    case OBC_BF16: return launch_sub<OBC_BF16>(ctx, a, L.SUB, y_type);
    default: return launch_sub<OBC_I8>(ctx, a, L.SUB, y_type);
    }
}

}  // extern "C"
