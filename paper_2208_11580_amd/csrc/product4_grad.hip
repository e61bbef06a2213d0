// obc_product4_grad: dx = dy W, the gradient of the inputs of a product with 4-bit weights.
//
//   dx[t, c] = sum_r dy[t, r] (offset + delta code)[r, c]
// The sum runs over the rows, whose steps differ, so the weights are formed before the product: in fp32, then
// rounded to dy's 16-bit type, or split into three bf16 terms for fp32 (six of the nine products of terms; what is left
// out is below 2^-24).  A packed tile has the rows along its lanes; it is turned in LDS.
#include "product4.h"

namespace {

struct Args {
    const uintx4 *codes;
    const unsigned *scales;
    const void *dy;
    void *dx;
    int T, R, d, RB, KT, NG, tpg;
    int64_t lddy, lddx;
};

constexpr int TM = 64;          // tokens of a workgroup
constexpr int LD = 32 + 8;      // LDS stride of 32 rows, in 16-bit elements

template <int TYPE>
__device__ inline unsigned short round16(float v)
{
    return TYPE == OBC_F16 ? __builtin_bit_cast(unsigned short, (_Float16)v) : __builtin_bit_cast(unsigned short, (__bf16)v);
}

// TM tokens x 128 columns to a workgroup of four waves, 32 columns each; 32 rows of W at a time.
template <int TYPE, int SUB>
__global__ __launch_bounds__(256) void product4_grad_kernel(Args a)
{
    constexpr int P = TYPE == OBC_F32 ? 3 : 1;
    __shared__ __align__(16) unsigned short As[P][TM][LD], Bs[P][128][LD];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = lane & 15, quad = lane >> 4;
    const int kt = blockIdx.x;
    const int t0 = blockIdx.y * TM;
    floatx4 acc[TM / 16][2];
#pragma unroll
    for (int m = 0; m < TM / 16; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[m][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < a.RB * 16; r0 += 32) {
        // weights: dword s of lane l of the two tiles
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int rb = r0 / 16 + u, l = tid >> 2, s = tid & 3;
            unsigned w = 0, sc = 0;
            if (rb < a.RB) {
                w = ((const unsigned *)a.codes)[((int64_t)rb * a.KT + kt) * 256 + tid];
                sc = SUB > 1 ? a.scales[(((int64_t)rb * a.KT + kt) * 16 + (l & 15)) * SUB + s * SUB / 4]
                             : a.scales[((int64_t)rb * a.NG + kt / a.tpg) * 16 + (l & 15)];
            }
            const float step = half_lo(sc), off = half_hi(sc);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = fmaf(step, (float)((w >> (4 * ((j >> 1) + 4 * (j & 1)))) & 15u), off);
                const int c = 32 * s + 8 * (l >> 4) + j, r = 16 * u + (l & 15);
                if (P == 3) {
                    float h, m, e;
                    split3(v, h, m, e);
                    Bs[0][c][r] = round16<OBC_BF16>(h);
                    Bs[P > 1 ? 1 : 0][c][r] = round16<OBC_BF16>(m);
                    Bs[P > 2 ? 2 : 0][c][r] = round16<OBC_BF16>(e);
                } else {
                    Bs[0][c][r] = round16<TYPE>(v);
                }
            }
        }
        // dy: zeros beyond the last token and the last row
        for (int e = tid; e < TM * 32; e += 256) {
            const int t = e >> 5, r = e & 31;
            const bool in = t0 + t < a.T && r0 + r < a.R;
            const int64_t at = (int64_t)(t0 + t) * a.lddy + r0 + r;
            if (P == 3) {
                float h, m, l;
                split3(in ? ((const float *)a.dy)[at] : 0.f, h, m, l);
                As[0][t][r] = round16<OBC_BF16>(h);
                As[P > 1 ? 1 : 0][t][r] = round16<OBC_BF16>(m);
                As[P > 2 ? 2 : 0][t][r] = round16<OBC_BF16>(l);
            } else {
                As[0][t][r] = in ? ((const unsigned short *)a.dy)[at] : (unsigned short)0;
            }
        }
        __syncthreads();
        uintx4 B[P][2];
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < 2; ++j) B[p][j] = *(const uintx4 *)&Bs[p][32 * wave + 16 * j + n][8 * quad];
#pragma unroll
        for (int m = 0; m < TM / 16; ++m) {
            uintx4 A[P];
#pragma unroll
            for (int p = 0; p < P; ++p) A[p] = *(const uintx4 *)&As[p][16 * m + n][8 * quad];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (P == 3) {
#pragma unroll
                    for (int o = 2; o >= 0; --o)
#pragma unroll
                        for (int p = 0; p <= o; ++p) acc[m][j] = mfma_bf16(A[p < P ? p : 0], B[o - p < P ? o - p : 0][j], acc[m][j]);
                } else {
                    acc[m][j] = TYPE == OBC_F16 ? mfma_f16(A[0], B[0][j], acc[m][j]) : mfma_bf16(A[0], B[0][j], acc[m][j]);
                }
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int m = 0; m < TM / 16; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = t0 + 16 * m + 4 * quad + i, c = kt * 128 + 32 * wave + 16 * j + n;
                if (t < a.T && c < a.d) store_as<TYPE>(a.dx, (int64_t)t * a.lddx + c, acc[m][j][i]);
            }
}

template <int TYPE>
int launch(obc_ctx *ctx, const Args &a, int sub)
{
    const int blocks = a.T / TM + (a.T % TM != 0);
    for (int b0 = 0; b0 < blocks; b0 += 65535) {
        Args c = a;
        const int64_t t0 = (int64_t)b0 * TM;
        c.dy = (const char *)a.dy + t0 * a.lddy * (int64_t)size_of_type(TYPE);
        c.dx = (char *)a.dx + t0 * a.lddx * (int64_t)size_of_type(TYPE);
        c.T = a.T - (int)t0;
        const dim3 grid(a.KT, blocks - b0 < 65535 ? blocks - b0 : 65535);
        if (sub == 1) product4_grad_kernel<TYPE, 1><<<grid, 256, 0, ctx->stream>>>(c);
        else if (sub == 2) product4_grad_kernel<TYPE, 2><<<grid, 256, 0, ctx->stream>>>(c);
        else product4_grad_kernel<TYPE, 4><<<grid, 256, 0, ctx->stream>>>(c);
        OBC_LAUNCH_CHECK(ctx, "product4_grad_kernel");
    }
    return OBC_OK;
}

}  // namespace

extern "C" {

int obc_product4_grad_workspace_bytes(int T, int R, int d, int group, int type, size_t *bytes)
{
    pack4_layout L;
    if (!bytes || T < 0 || R < 0 || d <= 0 || !float_type(type) || !pack4_layout_of(R, d, group, &L)) return OBC_ERR_BAD_ARG;
    *bytes = 0;
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
    (void)ws;
    (void)ws_bytes;
    Args a;
    a.codes = (const uintx4 *)packed;
    a.scales = (const unsigned *)((const char *)packed + L.scales);
    a.dy = dy; a.dx = dx;
    a.T = T; a.R = R; a.d = d; a.RB = L.RB; a.KT = L.KT; a.NG = L.NG; a.tpg = L.tpg;
    a.lddy = lddy; a.lddx = lddx;
    return type == OBC_F32 ? launch<OBC_F32>(ctx, a, L.SUB) : type == OBC_F16 ? launch<OBC_F16>(ctx, a, L.SUB) : launch<OBC_BF16>(ctx, a, L.SUB);
}

}  // extern "C"
