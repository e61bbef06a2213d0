// obc_rmsnorm and obc_rmsnorm_grad: root-mean-square norm with the residual's addition, an output in 8 bits, and
// the backward pass.  A row is read once and kept in registers between the reduction and the output; the largest
// |y| that 8 bits need comes out of the same reduction as the squares (max|h gain| times rstd).
//
// Memory-bound: 4096 x 8192 in bf16 with residual and sum, 268 MB, takes 54 us (4.9 TB/s; a large copy reaches 5.2), one row of 4096
// 2.7 us.  The backward pass keeps each workgroup's share of the gain's gradient in registers over its rows and has the next row's loads
// under way: 4096 x 4096 in bf16 with the residual's gradient, 134 MB, takes 33 us, 27 of them the rows (5.0 TB/s), the rest the sum of the shares.
#include "row_io.h"

namespace {

constexpr int kMaxCols = 65536;

// Sum (and largest magnitude) over a workgroup, the same value in every thread.
template <int NT, bool MAX>
__device__ inline void reduce(float &sum, float &top, float (*buf)[2])
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        sum += __shfl_xor(sum, off, 64);
        if (MAX) top = larger(top, __shfl_xor(top, off, 64));
    }
    if (NT == 64) return;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
        buf[wave][0] = sum;
        if (MAX) buf[wave][1] = top;
    }
    __syncthreads();
    sum = buf[0][0];
    if (MAX) top = buf[0][1];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) {
        sum += buf[w][0];
        if (MAX) top = larger(top, buf[w][1]);
    }
}

struct NormArgs {
    const void *x, *residual;
    const float *gain;
    void *h, *y;
    float *y_scale, *rstd;
    float eps;
    int T, d;
};

template <int TYPE, bool Q8, int NT, int CH>
__global__ __launch_bounds__(NT) void rmsnorm_kernel(NormArgs a)
{
    __shared__ float buf[NT / 64][2];
    const int64_t row = blockIdx.x, base = row * a.d;
    float v[CH][8];
    float sum = 0.f, top = 0.f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * NT + (int)threadIdx.x) * 8, left = a.d - c;
        if (left <= 0) continue;
        load8<TYPE>(a.x, base + c, left, v[k]);
        if (a.residual) {
            float r[8];
            load8<TYPE>(a.residual, base + c, left, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] += r[j];
        }
        if (a.h) store8<TYPE>(a.h, base + c, left, v[k]);
        float g[8];
        load8<OBC_F32>(a.gain, c, left, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum = fmaf(v[k][j], v[k][j], sum);
            v[k][j] *= g[j];
            if (Q8) top = larger(top, v[k][j]);
        }
    }
    reduce<NT, Q8>(sum, top, buf);
    const float rstd = 1.f / sqrtf(sum / (float)a.d + a.eps);
    if (threadIdx.x == 0 && a.rstd) a.rstd[row] = rstd;
    float mul = rstd;
    bool lost = false;
    if (Q8) {
        // codes are h gain / max|h gain| * 127: rstd cancels.  A row whose largest value is next to nothing is
        // scaled up first, so that its reciprocal stays finite.
        lost = !(sum < __builtin_inff()) || !(top < __builtin_inff());
        const float up = top < 1e-30f ? 0x1p90f : 1.f;
        mul = top > 0.f ? 127.f / (top * up) : 0.f;
        if (threadIdx.x == 0) a.y_scale[row] = lost ? __builtin_nanf("") : top > 0.f ? top * rstd / 127.f : 1.f;
#pragma unroll
        for (int k = 0; k < CH; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] *= up;
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * NT + (int)threadIdx.x) * 8, left = a.d - c;
        if (left <= 0) continue;
        if (Q8) {
            unsigned w[2] = {0u, 0u};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float q = fminf(fmaxf(rintf(v[k][j] * mul), -127.f), 127.f);
                w[j >> 2] |= lost ? 0u : ((unsigned)(int)q & 0xffu) << (8 * (j & 3));
            }
            uint8_t *p = (uint8_t *)a.y + base + c;
            if (left >= 8) *(uintx2_at1 *)p = uintx2{w[0], w[1]};
            else
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < left) p[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] *= mul;
            store8<TYPE>(a.y, base + c, left, v[k]);
        }
    }
}

struct GradArgs {
    const void *h, *dy, *dh;
    const float *gain, *rstd;
    void *dx;
    float *part;
    int T, d;
};

// Workgroup b takes the rows b, b + gridDim.x, ... and keeps its columns' share of dgain in registers; the next row's
// loads are on their way while it reduces this one.
template <int TYPE, int NT, int CH>
__global__ __launch_bounds__(NT) void rmsnorm_grad_kernel(GradArgs a)
{
    __shared__ float buf[2][NT / 64][2];
    float dg[CH][8], gain[CH][8];
    Eight<TYPE> h[CH], dy[CH];
    const int tid = threadIdx.x;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * NT + tid) * 8, left = a.d - c;
#pragma unroll
        for (int j = 0; j < 8; ++j) dg[k][j] = gain[k][j] = 0.f;
        if (left <= 0) continue;
        load8<OBC_F32>(a.gain, c, left, gain[k]);
        h[k].load(a.h, (int64_t)blockIdx.x * a.d + c, left);
        dy[k].load(a.dy, (int64_t)blockIdx.x * a.d + c, left);
    }
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x, turn ^= 1) {
        const int64_t base = row * a.d, next = row + gridDim.x < a.T ? base + (int64_t)gridDim.x * a.d : base;
        const float rstd = a.rstd[row];
        Eight<TYPE> dh[CH];
        float x[CH][8], g[CH][8];
        float sum = 0.f, none = 0.f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * NT + tid) * 8, left = a.d - c;
            if (left <= 0) continue;
            h[k].get(x[k]);
            dy[k].get(g[k]);
            if (a.dh) dh[k].load(a.dh, base + c, left);
            h[k].load(a.h, next + c, left);
            dy[k].load(a.dy, next + c, left);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[k][j] *= rstd;
                dg[k][j] = fmaf(g[k][j], x[k][j], dg[k][j]);
                g[k][j] *= gain[k][j];
                sum = fmaf(g[k][j], x[k][j], sum);
            }
        }
        reduce<NT, false>(sum, none, buf[turn]);
        const float mean = sum / (float)a.d;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * NT + tid) * 8, left = a.d - c;
            if (left <= 0) continue;
            float r[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) r[j] = 0.f;
            if (a.dh) dh[k].get(r);
#pragma unroll
            for (int j = 0; j < 8; ++j) r[j] = fmaf(rstd, fmaf(-x[k][j], mean, g[k][j]), r[j]);
            store8<TYPE>(a.dx, base + c, left, r);
        }
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * NT + tid) * 8, left = a.d - c;
        if (left > 0) store8<OBC_F32>(a.part, (int64_t)blockIdx.x * a.d + c, left, dg[k]);
    }
}

// Rows too wide for registers beside their share of dgain: read a second time, from the caches (rows that fit take 92 us this way
// against 70, 2048 x 16384 in bf16).
template <int TYPE>
__global__ __launch_bounds__(1024) void rmsnorm_grad_wide_kernel(GradArgs a)
{
    constexpr int NT = 1024, CH = kMaxCols / (NT * 8);
    __shared__ float buf[2][NT / 64][2];
    float dg[CH][8];
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) dg[k][j] = 0.f;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x, turn ^= 1) {
        const int64_t base = row * a.d;
        const float rstd = a.rstd[row];
        float sum = 0.f, none = 0.f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * NT + (int)threadIdx.x) * 8, left = a.d - c;
            if (left <= 0) continue;
            float x[8], g[8], w[8];
            load8<TYPE>(a.h, base + c, left, x);
            load8<TYPE>(a.dy, base + c, left, g);
            load8<OBC_F32>(a.gain, c, left, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float t = g[j] * (x[j] * rstd);
                dg[k][j] += t;
                sum = fmaf(w[j], t, sum);
            }
        }
        reduce<NT, false>(sum, none, buf[turn]);
        const float mean = sum / (float)a.d;
        for (int c = threadIdx.x * 8; c < a.d; c += NT * 8) {
            const int left = a.d - c;
            float x[8], g[8], w[8], r[8];
            load8<TYPE>(a.h, base + c, left, x);
            load8<TYPE>(a.dy, base + c, left, g);
            load8<OBC_F32>(a.gain, c, left, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) r[j] = 0.f;
            if (a.dh) load8<TYPE>(a.dh, base + c, left, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) r[j] = fmaf(rstd, fmaf(-x[j] * rstd, mean, g[j] * w[j]), r[j]);
            store8<TYPE>(a.dx, base + c, left, r);
        }
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * NT + (int)threadIdx.x) * 8, left = a.d - c;
        if (left > 0) store8<OBC_F32>(a.part, (int64_t)blockIdx.x * a.d + c, left, dg[k]);
    }
}

// dgain[c] = sum of the workgroups' shares, in a fixed order; 64 columns to a workgroup of 16 waves
__global__ __launch_bounds__(1024) void rmsnorm_dgain_kernel(const float *__restrict__ part, int parts, int d,
                                                             float *__restrict__ dgain)
{
    __shared__ float buf[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c < d) {
        int p = wave;
        for (; p + 7 * 16 < parts; p += 8 * 16)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += part[(int64_t)(p + i * 16) * d + c];
        for (; p < parts; p += 16) s[0] += part[(int64_t)p * d + c];
    }
    buf[wave][lane] = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
    __syncthreads();
    if (wave == 0 && c < d) {
        float v = buf[0][lane];
#pragma unroll
        for (int w = 1; w < 16; ++w) v += buf[w][lane];
        dgain[c] = v;
    }
}

inline int grad_parts(int T) { return T < 512 ? T : 512; }

template <int TYPE, bool Q8>
void launch_norm(obc_ctx *ctx, const NormArgs &a)
{
    // few rows: as many threads to a row as it has pieces, for the sooner end of each (bf16, captured in a graph: 1 x 4096 in
    // 2.7 us against 3.25, 300 x 8192 in 6.05 against 7.3; from 1000 rows on the fewer threads win: 1000 x 8192 in 12.2 against 13.8)
    const bool few = a.T <= 512;
    if (a.d <= 2048) rmsnorm_kernel<TYPE, Q8, 256, 1><<<a.T, 256, 0, ctx->stream>>>(a);
    else if (a.d <= 4096 && few) rmsnorm_kernel<TYPE, Q8, 512, 1><<<a.T, 512, 0, ctx->stream>>>(a);
    else if (a.d <= 4096) rmsnorm_kernel<TYPE, Q8, 256, 2><<<a.T, 256, 0, ctx->stream>>>(a);
    else if (a.d <= 8192 && few) rmsnorm_kernel<TYPE, Q8, 1024, 1><<<a.T, 1024, 0, ctx->stream>>>(a);
    else if (a.d <= 8192) rmsnorm_kernel<TYPE, Q8, 256, 4><<<a.T, 256, 0, ctx->stream>>>(a);
    else if (a.d <= 16384) rmsnorm_kernel<TYPE, Q8, 512, 4><<<a.T, 512, 0, ctx->stream>>>(a);
    else rmsnorm_kernel<TYPE, Q8, 1024, 8><<<a.T, 1024, 0, ctx->stream>>>(a);
}

template <int TYPE>
void launch_grad(obc_ctx *ctx, const GradArgs &a)
{
    const int blocks = grad_parts(a.T);
    if (a.d <= 2048) rmsnorm_grad_kernel<TYPE, 256, 1><<<blocks, 256, 0, ctx->stream>>>(a);
    else if (a.d <= 4096) rmsnorm_grad_kernel<TYPE, 512, 1><<<blocks, 512, 0, ctx->stream>>>(a);
    else if (a.d <= 8192) rmsnorm_grad_kernel<TYPE, 1024, 1><<<blocks, 1024, 0, ctx->stream>>>(a);
    else if (a.d <= 16384 && TYPE != OBC_F32) rmsnorm_grad_kernel<TYPE == OBC_F32 ? OBC_BF16 : TYPE, 1024, 2><<<blocks, 1024, 0, ctx->stream>>>(a);
    else rmsnorm_grad_wide_kernel<TYPE><<<blocks, 1024, 0, ctx->stream>>>(a);
}

}  // namespace

extern "C" {

int obc_rmsnorm(obc_ctx *ctx, const void *x, const void *residual, int x_type, const float *gain, float eps, int T, int d,
                void *h, void *y, int y_type, float *y_scale, float *rstd)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (T < 0 || d <= 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_rmsnorm: bad size");
    if (d > kMaxCols) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_rmsnorm: d (%d) > %d", d, kMaxCols);
    if (!float_type(x_type) || (y_type != x_type && y_type != OBC_I8))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_rmsnorm: x_type %d, y_type %d", x_type, y_type);
    if (!(eps >= 0.f)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_rmsnorm: eps is not >= 0");
    if (T == 0) return OBC_OK;
    if (!x || !gain || !y) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_rmsnorm: null x, gain or y");
    if ((y_type == OBC_I8) != (y_scale != nullptr))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_rmsnorm: y_scale goes with 8-bit outputs");
    if ((((uintptr_t)x | (uintptr_t)residual | (uintptr_t)h | (y_type == OBC_I8 ? 0 : (uintptr_t)y)) & (size_of_type(x_type) - 1)) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_rmsnorm: an array is not aligned to its elements");
    const bool q8 = y_type == OBC_I8;
    const size_t in = size_of_type(x_type), out = size_of_type(y_type);
    constexpr int kMost = 1 << 21;      // rows of a launch
    for (int t0 = 0; t0 < T; t0 += kMost) {
        const size_t at = (size_t)t0 * d;
        const NormArgs a = {(const char *)x + at * in, residual ? (const char *)residual + at * in : nullptr, gain,
                            h ? (char *)h + at * in : nullptr, (char *)y + at * out, y_scale ? y_scale + t0 : nullptr,
                            rstd ? rstd + t0 : nullptr, eps, T - t0 < kMost ? T - t0 : kMost, d};
        if (x_type == OBC_F32) q8 ? launch_norm<OBC_F32, true>(ctx, a) : launch_norm<OBC_F32, false>(ctx, a);
        else if (x_type == OBC_F16) q8 ? launch_norm<OBC_F16, true>(ctx, a) : launch_norm<OBC_F16, false>(ctx, a);
        else q8 ? launch_norm<OBC_BF16, true>(ctx, a) : launch_norm<OBC_BF16, false>(ctx, a);
        OBC_LAUNCH_CHECK(ctx, "rmsnorm_kernel");
        if (T - t0 <= kMost) break;
    }
    return OBC_OK;
}

int obc_rmsnorm_grad_workspace_bytes(int T, int d, size_t *bytes)
{
    if (!bytes || T < 0 || d <= 0) return OBC_ERR_BAD_ARG;
    *bytes = (size_t)grad_parts(T) * d * 4;
    return OBC_OK;
}

int obc_rmsnorm_grad(obc_ctx *ctx, const void *h, const float *gain, const float *rstd, const void *dy, const void *dh, int type,
                     int T, int d, void *dx, float *dgain, void *ws, size_t ws_bytes)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (T < 0 || d <= 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_rmsnorm_grad: bad size");
    if (d > kMaxCols) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_rmsnorm_grad: d (%d) > %d", d, kMaxCols);
    if (!float_type(type)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_rmsnorm_grad: type %d is not a floating type", type);
    if (!dgain || (T > 0 && (!h || !gain || !rstd || !dy || !dx))) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_rmsnorm_grad: null argument");
    if ((((uintptr_t)h | (uintptr_t)dy | (uintptr_t)dh | (uintptr_t)dx) & (size_of_type(type) - 1)) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_rmsnorm_grad: an array is not aligned to its elements");
    size_t need = 0;
    (void)obc_rmsnorm_grad_workspace_bytes(T, d, &need);
    if (need > 0 && (!ws || ((uintptr_t)ws & 15) != 0 || ws_bytes < need))
        return obc_fail(ctx, OBC_ERR_WORKSPACE, "obc_rmsnorm_grad: workspace of %zu bytes needed", need);
    if (T > 0) {
        const GradArgs a = {h, dy, dh, gain, rstd, dx, (float *)ws, T, d};
        if (type == OBC_F32) launch_grad<OBC_F32>(ctx, a);
        else if (type == OBC_F16) launch_grad<OBC_F16>(ctx, a);
        else launch_grad<OBC_BF16>(ctx, a);
        OBC_LAUNCH_CHECK(ctx, "rmsnorm_grad_kernel");
    }
    rmsnorm_dgain_kernel<<<(d + 63) / 64, 1024, 0, ctx->stream>>>((const float *)ws, grad_parts(T), d, dgain);
    OBC_LAUNCH_CHECK(ctx, "rmsnorm_dgain_kernel");
    return OBC_OK;
}

}  // extern "C"
