// obc_layernorm and obc_layernorm_grad: layer norm with the residual's addition, an output in 8 bits, and the backward pass.
//
//   mean = sum h / d, var = sum (h - mean)^2 / d, y = (h - mean) rstd gain + bias
// A row is read once and kept in registers: the mean first, then what is left, c = h - mean, and its squares.  The mean is rounded, which would move
// all of y alike, so c is summed beside its squares: with e = sum c / d, the mean is off by e, y = (c - e) rstd gain + bias and
// var = sum c^2 / d - e^2.  A large mean so costs no digits of either.  8 bits take a third reduction, the largest |y|.
//
// Memory-bound: 4096 x 8192 in bf16 with residual and sum, 268 MB, takes 52 us with fresh inputs (5.2 TB/s; a large copy reaches 5.2), one row of
// 768 2.8 us in a graph, of which an empty launch is 2.  The backward pass keeps each workgroup's shares of the gain's and the bias's gradient in registers
// over its rows: 4096 x 4096 in bf16 with the residual's gradient, 134 MB, takes 29 to 37 us (fresh inputs), 24 to 31 of them the
// rows and 5 the sum of 512 shares.
#include "row_io.h"

namespace {

constexpr int kMaxCols = 65536;

// Sums over a workgroup, the same values in every thread.  A buffer may be used again two reductions later.
template <int NT, int N>
__device__ inline void sums(float (&v)[N], float (*buf)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = sum_lanes(v[i]);
    if (NT == 64) return;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) buf[threadIdx.x >> 6][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = buf[0][i];
#pragma unroll
        for (int w = 1; w < NT / 64; ++w) v[i] += buf[w][i];
    }
}

// The largest of magnitudes (a NaN is larger than any number)
template <int NT>
__device__ inline float largest(float v, float *buf)
{
    v = join_lanes(v, larger);
    if (NT == 64) return v;
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    v = buf[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v = larger(v, buf[w]);
    return v;
}

struct NormArgs {
    const void *x, *residual;
    const float *gain, *bias;
    void *h, *y;
    float *y_scale, *mean, *rstd;
    float eps;
    int T, d;
    bool past;
};

template <int TYPE, bool Q8, int NT, int CH>
__global__ __launch_bounds__(NT) void layernorm_kernel(NormArgs a)
{
    __shared__ float buf1[NT / 64][1], buf2[NT / 64][2], buf3[NT / 64];
    const int64_t row = blockIdx.x, base = row * a.d;
    float v[CH][8];
    float sum[1] = {0.f};
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
        if (a.h) put8<TYPE>(a.h, base + c, left, v[k], a.past);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[0] += v[k][j];      // (zeros beyond the row's end)
    }
    sums<NT>(sum, buf1);
    const float mean = sum[0] / (float)a.d;
    float sq[2] = {0.f, 0.f};      // of c^2, of c
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int left = a.d - (k * NT + (int)threadIdx.x) * 8;
        if (left <= 0) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[k][j] = j < left ? v[k][j] - mean : 0.f;
            sq[0] = fmaf(v[k][j], v[k][j], sq[0]);
            sq[1] += v[k][j];
        }
    }
    sums<NT>(sq, buf2);
    const float off = sq[1] / (float)a.d;
    float var = fmaf(-off, off, sq[0] / (float)a.d);
    var = var < 0.f ? 0.f : var;      // (rows of one value; a NaN stays one)
    const float rstd = 1.f / sqrtf(var + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean + off;
        if (a.rstd) a.rstd[row] = rstd;
    }
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * NT + (int)threadIdx.x) * 8, left = a.d - c;
        if (left <= 0) continue;
        float g[8], b[8];
        load8<OBC_F32>(a.gain, c, left, g);
        if (a.bias) load8<OBC_F32>(a.bias, c, left, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[k][j] = fmaf((v[k][j] - off) * rstd, g[j], a.bias ? b[j] : 0.f);
            if (Q8) top = larger(top, v[k][j]);
        }
        if (!Q8) put8<TYPE>(a.y, base + c, left, v[k], a.past);
    }
    if (!Q8) return;
    top = largest<NT>(top, buf3);
    // A row whose largest value is next to nothing is scaled up first, so that its reciprocal stays finite.
    const bool lost = !(sq[0] < __builtin_inff()) || !(top < __builtin_inff());
    const float up = top < 1e-30f ? 0x1p90f : 1.f, mul = top > 0.f ? 127.f / (top * up) : 0.f;
    if (threadIdx.x == 0) a.y_scale[row] = lost ? __builtin_nanf("") : top > 0.f ? top / 127.f : 1.f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * NT + (int)threadIdx.x) * 8, left = a.d - c;
        if (left <= 0) continue;
        unsigned w[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float q = fminf(fmaxf(rintf(v[k][j] * up * mul), -127.f), 127.f);
            w[j >> 2] |= lost ? 0u : ((unsigned)(int)q & 0xffu) << (8 * (j & 3));
        }
        uint8_t *p = (uint8_t *)a.y + base + c;
        if (left >= 8) *(uintx2_at1 *)p = uintx2{w[0], w[1]};
        else
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < left) p[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
    }
}

struct GradArgs {
    const void *h, *dy, *dh;
    const float *gain, *mean, *rstd;
    void *dx;
    float *part;      // per workgroup: its rows' share of dgain, then of dbias
    int T, d;
    bool past;
};

// Workgroup b takes the rows b, b + gridDim.x, ... and keeps its columns' shares of dgain and dbias in registers; the next
// row's loads are on their way while it reduces this one.
template <int TYPE, int NT, int CH>
__global__ __launch_bounds__(NT) void layernorm_grad_kernel(GradArgs a)
{
    __shared__ float buf[2][NT / 64][2];
    float dg[CH][8], db[CH][8], gain[CH][8];
    Eight<TYPE> h[CH], dy[CH];
    const int tid = threadIdx.x;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * NT + tid) * 8, left = a.d - c;
#pragma unroll
        for (int j = 0; j < 8; ++j) dg[k][j] = db[k][j] = gain[k][j] = 0.f;
        if (left <= 0) continue;
        load8<OBC_F32>(a.gain, c, left, gain[k]);
        h[k].load(a.h, (int64_t)blockIdx.x * a.d + c, left);
        dy[k].load(a.dy, (int64_t)blockIdx.x * a.d + c, left);
    }
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x, turn ^= 1) {
        const int64_t base = row * a.d, next = row + gridDim.x < a.T ? base + (int64_t)gridDim.x * a.d : base;
        const float rstd = a.rstd[row], mean = a.mean[row];
        Eight<TYPE> dh[CH];
        float x[CH][8], g[CH][8];
        float s[2] = {0.f, 0.f};
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
            for (int j = 0; j < 8; ++j) {      // (beyond the row's end dy and the gain are zero)
                x[k][j] = (x[k][j] - mean) * rstd;
                dg[k][j] = fmaf(g[k][j], x[k][j], dg[k][j]);
                db[k][j] += g[k][j];
                g[k][j] *= gain[k][j];
                s[0] += g[k][j];
                s[1] = fmaf(g[k][j], x[k][j], s[1]);
            }
        }
        sums<NT>(s, buf[turn]);
        const float m0 = s[0] / (float)a.d, m1 = s[1] / (float)a.d;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * NT + tid) * 8, left = a.d - c;
            if (left <= 0) continue;
            float r[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) r[j] = 0.f;
            if (a.dh) dh[k].get(r);
#pragma unroll
            for (int j = 0; j < 8; ++j) r[j] = fmaf(rstd, fmaf(-x[k][j], m1, g[k][j] - m0), r[j]);
            put8<TYPE>(a.dx, base + c, left, r, a.past);
        }
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * NT + tid) * 8, left = a.d - c;
        if (left <= 0) continue;
        store8<OBC_F32>(a.part, (int64_t)blockIdx.x * 2 * a.d + c, left, dg[k]);
        store8<OBC_F32>(a.part, ((int64_t)blockIdx.x * 2 + 1) * a.d + c, left, db[k]);
    }
}

// Rows too wide for registers beside their shares: read a second time, from the caches.  SHARES false: rows whose shares alone
// are too many; layernorm_grad_columns_kernel forms them.
template <int TYPE, int CH, bool SHARES>
__global__ __launch_bounds__(1024) void layernorm_grad_wide_kernel(GradArgs a)
{
    constexpr int NT = 1024, KEPT = SHARES ? CH : 1;
    __shared__ float buf[2][NT / 64][2];
    float dg[KEPT][8], db[KEPT][8];
#pragma unroll
    for (int k = 0; k < KEPT; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) dg[k][j] = db[k][j] = 0.f;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x, turn ^= 1) {
        const int64_t base = row * a.d;
        const float rstd = a.rstd[row], mean = a.mean[row];
        float s[2] = {0.f, 0.f};
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
                const float xhat = (x[j] - mean) * rstd;
                if (SHARES) {
                    dg[k % KEPT][j] = fmaf(g[j], xhat, dg[k % KEPT][j]);
                    db[k % KEPT][j] += g[j];
                }
                g[j] *= w[j];
                s[0] += g[j];
                s[1] = fmaf(g[j], xhat, s[1]);
            }
        }
        sums<NT>(s, buf[turn]);
        const float m0 = s[0] / (float)a.d, m1 = s[1] / (float)a.d;
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
            for (int j = 0; j < 8; ++j) r[j] = fmaf(rstd, fmaf(-(x[j] - mean) * rstd, m1, g[j] * w[j] - m0), r[j]);
            put8<TYPE>(a.dx, base + c, left, r, a.past);
        }
    }
    if (!SHARES) return;
#pragma unroll
    for (int k = 0; k < KEPT; ++k) {
        const int c = (k * NT + (int)threadIdx.x) * 8, left = a.d - c;
        if (left <= 0) continue;
        store8<OBC_F32>(a.part, (int64_t)blockIdx.x * 2 * a.d + c, left, dg[k]);
        store8<OBC_F32>(a.part, ((int64_t)blockIdx.x * 2 + 1) * a.d + c, left, db[k]);
    }
}

// The shares of the rows blockIdx.x, blockIdx.x + gridDim.x, ... in 2048 columns
template <int TYPE>
__global__ __launch_bounds__(256) void layernorm_grad_columns_kernel(GradArgs a)
{
    const int c = (blockIdx.y * 256 + threadIdx.x) * 8, left = a.d - c;
    if (left <= 0) return;
    float dg[8], db[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[j] = db[j] = 0.f;
#pragma unroll 2
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
        const float rstd = a.rstd[row], mean = a.mean[row];
        float x[8], g[8];
        load8<TYPE>(a.h, row * a.d + c, left, x);
        load8<TYPE>(a.dy, row * a.d + c, left, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            dg[j] = fmaf(g[j], (x[j] - mean) * rstd, dg[j]);
            db[j] += g[j];
        }
    }
    store8<OBC_F32>(a.part, (int64_t)blockIdx.x * 2 * a.d + c, left, dg);
    store8<OBC_F32>(a.part, ((int64_t)blockIdx.x * 2 + 1) * a.d + c, left, db);
}

// dgain and dbias: the sums of the workgroups' shares, in a fixed order; 64 of their 2 d values to a workgroup of 16 waves
__global__ __launch_bounds__(1024) void layernorm_shares_kernel(const float *__restrict__ part, int parts, int d, float *__restrict__ dgain,
                                                                float *__restrict__ dbias)
{
    __shared__ float buf[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane, n = 2 * d;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c < n) {
        int p = wave;
        for (; p + 7 * 16 < parts; p += 8 * 16)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += part[(int64_t)(p + i * 16) * n + c];
        for (; p < parts; p += 16) s[0] += part[(int64_t)p * n + c];
    }
    buf[wave][lane] = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
    __syncthreads();
    if (wave == 0 && c < n) {
        float v = buf[0][lane];
#pragma unroll
        for (int w = 1; w < 16; ++w) v += buf[w][lane];
        if (c < d) dgain[c] = v;
        else if (dbias) dbias[c - d] = v;
    }
}

inline int grad_parts(int T) { return T < 512 ? T : 512; }

template <int TYPE, bool Q8>
void launch_norm(obc_ctx *ctx, const NormArgs &a)
{
    // Few rows: as many threads to a row as it has pieces, for the sooner end of each.  Many: the fewest that leave a row's values in
    // registers without giving up waves (fresh inputs: 4096 x 8192 in bf16 with 512 threads 54 us, 256 59, 1024 55 to 57; 2000 x 8000 in fp32
    // with 1024 54 us, 512 60, 256 63; 4096 x 4096 in bf16 22.3 us with 256 or 512)
    const bool few = a.T <= 512;
    if (a.d <= 2048) layernorm_kernel<TYPE, Q8, 256, 1><<<a.T, 256, 0, ctx->stream>>>(a);
    else if (a.d <= 4096 && few) layernorm_kernel<TYPE, Q8, 512, 1><<<a.T, 512, 0, ctx->stream>>>(a);
    else if (a.d <= 4096) layernorm_kernel<TYPE, Q8, 256, 2><<<a.T, 256, 0, ctx->stream>>>(a);
    else if (a.d <= 8192 && (few || TYPE == OBC_F32)) layernorm_kernel<TYPE, Q8, 1024, 1><<<a.T, 1024, 0, ctx->stream>>>(a);
    else if (a.d <= 8192) layernorm_kernel<TYPE, Q8, 512, 2><<<a.T, 512, 0, ctx->stream>>>(a);
    else if (a.d <= 16384) layernorm_kernel<TYPE, Q8, 512, 4><<<a.T, 512, 0, ctx->stream>>>(a);
    else layernorm_kernel<TYPE, Q8, 1024, 8><<<a.T, 1024, 0, ctx->stream>>>(a);
}

template <int TYPE>
void launch_grad(obc_ctx *ctx, const GradArgs &a)
{
    const int blocks = grad_parts(a.T);
    if (a.d <= 2048) layernorm_grad_kernel<TYPE, 256, 1><<<blocks, 256, 0, ctx->stream>>>(a);
    else if (a.d <= 4096) layernorm_grad_kernel<TYPE, 512, 1><<<blocks, 512, 0, ctx->stream>>>(a);
    else if (a.d <= 8192) layernorm_grad_kernel<TYPE, 1024, 1><<<blocks, 1024, 0, ctx->stream>>>(a);
    else if (a.d <= 16384) layernorm_grad_wide_kernel<TYPE, 2, true><<<blocks, 1024, 0, ctx->stream>>>(a);
    else if (a.d <= 32768) layernorm_grad_wide_kernel<TYPE, 4, true><<<blocks, 1024, 0, ctx->stream>>>(a);
    else {
        // (the shares first: dx may take dy's place)
        layernorm_grad_columns_kernel<TYPE><<<dim3(blocks, (a.d + 2047) / 2048), 256, 0, ctx->stream>>>(a);
        layernorm_grad_wide_kernel<TYPE, kMaxCols / (1024 * 8), false><<<blocks, 1024, 0, ctx->stream>>>(a);
    }
}

}  // namespace

extern "C" {

int obc_layernorm(obc_ctx *ctx, const void *x, const void *residual, int x_type, const float *gain, const float *bias, float eps, int T,
                  int d, void *h, void *y, int y_type, float *y_scale, float *mean, float *rstd)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (T < 0 || d <= 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_layernorm: bad size");
    if (d > kMaxCols) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_layernorm: d (%d) > %d", d, kMaxCols);
    if (!float_type(x_type) || (y_type != x_type && y_type != OBC_I8))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_layernorm: x_type %d, y_type %d", x_type, y_type);
    if (!(eps >= 0.f)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_layernorm: eps is not >= 0");
    if (T == 0) return OBC_OK;
    if (!x || !gain || !y) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_layernorm: null x, gain or y");
    if ((y_type == OBC_I8) != (y_scale != nullptr))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_layernorm: y_scale goes with 8-bit outputs");
    if ((((uintptr_t)x | (uintptr_t)residual | (uintptr_t)h | (y_type == OBC_I8 ? 0 : (uintptr_t)y)) & (size_of_type(x_type) - 1)) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_layernorm: an array is not aligned to its elements");
    const bool q8 = y_type == OBC_I8;
    const size_t in = size_of_type(x_type), out = size_of_type(y_type);
    constexpr int kMost = 1 << 21;      // rows of a launch
    for (int64_t t0 = 0; t0 < T; t0 += kMost) {
        const size_t at = (size_t)t0 * d;
        const NormArgs a = {(const char *)x + at * in, residual ? (const char *)residual + at * in : nullptr, gain, bias,
                            h ? (char *)h + at * in : nullptr, (char *)y + at * out, y_scale ? y_scale + t0 : nullptr,
                            mean ? mean + t0 : nullptr, rstd ? rstd + t0 : nullptr, eps, T - t0 < kMost ? (int)(T - t0) : kMost, d, (int64_t)T * d * (int64_t)(out + (h ? in : 0)) > kCaches};
        if (x_type == OBC_F32) q8 ? launch_norm<OBC_F32, true>(ctx, a) : launch_norm<OBC_F32, false>(ctx, a);
        else if (x_type == OBC_F16) q8 ? launch_norm<OBC_F16, true>(ctx, a) : launch_norm<OBC_F16, false>(ctx, a);
        else q8 ? launch_norm<OBC_BF16, true>(ctx, a) : launch_norm<OBC_BF16, false>(ctx, a);
        OBC_LAUNCH_CHECK(ctx, "layernorm_kernel");
    }
    return OBC_OK;
}

int obc_layernorm_grad_workspace_bytes(int T, int d, size_t *bytes)
{
    if (!bytes || T < 0 || d <= 0) return OBC_ERR_BAD_ARG;
    *bytes = (size_t)grad_parts(T) * d * 8;
    return OBC_OK;
}

int obc_layernorm_grad(obc_ctx *ctx, const void *h, const float *gain, const float *mean, const float *rstd, const void *dy, const void *dh,
                       int type, int T, int d, void *dx, float *dgain, float *dbias, void *ws, size_t ws_bytes)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (T < 0 || d <= 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_layernorm_grad: bad size");
    if (d > kMaxCols) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_layernorm_grad: d (%d) > %d", d, kMaxCols);
    if (!float_type(type)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_layernorm_grad: type %d is not a floating type", type);
    if (!dgain || (T > 0 && (!h || !gain || !mean || !rstd || !dy || !dx)))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_layernorm_grad: null argument");
    if ((((uintptr_t)h | (uintptr_t)dy | (uintptr_t)dh | (uintptr_t)dx) & (size_of_type(type) - 1)) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_layernorm_grad: an array is not aligned to its elements");
    size_t need = 0;
    (void)obc_layernorm_grad_workspace_bytes(T, d, &need);
    if (need > 0 && (!ws || ((uintptr_t)ws & 15) != 0 || ws_bytes < need))
        return obc_fail(ctx, OBC_ERR_WORKSPACE, "obc_layernorm_grad: workspace of %zu bytes needed", need);
    if (T > 0) {
        const GradArgs a = {h, dy, dh, gain, mean, rstd, dx, (float *)ws, T, d, (int64_t)T * d * (int64_t)size_of_type(type) > kCaches};
        if (type == OBC_F32) launch_grad<OBC_F32>(ctx, a);
        else if (type == OBC_F16) launch_grad<OBC_F16>(ctx, a);
        else launch_grad<OBC_BF16>(ctx, a);
        OBC_LAUNCH_CHECK(ctx, "layernorm_grad_kernel");
    }
    layernorm_shares_kernel<<<(2 * d + 63) / 64, 1024, 0, ctx->stream>>>((const float *)ws, grad_parts(T), d, dgain, dbias);
    OBC_LAUNCH_CHECK(ctx, "layernorm_shares_kernel");
    return OBC_OK;
}

}  // extern "C"
