// obc_group_grid and obc_pack4: the grid of every group of a layer's columns, and the layer's codes in the
// order in which the products' matrix instructions take them (pack4.h).  Once per layer, at a third of the
// rate of a copy: loads of four bytes, few of them on their way (8192 x 8192: 167 us, 1.8 TB/s; the grid of its groups of 128 160 us).
#include "pack4.h"

namespace {

__device__ inline _Float16 next_half(_Float16 h)
{
    return __builtin_bit_cast(_Float16, (unsigned short)(__builtin_bit_cast(unsigned short, h) + 1));
}

// |v| in half precision, rounded away from zero or towards it
__device__ inline float half_up(float v)
{
    const _Float16 h = (_Float16)v;
    return (float)((float)h < v ? next_half(h) : h);
}

__device__ inline float half_down(float v)
{
    _Float16 h = (_Float16)v;
    if ((float)h > v) h = __builtin_bit_cast(_Float16, (unsigned short)(__builtin_bit_cast(unsigned short, h) - 1));
    return (float)h;
}

// The smallest number of 7 significant bits (and a multiple of half precision's smallest) that is >= v > 0:
// its products with a code, 11 bits, are exact in half precision.
__device__ inline float up7(float v)
{
    int e;
    (void)frexpf(v, &e);
    const float unit = ldexpf(1.f, e - 7 > -24 ? e - 7 : -24);
    return ceilf(v / unit) * unit;
}

// One wavefront per row and group.
__global__ __launch_bounds__(256) void group_grid_kernel(const float *__restrict__ W, const uint8_t *__restrict__ live,
                                                         int64_t jobs, int d, int G, int NG, int maxq, int flags,
                                                         float *__restrict__ delta, float *__restrict__ offset,
                                                         int *__restrict__ status)
{
    const int64_t job = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (job >= jobs) return;
    const int64_t row = job / NG;
    const int c0 = (int)(job - row * NG) * G;
    const int c1 = c0 + G < d ? c0 + G : d;
    float lo = __builtin_inff(), hi = -__builtin_inff();
    bool bad = false;
    for (int c = c0 + lane; c < c1; c += 64) {
        if (live && !live[row * d + c]) continue;
        const float v = W[row * d + c];
        bad |= !(fabsf(v) <= 65504.f);
        lo = fminf(lo, v);
        hi = fmaxf(hi, v);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        lo = fminf(lo, __shfl_xor(lo, off, 64));
        hi = fmaxf(hi, __shfl_xor(hi, off, 64));
    }
    bad = __any(bad);
    if (lane != 0) return;
    float step = 1.f, off = 0.f;
    if (lo <= hi && !bad) {
        const float m = fmaxf(fabsf(lo), fabsf(hi)), q = (float)maxq;
        if (flags & OBC_GRID_ZERO) {
            // the zero's code z: of the two beside -lo / delta the one with the finer grid
            const float a = flags & OBC_GRID_SYMMETRIC ? m : fmaxf(-lo, 0.f), b = flags & OBC_GRID_SYMMETRIC ? m : fmaxf(hi, 0.f);
            if (a + b > 0.f) {
                const float z0 = flags & OBC_GRID_SYMMETRIC ? floorf(0.5f * q) : floorf(a / (a + b) * q);
                float best = __builtin_inff(), bz = 0.f;
                for (float z = z0; z <= z0 + 1.f && z <= q; z += 1.f) {
                    const float need = fmaxf(a > 0.f ? (z > 0.f ? a / z : __builtin_inff()) : 0.f,
                                             b > 0.f ? (z < q ? b / (q - z) : __builtin_inff()) : 0.f);
                    if (need < best) { best = need; bz = z; }
                }
                step = up7(best);
                off = -step * bz;
            }
        } else if (flags & OBC_GRID_SYMMETRIC) {
            if (m > 0.f) {
                off = -half_up(m);
                step = half_up(-2.f * off / q);
            }
        } else {
            off = lo < 0.f ? -half_up(-lo) : half_down(lo);
            if (hi > off) {
                step = half_up((hi - off) / q);
                // (the range, rounded down, may have been such a number times q)
                if ((double)off + (double)q * step < (double)hi) step = (float)next_half((_Float16)step);
            }
        }
        bad = !(step <= 65504.f) || !(fabsf(off) <= 65504.f);
    }
    if (bad) obc_latch(status, OBC_ERR_NUMERIC);
    delta[job] = step;
    offset[job] = off;
}

__device__ inline unsigned half_bits(float v) { return __builtin_bit_cast(unsigned short, (_Float16)v); }

// One thread per dword of codes: eight consecutive columns of a row.
__global__ __launch_bounds__(256) void pack4_codes_kernel(const int32_t *__restrict__ codes, const float *__restrict__ delta,
                                                          const float *__restrict__ offset, pack4_layout L, int G,
                                                          unsigned *__restrict__ out, int *__restrict__ status)
{
    const int64_t tile = blockIdx.x;
    const int rb = (int)(tile / L.KT), kt = (int)(tile - (int64_t)rb * L.KT);
    const int lane = threadIdx.x >> 2, s = threadIdx.x & 3;
    const int64_t row = (int64_t)rb * 16 + (lane & 15);
    const int c0 = kt * 128 + 32 * s + 8 * (lane >> 4);
    unsigned word = 0;
    bool bad = false;
    if (row < L.R) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (c0 + j >= L.d) break;
            int q = codes[row * L.d + c0 + j];
            if (q == -1) {
                const int64_t e = row * L.NG + (c0 + j) / G;
                const float step = (float)(_Float16)delta[e], off = (float)(_Float16)offset[e];
                const float z = rintf(-off / step);
                q = z >= 0.f && z <= 15.f && off + step * z == 0.f ? (int)z : -1;
            }
            if (q < 0 || q > 15) { bad = true; q = 0; }
            word |= (unsigned)q << (4 * ((j >> 1) + 4 * (j & 1)));
        }
    }
    if (bad) obc_latch(status, OBC_ERR_BAD_ARG);
    out[tile * 256 + threadIdx.x] = word;
}

// One thread per (row, group) entry, those that pad included.
__global__ __launch_bounds__(256) void pack4_scales_kernel(const float *__restrict__ delta, const float *__restrict__ offset,
                                                           pack4_layout L, int per_row, int64_t entries,
                                                           unsigned *__restrict__ out, int *__restrict__ status)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= entries) return;
    const int64_t row = i / per_row;
    const int g = (int)(i - row * per_row);
    unsigned word = 0;
    if (row < L.R && g < L.NG) {
        const float step = delta[row * L.NG + g], off = offset[row * L.NG + g];
        if (!(fabsf((float)(_Float16)step) <= 65504.f) || !(fabsf((float)(_Float16)off) <= 65504.f))
            obc_latch(status, OBC_ERR_NUMERIC);
        word = half_bits(step) | half_bits(off) << 16;
    }
    const int64_t rb = row >> 4;
    const int n = (int)(row & 15);
    const int64_t at = L.SUB > 1 ? ((rb * L.KT + g / L.SUB) * 16 + n) * L.SUB + g % L.SUB : (rb * L.NG + g) * 16 + n;
    out[at] = word;
}

}  // namespace

extern "C" {

int obc_group_grid(obc_ctx *ctx, const float *W, const uint8_t *live, int R, int d, int group, int maxq, int flags,
                   float *delta, float *offset)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (R < 0 || d <= 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_group_grid: bad size");
    if (maxq < 1 || maxq > 15) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_group_grid: maxq (%d) outside 1..15", maxq);
    if (flags & ~(OBC_GRID_SYMMETRIC | OBC_GRID_ZERO))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_group_grid: unknown flags 0x%x", flags);
    if ((flags & OBC_GRID_ZERO) && maxq < 2)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_group_grid: a grid with a zero inside has at least 3 values");
    pack4_layout L;
    if (!pack4_layout_of(R, d, group, &L))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_group_grid: group (%d) is not 0, 32, 64 or a multiple of 128", group);
    if (R == 0) return OBC_OK;
    if (!W || !delta || !offset) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_group_grid: null argument");
    const int64_t jobs = (int64_t)R * L.NG, blocks = (jobs + 3) / 4;
    if (!obc_grid_fits(blocks, 256)) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_group_grid: too many groups");
    const int G = L.NG == 1 ? d : group;
    group_grid_kernel<<<(unsigned)blocks, 256, 0, ctx->stream>>>(W, live, jobs, d, G, L.NG, maxq, flags, delta, offset,
                                                                 ctx->d_status);
    OBC_LAUNCH_CHECK(ctx, "group_grid_kernel");
    return OBC_OK;
}

int obc_pack4_bytes(int R, int d, int group, size_t *bytes)
{
    pack4_layout L;
    if (!bytes || R < 0 || d <= 0 || !pack4_layout_of(R, d, group, &L)) return OBC_ERR_BAD_ARG;
    *bytes = L.bytes;
    return OBC_OK;
}

int obc_pack4(obc_ctx *ctx, const int32_t *codes, const float *delta, const float *offset, int R, int d, int group,
              void *packed)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (R < 0 || d <= 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_pack4: bad size");
    pack4_layout L;
    if (!pack4_layout_of(R, d, group, &L))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_pack4: group (%d) is not 0, 32, 64 or a multiple of 128", group);
    if (R == 0) return OBC_OK;
    if (!codes || !delta || !offset || !packed) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_pack4: null argument");
    if (((uintptr_t)packed & 15) != 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_pack4: packed is not aligned to 16 bytes");
    const int per_row = L.SUB > 1 ? L.KT * L.SUB : L.NG;
    const int64_t tiles = (int64_t)L.RB * L.KT, entries = (int64_t)L.RB * 16 * per_row;
    if (!obc_grid_fits(tiles, 256) || !obc_grid_fits((entries + 255) / 256, 256))
        return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_pack4: too many tiles");
    const int G = L.NG == 1 ? d : group;
    pack4_codes_kernel<<<(unsigned)tiles, 256, 0, ctx->stream>>>(codes, delta, offset, L, G, (unsigned *)packed, ctx->d_status);
    OBC_LAUNCH_CHECK(ctx, "pack4_codes_kernel");
    pack4_scales_kernel<<<(unsigned)((entries + 255) / 256), 256, 0, ctx->stream>>>(
        delta, offset, L, per_row, entries, (unsigned *)((char *)packed + L.scales), ctx->d_status);
    OBC_LAUNCH_CHECK(ctx, "pack4_scales_kernel");
    return OBC_OK;
}

}  // extern "C"
