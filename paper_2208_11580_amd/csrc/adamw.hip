// obc_adamw: a step of AdamW over many tensors in one launch for every kTensors of them.
//
//   g' = g grad_scale;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2
//   p = p (1 - lr decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// Moments are fp32, or 8-bit floating-point numbers times an fp32 scale per 256 of them, of m and of sqrt(v) (whose range is
// half of v's).  Those are rounded up or down by chance, from a hash of seed, step, tensor and element: rounded to nearest, v would
// stay where it is, since a step changes it by a thousandth and the nearest 8-bit numbers are an eighth away.  A root that is not
// zero does not become zero, or the next step would be divided by next to nothing.
#include "row_io.h"

namespace {

constexpr int kTensors = 32;      // of a launch: their descriptors go with its arguments
constexpr int NT = 256, E = 8, kChunk = NT * E;
constexpr int kScaled = 256;      // 8-bit moments that share a scale: 32 lanes' elements
constexpr float kTop8 = 448.f;    // the largest of the 8-bit numbers (4 bits of exponent, 3 of mantissa)

struct Args {
    obc_adamw_tensor t[kTensors];
    unsigned first[kTensors];      // the first workgroup of each tensor
    int tensors, ordinal;
    const int64_t *step;
    const float *lr_at, *grad_scale;
    double beta1, beta2;
    float lr, c1, c2, eps;
    unsigned key;                  // the seed's part of the hash
    int *status;
};

// 1 - b^t in 64 bits
__device__ inline double one_minus_power(double b, int64_t t)
{
    double r = 1.0;
    for (; t > 0; t >>= 1) {
        if (t & 1) r *= b;
        b *= b;
    }
    return 1.0 - r;
}

// 32 bits from an element's place: odd multipliers (of the fractions of the golden ratio, the root of 2, and pi) and shifts
__device__ inline unsigned mix(unsigned h)
{
    h *= 0x9E3779B1u;
    h ^= h >> 15;
    h *= 0x6A09E667u;
    h ^= h >> 14;
    h *= 0x243F6A89u;
    return h ^ h >> 16;
}

// a (0 .. 448) on the 8-bit numbers' grid: eight steps to an octave, down to 2^-9; up with a chance of the distance
__device__ inline float on_grid(float a, unsigned u16)
{
    const int e = max((int)(__builtin_bit_cast(unsigned, a) >> 23), 127 - 6) - 3;      // exponent of the grid's step
    const float q = __builtin_bit_cast(float, (unsigned)e << 23), per = __builtin_bit_cast(float, (unsigned)(254 - e) << 23);
    return floorf(a * per + (float)u16 * 0x1p-16f) * q;
}

__device__ inline float over_block(float v)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v = larger(v, __shfl_xor(v, off, 64));
    return v;
}

__device__ inline void load_bytes(const void *p, int64_t at, int left, unsigned (&w)[2])
{
    const uint8_t *q = (const uint8_t *)p + at;
    if (left >= 8) {
        const uintx2 x = *(const uintx2_at1 *)q;
        w[0] = x.x;
        w[1] = x.y;
        return;
    }
    w[0] = w[1] = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) w[j >> 2] |= (unsigned)q[j] << (8 * (j & 3));
}

__device__ inline void store_bytes(void *p, int64_t at, int left, const unsigned (&w)[2])
{
    uint8_t *q = (uint8_t *)p + at;
    if (left >= 8) {
        *(uintx2_at1 *)q = uintx2{w[0], w[1]};
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) q[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
}

__device__ inline void decode(const unsigned (&w)[2], float scale, float (&v)[8])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const auto pair = j & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(w[j >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8(w[j >> 1], false);
        v[2 * j] = pair[0] * scale;
        v[2 * j + 1] = pair[1] * scale;
    }
}

// (numbers of the grid: the conversion rounds nothing)
__device__ inline void encode(const float (&v)[8], unsigned (&w)[2])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
        w[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], x, true);
    }
}

template <int TYPE, bool BITS8>
__global__ __launch_bounds__(NT) void adamw_kernel(Args a)
{
    __shared__ float shared[2];
    const int tid = threadIdx.x;
    // the tensor: the last that begins at or before this workgroup
    const int lane = tid & 63;
    const unsigned begins = a.first[lane < kTensors ? lane : 0];
    const int n_before = __popcll(__ballot(lane < a.tensors && lane < kTensors && begins <= blockIdx.x));
    const int ti = __builtin_amdgcn_readfirstlane(n_before - 1);
    const obc_adamw_tensor t = a.t[ti];
    const int64_t at = (int64_t)(blockIdx.x - a.first[ti]) * kChunk + tid * E, left64 = t.n - at;
    const int left = left64 < 0 ? 0 : left64 > E ? E : (int)left64;
    const bool master = t.master != nullptr;

    float p[8], g[8], m[8], v[8];
    unsigned m8[2], v8[2];
    float m_scale = 0.f, v_scale = 0.f;
    if (master) load8<OBC_F32>(t.master, at, left, p);
    else load8<TYPE>(t.p, at, left, p);
    load8<TYPE>(t.g, at, left, g);
    if (BITS8) {
        load_bytes(t.m, at, left, m8);
        load_bytes(t.v, at, left, v8);
        if (left > 0) {
            m_scale = t.m_scale[at / kScaled];
            v_scale = t.v_scale[at / kScaled];
        }
    } else {
        load8<OBC_F32>(t.m, at, left, m);
        load8<OBC_F32>(t.v, at, left, v);
    }
    float c1 = a.c1, c2 = a.c2;
    const int64_t step = a.step ? *a.step : 0;
    unsigned key = a.key;
    if (a.step) {
        if (tid == 0) shared[0] = (float)(1.0 / one_minus_power(a.beta1, step));
        if (tid == 64) shared[1] = (float)(1.0 / sqrt(one_minus_power(a.beta2, step)));
        __syncthreads();
        c1 = shared[0];
        c2 = shared[1];
        key += (unsigned)step * 0xBB67AE85u;
    }
    const float lr = a.lr_at ? *a.lr_at : a.lr, gs = a.grad_scale ? *a.grad_scale : 1.f;
    const float b1 = (float)a.beta1, b2 = (float)a.beta2, n1 = (float)(1.0 - a.beta1), n2 = (float)(1.0 - a.beta2);
    const bool skip = !(fabsf(gs) < __builtin_inff()) || (a.step && step < 1);
    if (a.step && step < 1 && blockIdx.x == 0 && tid == 0) obc_latch(a.status, OBC_ERR_BAD_ARG);
    const float keep = (float)(1.0 - (double)lr * (double)t.decay), rate = lr * c1;
    float root[8];
    if (BITS8) {
        decode(m8, m_scale, m);
        decode(v8, v_scale, root);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = root[j] * root[j];
    }
    if (!skip) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float x = g[j] * gs;
            m[j] = fmaf(m[j], b1, x * n1);
            v[j] = fmaf(v[j], b2, x * x * n2);
            root[j] = sqrtf(v[j]);
            p[j] = p[j] * keep - rate * m[j] / fmaf(root[j], c2, a.eps);
        }
    }
    if (left > 0) {
        if (master) store8<OBC_F32>(t.master_out, at, left, p);
        if (!(skip && master)) store8<TYPE>(t.p_out, at, left, p);
    }
    if (skip && master && left > 0) {      // the parameters as they were, which need not be the copies rounded
        float old[8];
        load8<TYPE>(t.p, at, left, old);
        store8<TYPE>(t.p_out, at, left, old);
    }
    if (!BITS8) {
        if (left > 0) {
            store8<OBC_F32>(t.m_out, at, left, m);
            store8<OBC_F32>(t.v_out, at, left, v);
        }
        return;
    }
    if (!skip) {
        float top_m = 0.f, top_v = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            top_m = larger(top_m, j < left ? m[j] : 0.f);
            top_v = larger(top_v, j < left ? root[j] : 0.f);
        }
        top_m = over_block(top_m);
        top_v = over_block(top_v);
        // (a block whose largest number is next to nothing, below 1e-30, is taken for zeros: its reciprocal would not be finite)
        const bool lost_m = !(top_m < __builtin_inff()), lost_v = !(top_v < __builtin_inff());
        const float up_m = !lost_m && top_m > 1e-30f ? kTop8 / top_m : 0.f, up_v = !lost_v && top_v > 1e-30f ? kTop8 / top_v : 0.f;
        m_scale = lost_m ? __builtin_nanf("") : top_m > 1e-30f ? top_m / kTop8 : 0.f;
        v_scale = lost_v ? __builtin_nanf("") : top_v > 1e-30f ? top_v / kTop8 : 0.f;
        const unsigned base = key + (unsigned)(a.ordinal + ti) * 0x3C6EF373u + (unsigned)((uint64_t)at >> 32) * 0x243F6A89u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned u = mix(((unsigned)at + j) ^ base);
            const float am = lost_m ? 0.f : fminf(fabsf(m[j]) * up_m, kTop8), av = lost_v ? 0.f : fminf(root[j] * up_v, kTop8);
            m[j] = copysignf(on_grid(am, u & 0xffffu), m[j]);
            root[j] = on_grid(av, u >> 16);
            if (av > 0.f) root[j] = fmaxf(root[j], 0x1p-9f);
        }
        encode(m, m8);
        encode(root, v8);
    }
    if (left > 0) {
        store_bytes(t.m_out, at, left, m8);
        store_bytes(t.v_out, at, left, v8);
        if (at % kScaled == 0) {
            t.m_scale_out[at / kScaled] = m_scale;
            t.v_scale_out[at / kScaled] = v_scale;
        }
    }
}

template <int TYPE>
void launch(obc_ctx *ctx, const Args &a, unsigned blocks, bool bits8)
{
    if (bits8) adamw_kernel<TYPE, true><<<blocks, NT, 0, ctx->stream>>>(a);
    else adamw_kernel<TYPE, false><<<blocks, NT, 0, ctx->stream>>>(a);
}

}  // namespace

extern "C" int obc_adamw(obc_ctx *ctx, const obc_adamw_tensor *tensors, int count, int type, int bits, int64_t step, const int64_t *step_at,
                         float lr, const float *lr_at, double beta1, double beta2, float eps, const float *grad_scale, uint32_t seed)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (count < 0 || (count > 0 && !tensors)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: no tensors");
    if (!float_type(type) || (bits != 8 && bits != 32)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: type %d, moments of %d bits", type, bits);
    if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: betas are in [0, 1)");
    if (!(eps > 0.f && eps < __builtin_inff())) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: eps is not positive and finite");
    if (!step_at && step < 1) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: steps count from 1");
    if (!lr_at && !(fabsf(lr) < __builtin_inff())) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: lr is not finite");
    if ((((uintptr_t)step_at) & 7) != 0 || (((uintptr_t)lr_at | (uintptr_t)grad_scale) & 3) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: step_at, lr_at or grad_scale is not aligned");
    const size_t e = size_of_type(type) - 1;
    for (int i = 0; i < count; ++i) {
        const obc_adamw_tensor &t = tensors[i];
        if (t.n < 0 || t.n > (int64_t)1 << 40) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: tensor %d: bad size", i);
        if (!(fabsf(t.decay) < __builtin_inff())) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: tensor %d: decay is not finite", i);
        if (t.n == 0) continue;
        if (!t.p || !t.p_out || !t.g || !t.m || !t.m_out || !t.v || !t.v_out || (t.master == nullptr) != (t.master_out == nullptr))
            return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: tensor %d: null argument", i);
        if (bits == 8 && (!t.m_scale || !t.m_scale_out || !t.v_scale || !t.v_scale_out))
            return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: tensor %d: moments of 8 bits have scales", i);
        const uintptr_t words = (uintptr_t)t.master | (uintptr_t)t.master_out |
                                (bits == 8 ? (uintptr_t)t.m_scale | (uintptr_t)t.m_scale_out | (uintptr_t)t.v_scale | (uintptr_t)t.v_scale_out
                                           : (uintptr_t)t.m | (uintptr_t)t.m_out | (uintptr_t)t.v | (uintptr_t)t.v_out);
        if (((((uintptr_t)t.p | (uintptr_t)t.p_out | (uintptr_t)t.g) & e) | (words & 3)) != 0)
            return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: tensor %d: an array is not aligned to its elements", i);
    }
    Args a;
    a.step = step_at;
    a.lr_at = lr_at;
    a.grad_scale = grad_scale;
    a.beta1 = beta1;
    a.beta2 = beta2;
    a.lr = lr;
    a.eps = eps;
    a.c1 = a.c2 = 1.f;
    a.key = seed * 0x6A09E667u;
    a.status = ctx->d_status;
    if (!step_at) {
        a.c1 = (float)(1.0 / -expm1((double)step * log(beta1)));
        a.c2 = (float)(1.0 / sqrt(-expm1((double)step * log(beta2))));
        a.key += (unsigned)step * 0xBB67AE85u;
    }
    constexpr int64_t kMostBlocks = 1 << 23;      // of a launch: below 2^32 threads
    int i = 0;
    while (i < count) {
        a.tensors = 0;
        a.ordinal = i;
        int64_t blocks = 0;
        for (; i < count && a.tensors < kTensors; ++i) {
            const int64_t more = (tensors[i].n + kChunk - 1) / kChunk;
            if (a.tensors > 0 && blocks + more > kMostBlocks) break;
            if (more > kMostBlocks) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_adamw: tensor %d: more than 2^34 - 1 elements", i);
            a.first[a.tensors] = (unsigned)blocks;
            a.t[a.tensors++] = tensors[i];
            blocks += more;
        }
        if (blocks == 0) continue;
        if (type == OBC_F32) launch<OBC_F32>(ctx, a, (unsigned)blocks, bits == 8);
        else if (type == OBC_F16) launch<OBC_F16>(ctx, a, (unsigned)blocks, bits == 8);
        else launch<OBC_BF16>(ctx, a, (unsigned)blocks, bits == 8);
        OBC_LAUNCH_CHECK(ctx, "adamw_kernel");
    }
    return OBC_OK;
}
