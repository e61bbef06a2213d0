// obc_adamw: a step of AdamW over many tensors in one launch; obc_adamw_plan writes their descriptors to device memory once.
//
//   g' = g grad_scale;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2
//   p = p (1 - lr decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// Moments are fp32, or 8-bit floating-point numbers times an fp32 scale per 256 of them, of m and of sqrt(v) (whose range is
// half of v's).  Those are rounded up or down by chance, from a hash of seed, step, tensor and element: rounded to nearest, v would
// stay where it is, since a step changes it by a thousandth and the nearest 8-bit numbers are an eighth away.  A root that is not
// zero does not become zero, or the next step would be divided by next to nothing.
//
// Memory-bound: 52 million parameters in bf16 with fp32 copies and 8-bit moments, 835 MB, take 152 to 174 us (4.8 to 5.5 TB/s), 26 million in fp32
// with fp32 moments, 728 MB, 132 us (5.5 TB/s); 50 tensors of 768 values 3.9 us.  With 8 bits the vector instructions, some 80 to a
// parameter, are busy for most of that time.
#include <algorithm>

#include "row_io.h"

namespace {

constexpr int kWritten = 24;      // descriptors that a launch of the plan's kernel takes with its arguments
constexpr int NT = 256, E = 8, kChunk = NT * E;
constexpr int64_t kMostBlocks = (1 << 24) - 1;      // a launch holds fewer than 2^32 threads
constexpr int kScaled = 256;      // 8-bit moments that share a scale: 32 lanes' elements
constexpr float kTop8 = 448.f;    // the largest of the 8-bit numbers (4 bits of exponent, 3 of mantissa)

// A plan: the tensors' descriptors, and from which workgroup on each is
struct Layout {
    size_t first, bytes;
};
inline Layout layout_of(int count)
{
    const size_t t = obc_align_up((size_t)count * sizeof(obc_adamw_tensor), 256);
    return Layout{t, t + obc_align_up((size_t)count * 4, 256)};
}

struct PlanArgs {
    obc_adamw_tensor t[kWritten];
    unsigned first[kWritten];
    int tensors;
    obc_adamw_tensor *to;
    unsigned *first_to;
};

__global__ __launch_bounds__(64) void adamw_plan_kernel(PlanArgs a)
{
    const int i = threadIdx.x;
    if (i >= a.tensors) return;
    a.to[i] = a.t[i];
    a.first_to[i] = a.first[i];
}

struct Args {
    const obc_adamw_tensor *t;
    const unsigned *first;
    int tensors;
    const int64_t *step;
    const float *lr_at, *grad_scale;
    double beta1, beta2, root_b2, root_n2;      // and the roots of beta2 and 1 - beta2
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

constexpr unsigned kClose = 6;      // units of a float's last place
constexpr float kSmall = 0x1p-100f;      // of v: its root is taken in another range

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

// a (0 .. 448) on the 8-bit numbers' grid: eight steps to an octave, down to 2^-9; up with a chance of the distance.  From 2^-6 on that
// is to add u, 20 bits of chance, to the 20 bits that go, and what is smaller is moved there first.  edge: how near to where the sum
// turns it fell, at least, in units of a float's last place.
__device__ inline float on_grid(float a, unsigned u, unsigned &edge)
{
    const float off = a < 0x1p-6f ? 0x1p-6f : 0.f;
    const unsigned sum = __builtin_bit_cast(unsigned, a + off) + u;
    edge = min(edge, (sum + kClose) & 0xfffffu);
    return __builtin_bit_cast(float, sum & 0xfff00000u) - off;
}

__device__ inline double on_grid(double a, unsigned u16)
{
    const int e = max((int)(__builtin_bit_cast(unsigned long long, a) >> 52), 1023 - 6) - 3;
    const double q = __builtin_bit_cast(double, (unsigned long long)e << 52), per = __builtin_bit_cast(double, (unsigned long long)(2046 - e) << 52);
    return floor(a * per + (double)u16 * 0x1p-16) * q;
}

// The first element to the end
template <typename V>
__device__ inline void turn(V (&v)[8])
{
    const V first = v[0];
#pragma unroll
    for (int j = 0; j < 7; ++j) v[j] = v[j + 1];
    v[7] = first;
}

__device__ inline void turn_bytes(unsigned (&w)[2])
{
    const unsigned lo = __builtin_amdgcn_alignbyte(w[1], w[0], 1), hi = __builtin_amdgcn_alignbyte(w[0], w[1], 1);
    w[0] = lo;
    w[1] = hi;
}

__device__ inline double over_block(double v)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const double o = __shfl_xor(v, off, 64);
        v = o > v ? o : v;
    }
    return v;
}

__device__ inline unsigned over_block(unsigned v)
{
    return join_lanes<32>(v, [](unsigned a, unsigned b) { return max(a, b); });
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

__device__ inline void decode(const unsigned (&w)[2], float (&v)[8])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const auto pair = j & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(w[j >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8(w[j >> 1], false);
        v[2 * j] = pair[0];
        v[2 * j + 1] = pair[1];
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
__global__ __launch_bounds__(NT, BITS8 ? 5 : 4) void adamw_kernel(Args a)
{
    __shared__ float shared[2];
    const int tid = threadIdx.x;
    // the tensor: the last that begins at or before this workgroup, 64 of them looked at in a step
    const int lane = tid & 63;
    int ti = 0;
    for (int span = a.tensors; span > 1;) {
        const int each = (span + 63) >> 6;
        const int i = lane * each;
        const int n = __popcll(__ballot(i < span && a.first[ti + (i < span ? i : 0)] <= blockIdx.x)) - 1;
        ti += n * each;
        span = min(each, span - n * each);
    }
    ti = __builtin_amdgcn_readfirstlane(ti);
    const obc_adamw_tensor t = a.t[ti];
    const int64_t at = (int64_t)(blockIdx.x - a.first[ti]) * kChunk + tid * E, left64 = t.n - at;
    const int left = left64 < 0 ? 0 : left64 > E ? E : (int)left64;
    const bool master = t.master != nullptr;
    const bool past = (int64_t)gridDim.x * kChunk * 8 > kCaches;      // (8 bytes are written for an element, or more)

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
    const bool skip = !(fabsf(gs) < __builtin_inff()) || (a.step && step < 1);
    if (a.step && step < 1 && blockIdx.x == 0 && tid == 0) obc_latch(a.status, OBC_ERR_BAD_ARG);
    const float keep = (float)(1.0 - (double)lr * (double)t.decay), rate = lr * c1;
    const float gm = (float)(gs * (1.0 - a.beta1)), gv = (float)(gs * a.root_n2), b1 = (float)a.beta1, b2 = (float)a.beta2;
    float root[8];
    if (BITS8) {
        decode(m8, m);
        decode(v8, root);
    }
    if (!skip) {
        const float sm = m_scale * b1, sv = v_scale * (float)a.root_b2;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float x = g[j] * gv;
            m[j] = fmaf(g[j], gm, m[j] * (BITS8 ? sm : b1));
            if (BITS8) {
                root[j] *= sv;
                v[j] = fmaf(root[j], root[j], x * x);
            } else {
                v[j] = fmaf(v[j], b2, x * x);
            }
        }
        if (BITS8) {
            // Roots down to fp32's least, though their squares are none of its numbers from about 1e-19 on: such ones (zeros too) are formed
            // from squares that are larger by 2^128, which their wave alone pays for.
            float least = v[0];
#pragma unroll
            for (int j = 1; j < 8; ++j) least = fminf(least, v[j]);
            if (__any(least < kSmall)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = g[j] * gv * 0x1p64f, old = root[j] * 0x1p64f;
                    root[j] = v[j] < kSmall ? __builtin_amdgcn_sqrtf(fmaf(old, old, x * x)) * 0x1p-64f : __builtin_amdgcn_sqrtf(v[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) root[j] = __builtin_amdgcn_sqrtf(v[j]);      // (to a unit in the last place)
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {      // (the instruction takes a v below 2^-126 for zero)
                const bool small = v[j] < kSmall;
                root[j] = __builtin_amdgcn_sqrtf(small ? v[j] * 0x1p64f : v[j]) * (small ? 0x1p-32f : 1.f);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = fmaf(p[j], keep, -rate * m[j] * __builtin_amdgcn_rcpf(fmaf(root[j], c2, a.eps)));
    }
    if (skip && master) {      // the parameters as they were, which need not be the copies rounded (read before the copies are written)
        if (left > 0) {
            float old[8];
            load8<TYPE>(t.p, at, left, old);
            put8<OBC_F32>(t.master_out, at, left, p, past);
            put8<TYPE>(t.p_out, at, left, old, past);
        }
    } else if (left > 0) {
        if (master) put8<OBC_F32>(t.master_out, at, left, p, past);
        put8<TYPE>(t.p_out, at, left, p, past);
    }
    if (!BITS8) {
        if (left > 0) {
            put8<OBC_F32>(t.m_out, at, left, m, past);
            put8<OBC_F32>(t.v_out, at, left, v, past);
        }
        return;
    }
    if (!skip) {
        // the largest magnitudes, by their bits: a NaN is larger than an infinity, that than any number.  (Beyond the end all are zero.)
        unsigned bits_m = 0u, bits_v = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            bits_m = max(bits_m, __builtin_bit_cast(unsigned, m[j]) & 0x7fffffffu);
            bits_v = max(bits_v, __builtin_bit_cast(unsigned, root[j]) & 0x7fffffffu);
        }
        const float top_m = __builtin_bit_cast(float, over_block(bits_m)), top_v = __builtin_bit_cast(float, over_block(bits_v));
        // (a block whose largest number is next to nothing, below 1e-30, is taken for zeros: its reciprocal would not be finite)
        const bool lost_m = !(top_m < __builtin_inff()), lost_v = !(top_v < __builtin_inff());
        const bool any_m = !lost_m && top_m > 1e-30f, any_v = !lost_v && top_v > 1e-30f;
        const float up_m = any_m ? kTop8 / top_m : 0.f, up_v = any_v ? kTop8 / top_v : 0.f;
        const float old_m = m_scale, old_v = v_scale;
        m_scale = lost_m ? __builtin_nanf("") : any_m ? top_m / kTop8 : 0.f;
        v_scale = lost_v ? __builtin_nanf("") : any_v ? top_v / kTop8 : 0.f;
        const unsigned base = key + (unsigned)ti * 0x3C6EF373u + (unsigned)((uint64_t)at >> 32) * 0x243F6A89u;
        unsigned edge = ~0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned u = mix(((unsigned)at + j) ^ base);
            const float am = fminf(fabsf(m[j]) * up_m, kTop8), av = fminf(root[j] * up_v, kTop8);
            m[j] = copysignf(on_grid(am, u << 16 >> 12, edge), m[j]);
            root[j] = fmaxf(on_grid(av, u >> 16 << 4, edge), av > 0.f ? 0x1p-9f : 0.f);
        }
        // Where a number lies so near to where the dither turns that fp32's roundings would decide (moments are off by a few halves
        // of their last place, mostly), the wave, one in eighty, does it all again in 64 bits: results are those of the
        // formula, not of an order of roundings.  (Not so a new m far smaller than its two terms, whose roundings are more of its last places than
        // that: a few of 16 million codes, small ones: 5e-8 of the norm of m.)
        if (__any(edge < 2 * kClose)) {
            // (one element after the other, the first of arrays that turn: in a loop that is not unrolled, so that the usual way needs no
            // registers for this one -- 119 with eight at once, at which a step of 64 million took 210 us instead of 165)
            auto again = [&](double &xm, double &xv) {
                const double x = (double)g[0] * gs, old = (double)__builtin_amdgcn_cvt_f32_fp8(v8[0], 0) * old_v;
                xm = (double)__builtin_amdgcn_cvt_f32_fp8(m8[0], 0) * old_m * a.beta1 + x * (1.0 - a.beta1);
                xv = old * old * a.beta2 + x * x * (1.0 - a.beta2);
                turn(g);
                turn_bytes(m8);
                turn_bytes(v8);
            };
            double tm = 0.0, tv = 0.0, xm, xv;
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
                again(xm, xv);
                if (j < left) {
                    tm = fmax(tm, fabs(xm));
                    tv = fmax(tv, xv);
                }
            }
            tm = over_block(tm) / (double)kTop8;
            tv = sqrt(over_block(tv)) / (double)kTop8;
            // (a block of zeros, or of what is not finite, stays as it is)
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
                again(xm, xv);
                const unsigned u = mix(((unsigned)at + j) ^ base);
                if (any_m) m[0] = copysignf((float)on_grid(fmin(fabs(xm) / tm, (double)kTop8), u & 0xffffu), (float)xm);
                if (any_v) {
                    root[0] = (float)on_grid(fmin(sqrt(xv) / tv, (double)kTop8), u >> 16);
                    if (xv > 0.0) root[0] = fmaxf(root[0], 0x1p-9f);
                }
                turn(m);
                turn(root);
            }
        }
        encode(m, m8);
        encode(root, v8);
        if (!any_m) m8[0] = m8[1] = 0u;
        if (!any_v) v8[0] = v8[1] = 0u;
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

// Memory that a step writes, for the check that no two arrays share any
struct Span {
    uintptr_t from, to;
    int tensor;
};
inline void put_span(Span *spans, int64_t &n, int tensor, const void *p, int64_t bytes)
{
    if (p && bytes > 0) spans[n++] = Span{(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, tensor};
}
// Whether an input is apart from all outputs (sorted, apart from each other), or is one of its own tensor's, element for element: a thread reads
// all inputs of its elements before it writes any.  `out`: its own output, if it has one.
inline bool apart(const Span *spans, int64_t n, int tensor, const void *in, const void *out, int64_t bytes)
{
    if (!in || bytes == 0 || in == out) return true;
    const uintptr_t from = (uintptr_t)in, to = from + (uintptr_t)bytes;
    for (const Span *s = std::lower_bound(spans, spans + n, from, [](const Span &x, uintptr_t f) { return x.to <= f; }); s < spans + n && s->from < to; ++s)
        if (s->tensor != tensor || s->from != from || s->to != to) return false;
    return true;
}

}  // namespace

extern "C" {

int obc_adamw_plan_bytes(int count, size_t *bytes)
{
    if (!bytes || count < 0) return OBC_ERR_BAD_ARG;
    *bytes = layout_of(count).bytes;
    return OBC_OK;
}

int obc_adamw_plan(obc_ctx *ctx, const obc_adamw_tensor *tensors, int count, int type, int bits, void *plan, int64_t *workgroups)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (count < 0 || !workgroups || (count > 0 && (!tensors || !plan))) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw_plan: null argument");
    if (!float_type(type) || (bits != 8 && bits != 32)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw_plan: type %d, moments of %d bits", type, bits);
    if (((uintptr_t)plan & 15) != 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw_plan: the plan is not aligned to 16 bytes");
    const size_t e = size_of_type(type) - 1;
    int64_t blocks = 0;
    for (int i = 0; i < count; ++i) {
        const obc_adamw_tensor &t = tensors[i];
        if (t.n < 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw_plan: tensor %d: bad size", i);
        if (!(fabsf(t.decay) < __builtin_inff())) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw_plan: tensor %d: decay is not finite", i);
        if (t.n == 0) continue;
        if (!t.p || !t.p_out || !t.g || !t.m || !t.m_out || !t.v || !t.v_out || (t.master == nullptr) != (t.master_out == nullptr))
            return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw_plan: tensor %d: null argument", i);
        if (bits == 8 && (!t.m_scale || !t.m_scale_out || !t.v_scale || !t.v_scale_out))
            return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw_plan: tensor %d: moments of 8 bits have scales", i);
        const uintptr_t words = (uintptr_t)t.master | (uintptr_t)t.master_out |
                                (bits == 8 ? (uintptr_t)t.m_scale | (uintptr_t)t.m_scale_out | (uintptr_t)t.v_scale | (uintptr_t)t.v_scale_out
                                           : (uintptr_t)t.m | (uintptr_t)t.m_out | (uintptr_t)t.v | (uintptr_t)t.v_out);
        if (((((uintptr_t)t.p | (uintptr_t)t.p_out | (uintptr_t)t.g) & e) | (words & 3)) != 0)
            return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw_plan: tensor %d: an array is not aligned to its elements", i);
        const int64_t more = t.n / kChunk + (t.n % kChunk != 0);
        if (more > kMostBlocks - blocks) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_adamw_plan: more elements than a launch takes");
        blocks += more;
    }
    Span *const spans = new (std::nothrow) Span[(size_t)count * 6 + 1];
    if (!spans) return obc_fail(ctx, OBC_ERR_HIP, "obc_adamw_plan: no host memory");
    int64_t written = 0;
    const auto sizes = [&](const obc_adamw_tensor &t, int64_t &p, int64_t &m, int64_t &s) {
        p = t.n * (int64_t)size_of_type(type);
        m = t.n * (bits / 8);
        s = bits == 8 ? (t.n + kScaled - 1) / kScaled * 4 : 0;
    };
    int64_t p, m, s;
    for (int i = 0; i < count; ++i) {
        const obc_adamw_tensor &t = tensors[i];
        if (t.n == 0) continue;
        sizes(t, p, m, s);
        put_span(spans, written, i, t.p_out, p);
        put_span(spans, written, i, t.m_out, m);
        put_span(spans, written, i, t.v_out, m);
        put_span(spans, written, i, t.master_out, 4 * t.n);
        put_span(spans, written, i, t.m_scale_out, s);
        put_span(spans, written, i, t.v_scale_out, s);
    }
    std::sort(spans, spans + written, [](const Span &a, const Span &b) { return a.from < b.from; });
    bool shared = false;
    for (int64_t i = 1; i < written; ++i) shared |= spans[i].from < spans[i - 1].to;
    int over = -1;
    for (int i = 0; i < count && !shared && over < 0; ++i) {
        const obc_adamw_tensor &t = tensors[i];
        if (t.n == 0) continue;
        sizes(t, p, m, s);
        const auto clear = [&](const void *in, const void *out, int64_t bytes) { return apart(spans, written, i, in, out, bytes); };
        if (!clear(t.p, t.p_out, p) || !clear(t.g, nullptr, p) || !clear(t.m, t.m_out, m) || !clear(t.v, t.v_out, m) ||
            !clear(t.master, t.master_out, 4 * t.n) || !clear(t.m_scale, t.m_scale_out, s) || !clear(t.v_scale, t.v_scale_out, s))
            over = i;
    }
    delete[] spans;
    if (shared) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw_plan: two outputs overlap (is a tensor listed twice?)");
    if (over >= 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw_plan: tensor %d: an input overlaps an output that is not these elements", over);
    *workgroups = blocks;
    unsigned first = 0;
    for (int i = 0; i < count; i += kWritten) {
        PlanArgs a;
        a.tensors = count - i < kWritten ? count - i : kWritten;
        a.to = (obc_adamw_tensor *)plan + i;
        a.first_to = (unsigned *)((char *)plan + layout_of(count).first) + i;
        for (int j = 0; j < a.tensors; ++j) {
            a.t[j] = tensors[i + j];
            a.first[j] = first;
            first += (unsigned)(a.t[j].n / kChunk + (a.t[j].n % kChunk != 0));
        }
        adamw_plan_kernel<<<1, 64, 0, ctx->stream>>>(a);
        OBC_LAUNCH_CHECK(ctx, "adamw_plan_kernel");
    }
    return OBC_OK;
}

int obc_adamw(obc_ctx *ctx, const void *plan, int count, int64_t workgroups, int type, int bits, int64_t step, const int64_t *step_at, float lr,
              const float *lr_at, double beta1, double beta2, float eps, const float *grad_scale, uint32_t seed)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (count < 0 || workgroups < 0 || workgroups > kMostBlocks || (workgroups > 0 && count == 0))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: not a plan's numbers");
    if (!float_type(type) || (bits != 8 && bits != 32)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: type %d, moments of %d bits", type, bits);
    if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: betas are in [0, 1)");
    if (!(eps >= 0x1p-120f && eps < __builtin_inff())) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: eps is not in [2^-120, inf)");
    if (!step_at && step < 1) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: steps count from 1");
    if (!lr_at && !(fabsf(lr) < __builtin_inff())) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: lr is not finite");
    if ((((uintptr_t)step_at) & 7) != 0 || (((uintptr_t)lr_at | (uintptr_t)grad_scale) & 3) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: step_at, lr_at or grad_scale is not aligned");
    if (workgroups == 0) return OBC_OK;
    if (!plan || ((uintptr_t)plan & 15) != 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_adamw: no plan");
    Args a;
    a.t = (const obc_adamw_tensor *)plan;
    a.first = (const unsigned *)((const char *)plan + layout_of(count).first);
    a.tensors = count;
    a.step = step_at;
    a.lr_at = lr_at;
    a.grad_scale = grad_scale;
    a.beta1 = beta1;
    a.beta2 = beta2;
    a.root_b2 = sqrt(beta2);
    a.root_n2 = sqrt(1.0 - beta2);
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
    if (type == OBC_F32) launch<OBC_F32>(ctx, a, (unsigned)workgroups, bits == 8);
    else if (type == OBC_F16) launch<OBC_F16>(ctx, a, (unsigned)workgroups, bits == 8);
    else launch<OBC_BF16>(ctx, a, (unsigned)workgroups, bits == 8);
    OBC_LAUNCH_CHECK(ctx, "adamw_kernel");
    return OBC_OK;
}

}  // extern "C"
