// obc_distill: a student's logits against a teacher's top logits, loss and gradient of a row in one go.
//
//   e[v] = exp((z[v] - max z) / tau), q[v] = e[v] / sum e;  log q[v] = (z[v] - max z) / tau - log sum e
//   loss = weight tau^2 sum_j p_j (log p_j - log q[i_j]);  dz[v] = weight tau (q[v] - sum_{j: i_j = v} p_j)
// Memory-bound: 2048 x 131072 in bf16 with its gradient, 1.07 GB, takes 260 us (4.1 TB/s; the plain copy kernel reaches 4.3 on a GB,
// the best copy 5.2): a workgroup of 1024 threads holds a row in its registers, one to a compute unit, so that loads and stores
// overlap only where a piece's gradient makes room for the next row's.  48 x 32000 in half precision takes 11 us: reductions one
// after the other, on 48 compute units.  Barriers that leave loads under way and stores past the caches changed nothing measurable (1 %).
//
// A row is read once and stays in registers; the teacher's entries are handled in fp32, and those that name the same
// token write the same value, so no order of writes changes the result.
#include "row_io.h"

namespace {

constexpr int kMaxEntries = 1024;
constexpr int CH = 16;          // 16-byte pieces of a row in a thread's registers

struct Args {
    const void *z;
    const int32_t *top_index;
    const float *top_logit, *weight;
    float *loss;
    void *dz;
    int T, V, k;
    int64_t ldz, lddz;
    float tau;
    int *status;
};

// N values reduced over a workgroup at a time, the first M by their maximum, the others by their sum; every thread gets
// them.  A buffer may be used again two reductions (of any buffers) later.
template <int NT, int M, int N>
__device__ inline void reduce(float (&v)[N], float (*buf)[N])
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float o = __shfl_xor(v[i], off, 64);
            v[i] = i < M ? fmaxf(v[i], o) : v[i] + o;
        }
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) buf[threadIdx.x >> 6][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = buf[threadIdx.x % (NT / 64)][i];
#pragma unroll
        for (int off = NT / 128; off > 0; off >>= 1) {
            const float o = __shfl_xor(v[i], off, 64);
            v[i] = i < M ? fmaxf(v[i], o) : v[i] + o;
        }
    }
}

// A workgroup's teacher entries: up to 1024 / NT to a thread.
template <int TYPE, int NT>
struct Teacher {
    static constexpr int N = kMaxEntries / NT;
    int index[N];
    float logit[N], z[N], p[N];

    __device__ void load(const Args &a, int64_t row)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int j = i * NT + threadIdx.x;
            index[i] = -1;
            logit[i] = -__builtin_inff();
            z[i] = 0.f;
            if (j < a.k) {
                index[i] = a.top_index[row * a.k + j];
                logit[i] = a.top_logit[row * a.k + j];
            }
            if (index[i] >= a.V) {
                obc_latch(a.status, OBC_ERR_BAD_ARG);
                index[i] = -1;
            }
            if (index[i] < 0 || logit[i] == -__builtin_inff()) {
                index[i] = -1;
                logit[i] = -__builtin_inff();
            }
            if (index[i] >= 0) z[i] = load_as<TYPE>(a.z, row * a.ldz + index[i]);
        }
    }
    __device__ float top() const
    {
        float t = logit[0];
#pragma unroll
        for (int i = 1; i < N; ++i) t = fmaxf(t, logit[i]);
        return t;
    }
    __device__ bool any() const
    {
        bool b = index[0] >= 0;
#pragma unroll
        for (int i = 1; i < N; ++i) b |= index[i] >= 0;
        return b;
    }
    __device__ float exps(float tmax, float inv)
    {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            p[i] = index[i] >= 0 ? expf((logit[i] - tmax) * inv) : 0.f;
            s += p[i];
        }
        return s;
    }
    // normalises p, turns z into (z - top) / tau, and returns this thread's share of the divergence
    __device__ float terms(float tmax, float esum, float top, float sum, float inv)
    {
        const float ln_e = logf(esum), ln_s = logf(sum);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (index[i] < 0) continue;
            p[i] = p[i] / esum;
            z[i] = (z[i] - top) * inv;
            // (a probability that underflows adds nothing, however unlikely the student holds the token)
            if (p[i] != 0.f) s += p[i] * (((logit[i] - tmax) * inv - ln_e) - (z[i] - ln_s));
        }
        return s;
    }
    __device__ void publish(int *is, float *ps) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            is[i * NT + threadIdx.x] = index[i];
            ps[i * NT + threadIdx.x] = p[i];
        }
    }
    // the named tokens' gradients, over what the row's pass wrote; alike entries write alike values
    __device__ void patch(const Args &a, int64_t row, const int *is, const float *ps, float g, float scale) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (index[i] < 0) continue;
            float all = 0.f;
            for (int j = 0; j < a.k; j += 8) {      // (what lies behind the last entry names no token)
                const intx4 i0 = *(const intx4 *)(is + j), i1 = *(const intx4 *)(is + j + 4);
                const floatx4 p0 = *(const floatx4 *)(ps + j), p1 = *(const floatx4 *)(ps + j + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) all += i0[e] == index[i] ? p0[e] : 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) all += i1[e] == index[i] ? p1[e] : 0.f;
            }
            store_as<TYPE>(a.dz, row * a.lddz + index[i], g * (__expf(z[i]) * scale - all));
        }
    }
};

// Rows of at most NT * CH pieces, in registers between the reductions and the gradient.  Workgroups stay and take every
// gridDim.x-th row: as a piece's gradient goes out, the next row's piece comes in its place.
template <int TYPE, int NT>
__global__ __launch_bounds__(NT, 1024 / NT * NT / 256) void distill_kernel(Args a)
{
    constexpr int E = Piece<TYPE>::E;
    __shared__ float buf1[NT / 64][3], buf2[NT / 64][2], buf3[NT / 64];
    __shared__ __align__(16) float ps[kMaxEntries];
    __shared__ __align__(16) int is[kMaxEntries];
    const int tid = threadIdx.x;
    const float inv = 1.f / a.tau;
    // exp((z - top) / tau) = 2^((z - top) c)
    const float c2 = 1.44269504088896f / a.tau;
    // pieces 0 .. whole - 1 are whole in every thread; the row ends inside the next one, x[CH] wherever that is
    const int whole = a.V / (NT * E), end = (whole * NT + tid) * E;
    Piece<TYPE> x[CH + 1];
    auto first = (const char *)a.z + blockIdx.x * a.ldz * (16 / E);
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (i < whole) x[i].load(first, (i * NT + tid) * E);
    x[CH].load_end(first, end, a.V);
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
        // (not known to be the same in every turn, or the compiler keeps sixteen offsets in registers)
        int me = tid;
        asm volatile("" : "+v"(me));
        const int ahead = row + gridDim.x < a.T ? whole : 0;
        char *const to = (char *)a.dz + row * a.lddz * (16 / E);
        const char *const after = (const char *)a.z + (row + gridDim.x < a.T ? row + gridDim.x : row) * a.ldz * (16 / E);
        const float weight = a.weight ? a.weight[row] : 1.f;
        Teacher<TYPE, NT> teacher;
        teacher.load(a, row);
        float v1[3] = {-__builtin_inff(), teacher.top(), teacher.any() ? 1.f : 0.f};
#pragma unroll
        for (int i = 0; i <= CH; ++i)
            if (i < whole || i == CH)
#pragma unroll
                for (int j = 0; j < E; ++j) v1[0] = fmaxf(v1[0], x[i][j]);
        reduce<NT, 3>(v1, buf1);
        const float top = v1[0], tmax = v1[1];
        const bool counts = v1[2] > 0.f && weight != 0.f;
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i <= CH; ++i)
            if (i < whole || i == CH) {
                x[i].forget();
#pragma unroll
                for (int j = 0; j < E; ++j) part[j & 1] += __builtin_amdgcn_exp2f((x[i][j] - top) * c2);
            }
        float v2[2] = {part[0] + part[1], teacher.exps(tmax, inv)};
        reduce<NT, 0>(v2, buf2);
        const float sum = v2[0], scale = 1.f / sum, g = counts ? weight * a.tau : 0.f;
        float term = teacher.terms(tmax, v2[1], top, sum, inv);
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) term += __shfl_xor(term, off, 64);
        if ((tid & 63) == 0) buf3[tid >> 6] = term;
        teacher.publish(is, ps);
        const float gs = g * scale;
        auto gradient = [&](Piece<TYPE> &p, float (&d)[E]) {
            p.forget();
#pragma unroll
            for (int j = 0; j < E; ++j) d[j] = counts ? gs * __builtin_amdgcn_exp2f((p[j] - top) * c2) : 0.f;
        };
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (i < whole) {
                const int c = (i * NT + me) * E;
                if (a.dz) {
                    float d[E];
                    gradient(x[i], d);
                    Piece<TYPE>::store(to, c, d);
                }
                if (i < ahead) x[i].load(after, c);
            }
        if (a.dz) {
            float d[E];
            gradient(x[CH], d);
            Piece<TYPE>::store_end(to, end, a.V, d);
        }
        if (row + gridDim.x < a.T) x[CH].load_end(after, end, a.V);
        __syncthreads();
        if (tid == 0) {
            float s = buf3[0];
#pragma unroll
            for (int w = 1; w < NT / 64; ++w) s += buf3[w];
            a.loss[row] = counts ? weight * a.tau * a.tau * s : 0.f;
        }
        if (a.dz && counts) teacher.patch(a, row, is, ps, g, scale);
    }
}

// Longer rows, read a second time for the gradient (rows that fit take 287 us this way against 261, 2048 x 131072 in bf16).
template <int TYPE>
__global__ __launch_bounds__(1024) void distill_long_kernel(Args a)
{
    constexpr int NT = 1024, E = Piece<TYPE>::E;
    __shared__ float buf1[NT / 64][3], buf2[NT / 64][2], buf3[NT / 64];
    __shared__ __align__(16) float ps[kMaxEntries];
    __shared__ __align__(16) int is[kMaxEntries];
    const int64_t row = blockIdx.x;
    const char *const z = (const char *)a.z + row * a.ldz * (16 / E);
    char *const to = (char *)a.dz + row * a.lddz * (16 / E);
    const int tid = threadIdx.x;
    const float inv = 1.f / a.tau, c2 = 1.44269504088896f / a.tau;
    const float weight = a.weight ? a.weight[row] : 1.f;
    Teacher<TYPE, NT> teacher;
    teacher.load(a, row);
    auto left = [&](int64_t c) { return (int)(a.V - c); };
    // each thread's running maximum and sum
    float top = -__builtin_inff(), sum = 0.f;
    for (int64_t c = tid * E; c < a.V; c += NT * E) {
        Piece<TYPE> x;
        x.load_end(z + c * (16 / E), 0, left(c));
        float t = top;
#pragma unroll
        for (int j = 0; j < E; ++j) t = fmaxf(t, x[j]);
        if (t > top) {
            sum *= __builtin_amdgcn_exp2f((top - t) * c2);
            top = t;
        }
        // (only -inf so far: nothing to add, and no difference to take)
        if (!(top == -__builtin_inff()))
#pragma unroll
            for (int j = 0; j < E; ++j) sum += __builtin_amdgcn_exp2f((x[j] - top) * c2);
        else
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (!(x[j] == x[j])) sum = x[j];
    }
    float v1[3] = {top, teacher.top(), teacher.any() ? 1.f : 0.f};
    reduce<NT, 3>(v1, buf1);
    const float own = top;
    top = v1[0];
    const float tmax = v1[1];
    const bool counts = v1[2] > 0.f && weight != 0.f;
    float v2[2] = {own == -__builtin_inff() ? (top == own ? __builtin_nanf("") : sum) : sum * __builtin_amdgcn_exp2f((own - top) * c2),
                   teacher.exps(tmax, inv)};
    reduce<NT, 0>(v2, buf2);
    sum = v2[0];
    const float scale = 1.f / sum, g = counts ? weight * a.tau : 0.f;
    float term = teacher.terms(tmax, v2[1], top, sum, inv);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) term += __shfl_xor(term, off, 64);
    if ((tid & 63) == 0) buf3[tid >> 6] = term;
    teacher.publish(is, ps);
    if (a.dz)
        for (int64_t c = tid * E; c < a.V; c += NT * E) {
            Piece<TYPE> x;
            x.load_end(z + c * (16 / E), 0, left(c));
            float d[E];
#pragma unroll
            for (int j = 0; j < E; ++j) d[j] = counts ? g * scale * __builtin_amdgcn_exp2f((x[j] - top) * c2) : 0.f;
            Piece<TYPE>::store_end(to + c * (16 / E), 0, left(c), d);
        }
    __syncthreads();
    if (tid == 0) {
        float s = buf3[0];
#pragma unroll
        for (int w = 1; w < NT / 64; ++w) s += buf3[w];
        a.loss[row] = counts ? weight * a.tau * a.tau * s : 0.f;
    }
    if (a.dz && counts) teacher.patch(a, row, is, ps, g, scale);
}

template <int TYPE>
void launch(obc_ctx *ctx, const Args &a)
{
    constexpr int E = Piece<TYPE>::E;
    auto stay = [&](int per_cu) { return a.T < 256 * per_cu ? a.T : 256 * per_cu; };
    // The fewest threads that hold a row, so that several rows share a compute unit -- but, where there are fewer rows than compute
    // units, as many as have four pieces each (500 x 5000 in bf16: 12 us with 256 threads, 20 with 1024; 48 x 32000 in half
    // precision: 11.6 with 1024)
    const bool few = a.T <= 256;
    if ((int64_t)a.V > 1024 * CH * E) distill_long_kernel<TYPE><<<a.T, 1024, 0, ctx->stream>>>(a);
    else if (a.V > 512 * (few ? 4 : CH) * E) distill_kernel<TYPE, 1024><<<stay(1), 1024, 0, ctx->stream>>>(a);
    else if (a.V > 256 * (few ? 4 : CH) * E) distill_kernel<TYPE, 512><<<stay(2), 512, 0, ctx->stream>>>(a);
    else distill_kernel<TYPE, 256><<<stay(4), 256, 0, ctx->stream>>>(a);
}

}  // namespace

extern "C" {

int obc_distill(obc_ctx *ctx, const void *z, int type, int T, int V, int64_t ldz, const int32_t *top_index, const float *top_logit,
                int k, float temperature, const float *weight, float *loss, void *dz, int64_t lddz)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (T < 0 || V <= 0 || k < 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_distill: bad size");
    if (k > kMaxEntries) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_distill: k (%d) > %d", k, kMaxEntries);
    if (!float_type(type)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_distill: type %d is not a floating type", type);
    if (!(temperature > 0.f) || !(temperature < __builtin_inff()))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_distill: temperature is not positive and finite");
    if (ldz < V || (dz && lddz < V)) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_distill: leading dimension below the row's length");
    if (dz == z && dz && lddz != ldz) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_distill: dz == z with another leading dimension");
    if (T == 0) return OBC_OK;
    if (!z || !loss || (k > 0 && (!top_index || !top_logit))) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_distill: null argument");
    if ((((uintptr_t)z | (uintptr_t)dz) & (size_of_type(type) - 1)) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_distill: z or dz is not aligned to its elements");
    if (!obc_grid_fits(T, 1024)) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_distill: too many rows");
    const Args a = {z, top_index, top_logit, weight, loss, dz, T, V, k, ldz, lddz, temperature, ctx->d_status};
    if (type == OBC_F32) launch<OBC_F32>(ctx, a);
    else if (type == OBC_F16) launch<OBC_F16>(ctx, a);
    else launch<OBC_BF16>(ctx, a);
    OBC_LAUNCH_CHECK(ctx, "distill_kernel");
    return OBC_OK;
}

}  // extern "C"
