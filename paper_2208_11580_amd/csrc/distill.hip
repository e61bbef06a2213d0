// obc_distill: a student's logits against a teacher's top logits, loss and gradient of a row in one go.
//
//   e[v] = exp((z[v] - max z) / tau), q[v] = e[v] / sum e;  log q[v] = (z[v] - max z) / tau - log sum e
//   loss = weight tau^2 sum_j p_j (log p_j - log q[i_j]);  dz[v] = weight tau (q[v] - sum_{j: i_j = v} p_j)
// One workgroup to a row.  The teacher's entries, at most as many as threads, are handled in fp32 in LDS; entries that
// name the same token write the same value, so no order of writes changes the result.
#include "product4.h"

namespace {

constexpr int NT = 1024;

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

template <int TYPE>
__device__ inline float load_as(const void *p, int64_t at)
{
    return TYPE == OBC_F32 ? ((const float *)p)[at] : TYPE == OBC_F16 ? (float)((const _Float16 *)p)[at] : (float)((const __bf16 *)p)[at];
}

template <bool MAX>
__device__ inline float reduce(float v, float *buf)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const float o = __shfl_xor(v, off, 64);
        v = MAX ? fmaxf(v, o) : v + o;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    v = buf[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v = MAX ? fmaxf(v, buf[w]) : v + buf[w];
    return v;
}

template <int TYPE>
__global__ __launch_bounds__(NT) void distill_kernel(Args a)
{
    __shared__ float buf[NT / 64];
    __shared__ float ps[NT];
    __shared__ int is[NT];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x;
    const int64_t zat = row * a.ldz, gat = row * a.lddz;
    int index = -1;
    float t = -__builtin_inff();
    if (tid < a.k) {
        index = a.top_index[row * a.k + tid];
        if (index >= a.V) {
            obc_latch(a.status, OBC_ERR_BAD_ARG);
            index = -1;
        }
        if (index >= 0) t = a.top_logit[row * a.k + tid];
        if (t == -__builtin_inff()) index = -1;
    }
    const bool any = __syncthreads_or(index >= 0);
    const float weight = a.weight ? a.weight[row] : 1.f;
    if (!any || weight == 0.f) {
        if (tid == 0) a.loss[row] = 0.f;
        if (a.dz)
            for (int v = tid; v < a.V; v += NT) store_as<TYPE>(a.dz, gat + v, 0.f);
        return;
    }
    const float inv = 1.f / a.tau;
    float top = -__builtin_inff();
    for (int v = tid; v < a.V; v += NT) top = fmaxf(top, load_as<TYPE>(a.z, zat + v));
    top = reduce<true>(top, buf);
    float sum = 0.f;
    for (int v = tid; v < a.V; v += NT) sum += __expf((load_as<TYPE>(a.z, zat + v) - top) * inv);
    sum = reduce<false>(sum, buf);
    // the teacher
    const float tmax = reduce<true>(t, buf);
    const float e = index >= 0 ? expf((t - tmax) * inv) : 0.f;
    const float esum = reduce<false>(e, buf);
    const float p = e / esum;
    float zsel = 0.f, term = 0.f;
    if (index >= 0) {
        zsel = (load_as<TYPE>(a.z, zat + index) - top) * inv;
        if (p > 0.f) term = p * (((t - tmax) * inv - logf(esum)) - (zsel - logf(sum)));
        else if (!(p == 0.f)) term = p;
    }
    const float total = reduce<false>(term, buf);
    if (tid == 0) a.loss[row] = weight * a.tau * a.tau * total;
    if (!a.dz) return;
    is[tid] = index;
    ps[tid] = p;
    __syncthreads();
    const float g = weight * a.tau, scale = 1.f / sum;
    for (int v = tid; v < a.V; v += NT)
        store_as<TYPE>(a.dz, gat + v, g * (__expf((load_as<TYPE>(a.z, zat + v) - top) * inv) * scale));
    __syncthreads();
    if (index >= 0) {
        float ptot = 0.f;
        for (int j = 0; j < a.k; ++j) ptot += is[j] == index ? ps[j] : 0.f;
        store_as<TYPE>(a.dz, gat + index, g * (__expf(zsel) * scale - ptot));
    }
}

}  // namespace

extern "C" {

int obc_distill(obc_ctx *ctx, const void *z, int type, int T, int V, int64_t ldz, const int32_t *top_index, const float *top_logit,
                int k, float temperature, const float *weight, float *loss, void *dz, int64_t lddz)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (T < 0 || V <= 0 || k < 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_distill: bad size");
    if (k > NT) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_distill: k (%d) > %d", k, NT);
    if (!float_type(type)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_distill: type %d is not a floating type", type);
    if (!(temperature > 0.f) || !(temperature < __builtin_inff()))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_distill: temperature is not positive and finite");
    if (ldz < V || (dz && lddz < V)) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_distill: leading dimension below the row's length");
    if (dz == z && dz && lddz != ldz) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_distill: dz == z with another leading dimension");
    if (T == 0) return OBC_OK;
    if (!z || !loss || (k > 0 && (!top_index || !top_logit))) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_distill: null argument");
    if ((((uintptr_t)z | (uintptr_t)dz) & (size_of_type(type) - 1)) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_distill: z or dz is not aligned to its elements");
    const Args a = {z, top_index, top_logit, weight, loss, dz, T, V, k, ldz, lddz, temperature, ctx->d_status};
    if (type == OBC_F32) distill_kernel<OBC_F32><<<T, NT, 0, ctx->stream>>>(a);
    else if (type == OBC_F16) distill_kernel<OBC_F16><<<T, NT, 0, ctx->stream>>>(a);
    else distill_kernel<OBC_BF16><<<T, NT, 0, ctx->stream>>>(a);
    OBC_LAUNCH_CHECK(ctx, "distill_kernel");
    return OBC_OK;
}

}  // extern "C"
