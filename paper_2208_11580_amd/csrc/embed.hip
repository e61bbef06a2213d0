// obc_embed and obc_embed_grad: rows of an embedding table for tokens' ids, and the table's gradient.
//
//   y[t] = scale table[ids[t]];   dtable[v] = scale sum over the tokens t with ids[t] = v of dy[t], in their order
// The gradient sorts the tokens by id first, without atomics on memory: a workgroup takes a slice of ids, looks through all tokens
// for its own, counts them per id and per wave, and so knows every one's place (tokens of lower ids are counted on the way).  Then
// a wave adds up the tokens of a table row in 2048 columns and writes the row, zeros where it has none.  Rows with more tokens than a
// stretch of the sorted ones holds are summed by stretches first, in parallel, and then over these.
#include "row_io.h"

namespace {

// ------------------------------------------------------------------------------------------------ lookup
struct LookupArgs {
    const void *table;
    const int32_t *ids;
    void *y;
    int V, d, T;
    int64_t ldt, ldy;
    float scale;
    int *status;
};

// Eight columns of a token to a thread; 2048 columns of a token to a workgroup
template <int TYPE, int YT>
__global__ __launch_bounds__(256) void embed_kernel(LookupArgs a)
{
    const int64_t t = blockIdx.x;
    const int c = (blockIdx.y * 256 + threadIdx.x) * 8, left = a.d - c;
    if (left <= 0) return;
    int id = a.ids[t];
    if (id >= a.V) {
        if (c == 0) obc_latch(a.status, OBC_ERR_BAD_ARG);
        id = -1;
    }
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
    if (id >= 0) load8<TYPE>(a.table, id * a.ldt + c, left, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = id >= 0 ? v[j] * a.scale : 0.f;
    store8<YT>(a.y, t * a.ldy + c, left, v);
}

// ------------------------------------------------------------------------------------------------ order
constexpr int kWaves = 16, kMostBins = 512;

struct SortArgs {
    const int32_t *ids;
    int32_t *start;      // V + 1: where each id's tokens begin in `order`
    int32_t *order;      // tokens by id, those of an id in their order
    int T, V, bins;      // ids of a slice: a power of two
    int *status;
};

__global__ __launch_bounds__(64 * kWaves) void embed_sort_kernel(SortArgs a)
{
    extern __shared__ int count[];                    // [kWaves][bins]
    __shared__ int below[kWaves], scan[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int lo = blockIdx.x * a.bins, hi = min(a.V, lo + a.bins) - lo;      // own ids: 0 <= id - lo < hi
    const int each = ((a.T + kWaves - 1) / kWaves + 63) / 64 * 64;
    const int64_t from = (int64_t)wave * each;
    const int to = (int)(from + each < a.T ? from + each : a.T);
    int *const own = count + wave * a.bins;
    for (int i = tid; i < kWaves * a.bins; i += 64 * kWaves) count[i] = 0;
    __syncthreads();
    int less = 0;
    bool bad = false;
    for (int64_t t0 = from; t0 < to; t0 += 256) {
        int id[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) id[i] = t0 + i * 64 + lane < to ? a.ids[t0 + i * 64 + lane] : -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            less += id[i] >= 0 && id[i] < lo;
            bad |= id[i] >= a.V;
            if ((unsigned)(id[i] - lo) < (unsigned)hi && id[i] >= 0) atomicAdd(&own[id[i] - lo], 1);
        }
    }
    if (blockIdx.x == 0 && bad) obc_latch(a.status, OBC_ERR_BAD_ARG);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) less += __shfl_xor(less, off, 64);
    if (lane == 0) below[wave] = less;
    __syncthreads();
    // thread b: id lo + b.  Its tokens in all waves, the ids' running sum, then where each wave's begin
    int sum = 0;
    if (tid < a.bins)
        for (int w = 0; w < kWaves; ++w) sum += count[w * a.bins + tid];
    int run = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(run, off, 64);
        if (lane >= off) run += o;
    }
    if (lane == 63) scan[wave] = run;
    __syncthreads();
    int at = run - sum;
    for (int w = 0; w < kWaves; ++w) at += below[w] + (w < wave ? scan[w] : 0);
    if (tid < hi) a.start[lo + tid] = at;
    if (tid == hi - 1 && lo + hi == a.V) a.start[a.V] = at + sum;
    if (tid < a.bins)
        for (int w = 0; w < kWaves; ++w) {
            const int n = count[w * a.bins + tid];
            count[w * a.bins + tid] = at;
            at += n;
        }
    __syncthreads();
    for (int64_t t0 = from; t0 < to; t0 += 64) {
        const int id = t0 + lane < to ? a.ids[t0 + lane] : -1;
        const bool mine = id >= 0 && (unsigned)(id - lo) < (unsigned)hi;
        unsigned long long same = __ballot(mine);
        if (same == 0) continue;
        // the lanes with this one's id
        const int b = id - lo;
        for (int bit = 1; bit < a.bins; bit <<= 1) {
            const unsigned long long has = __ballot(mine && (b & bit));
            same &= b & bit ? has : ~has;
        }
        if (!mine) same = 1ull << lane;
        const int first = __ffsll(same) - 1;
        int place = 0;
        if (mine && lane == first) place = atomicAdd(&own[b], __popcll(same));
        place = __shfl(place, first, 64) + __popcll(same & ((1ull << lane) - 1));
        if (mine) a.order[place] = (int)(t0 + lane);
    }
}

// ------------------------------------------------------------------------------------------------ sums
struct GradArgs {
    const int32_t *ids, *start, *order;
    const void *dy;
    void *dtable;
    float *part;         // per stretch: the sum of a row's tokens that go on from before it, and of one's that go on behind it
    int T, V, d, stretch;
    int64_t lddy, lddt;
    float scale;
    bool accumulate;
};

constexpr int kChunk = 512, kChunks = 4;      // columns of a wave's load, loads of a row

// The sum of the tokens order[from .. to) in the columns c0 + 512 i + 8 lane
template <int TYPE>
__device__ inline void add_tokens(const GradArgs &a, int from, int to, int c0, float (&acc)[kChunks][8])
{
    const int lane = threadIdx.x & 63;
    for (int n0 = from; n0 < to; n0 += 64) {
        const int mine = n0 + lane < to ? a.order[n0 + lane] : 0, n = min(64, to - n0);
#pragma unroll 2
        for (int i = 0; i < n; ++i) {
            const int64_t base = (int64_t)__builtin_amdgcn_readlane(mine, i) * a.lddy;
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                const int c = c0 + k * kChunk + lane * 8, left = a.d - c;
                if (left <= 0) continue;
                float v[8];
                load8<TYPE>(a.dy, base + c, left, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[k][j] += v[j];
            }
        }
    }
}

// The stretches' shares of rows with more than `stretch` tokens
template <int TYPE>
__global__ __launch_bounds__(64) void embed_stretch_kernel(GradArgs a)
{
    const int total = a.start[a.V], c0 = blockIdx.y * kChunk * kChunks;
    const int64_t from64 = (int64_t)blockIdx.x * a.stretch;
    if (from64 >= total) return;
    const int from = (int)from64, to = (int)min((int64_t)total, from64 + a.stretch);
    for (int half = 0; half < 2; ++half) {
        const int id = a.ids[a.order[half ? to - 1 : from]];
        const int s = a.start[id], e = a.start[id + 1];
        if (e - s <= a.stretch || (half && s <= from)) continue;
        float acc[kChunks][8] = {};
        add_tokens<TYPE>(a, max(s, from), min(e, to), c0, acc);
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
            const int c = c0 + k * kChunk + (threadIdx.x & 63) * 8, left = a.d - c;
            if (left > 0) store8<OBC_F32>(a.part, ((int64_t)blockIdx.x * 2 + half) * a.d + c, left, acc[k]);
        }
    }
}

// A table row in 2048 columns to a wave, four rows to a workgroup
template <int TYPE, int OT>
__global__ __launch_bounds__(256) void embed_grad_kernel(GradArgs a)
{
    const int lane = threadIdx.x & 63, c0 = blockIdx.y * kChunk * kChunks;
    const int64_t v = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (v >= a.V) return;
    const int s = a.start[v], e = a.start[v + 1];
    if (a.accumulate && s == e) return;
    float acc[kChunks][8] = {};
    if (e - s <= a.stretch) {
        add_tokens<TYPE>(a, s, e, c0, acc);
    } else {
        const int first = s / a.stretch, last = (e - 1) / a.stretch;
        for (int p = first; p <= last; ++p) {
            const int64_t base = ((int64_t)p * 2 + (p == first && s > p * a.stretch)) * a.d;
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                const int c = c0 + k * kChunk + lane * 8, left = a.d - c;
                if (left <= 0) continue;
                float x[8];
                load8<OBC_F32>(a.part, base + c, left, x);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[k][j] += x[j];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
        const int c = c0 + k * kChunk + lane * 8, left = a.d - c;
        if (left <= 0) continue;
        float old[8];
        if (a.accumulate) load8<OT>(a.dtable, v * a.lddt + c, left, old);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[k][j] = a.accumulate ? fmaf(acc[k][j], a.scale, old[j]) : s < e ? acc[k][j] * a.scale : 0.f;
        store8<OT>(a.dtable, v * a.lddt + c, left, acc[k]);
    }
}

inline int bins_of(int V)
{
    int bins = 64;
    while (bins < kMostBins && (int64_t)bins * 256 < V) bins *= 2;
    return bins;
}

// Tokens of a stretch: rows with more are summed in two steps
inline int stretch_of(int T)
{
    int n = 32;
    while ((int64_t)n * 512 < T) n *= 2;
    return n;
}

struct Plan {
    size_t start, order, part, bytes;
};

inline Plan plan_of(int T, int V, int d)
{
    Plan p;
    p.start = 0;
    p.order = obc_align_up(((size_t)V + 1) * 4, 256);
    p.part = p.order + obc_align_up((size_t)T * 4, 256);
    const int n = stretch_of(T);
    p.bytes = p.part + (T > n ? ((size_t)T + n - 1) / n * 2 * (size_t)d * 4 : 0);
    return p;
}

template <int TYPE, int YT>
void launch_lookup(obc_ctx *ctx, const LookupArgs &a)
{
    embed_kernel<TYPE, YT><<<dim3(a.T, (a.d + 2047) / 2048), 256, 0, ctx->stream>>>(a);
}

template <int TYPE>
void launch_lookup(obc_ctx *ctx, const LookupArgs &a, int y_type)
{
    if (y_type == OBC_F32) launch_lookup<TYPE, OBC_F32>(ctx, a);
    else if (y_type == OBC_F16) launch_lookup<TYPE, OBC_F16>(ctx, a);
    else launch_lookup<TYPE, OBC_BF16>(ctx, a);
}

template <int TYPE>
void launch_grad(obc_ctx *ctx, const GradArgs &a, int out_type)
{
    const unsigned chunks = (a.d + kChunk * kChunks - 1) / (kChunk * kChunks);
    if (a.T > a.stretch)
        embed_stretch_kernel<TYPE><<<dim3(((int64_t)a.T + a.stretch - 1) / a.stretch, chunks), 64, 0, ctx->stream>>>(a);
    const dim3 grid((unsigned)(((int64_t)a.V + 3) / 4), chunks);
    if (out_type == OBC_F32) embed_grad_kernel<TYPE, OBC_F32><<<grid, 256, 0, ctx->stream>>>(a);
    else if (out_type == OBC_F16) embed_grad_kernel<TYPE, OBC_F16><<<grid, 256, 0, ctx->stream>>>(a);
    else embed_grad_kernel<TYPE, OBC_BF16><<<grid, 256, 0, ctx->stream>>>(a);
}

constexpr int kMostCols = 1 << 20, kMostTokens = 1 << 30;

}  // namespace

extern "C" {

int obc_embed(obc_ctx *ctx, const void *table, int type, int V, int d, int64_t ldt, const int32_t *ids, int T, float scale, void *y,
              int y_type, int64_t ldy)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (T < 0 || V <= 0 || d <= 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_embed: bad size");
    if (d > kMostCols) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_embed: d (%d) > %d", d, kMostCols);
    if (!float_type(type) || !float_type(y_type)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_embed: type %d, y_type %d", type, y_type);
    if (ldt < d || ldy < d) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_embed: leading dimension below the row's length");
    if (T == 0) return OBC_OK;
    if (!table || !ids || !y) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_embed: null argument");
    if (((uintptr_t)table & (size_of_type(type) - 1)) != 0 || ((uintptr_t)y & (size_of_type(y_type) - 1)) != 0 || ((uintptr_t)ids & 3) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_embed: an array is not aligned to its elements");
    const int step = (1 << 23) / ((d + 2047) / 2048);      // tokens of a launch: below 2^32 threads
    for (int64_t t0 = 0; t0 < T; t0 += step) {
        const LookupArgs a = {table, ids + t0, (char *)y + t0 * ldy * (int64_t)size_of_type(y_type), V, d, T - t0 < step ? (int)(T - t0) : step, ldt, ldy,
                              scale, ctx->d_status};
        if (type == OBC_F32) launch_lookup<OBC_F32>(ctx, a, y_type);
        else if (type == OBC_F16) launch_lookup<OBC_F16>(ctx, a, y_type);
        else launch_lookup<OBC_BF16>(ctx, a, y_type);
        OBC_LAUNCH_CHECK(ctx, "embed_kernel");
    }
    return OBC_OK;
}

int obc_embed_grad_workspace_bytes(int T, int V, int d, size_t *bytes)
{
    if (!bytes || T < 0 || V <= 0 || d <= 0) return OBC_ERR_BAD_ARG;
    *bytes = plan_of(T, V, d).bytes;
    return OBC_OK;
}

int obc_embed_grad(obc_ctx *ctx, const int32_t *ids, int T, const void *dy, int type, int64_t lddy, float scale, int V, int d, int accumulate,
                   void *dtable, int dtable_type, int64_t lddt, void *ws, size_t ws_bytes)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (T < 0 || V <= 0 || d <= 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_embed_grad: bad size");
    if (d > kMostCols || T > kMostTokens)
        return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_embed_grad: d (%d) > %d or T (%d) > %d", d, kMostCols, T, kMostTokens);
    if (!float_type(type) || !float_type(dtable_type))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_embed_grad: type %d, dtable_type %d", type, dtable_type);
    if ((T > 0 && lddy < d) || lddt < d) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_embed_grad: leading dimension below the row's length");
    if (!dtable || (T > 0 && (!ids || !dy))) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_embed_grad: null argument");
    if ((T > 0 && (((uintptr_t)dy & (size_of_type(type) - 1)) != 0 || ((uintptr_t)ids & 3) != 0)) || ((uintptr_t)dtable & (size_of_type(dtable_type) - 1)) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_embed_grad: an array is not aligned to its elements");
    const int64_t chunks = (d + kChunk * kChunks - 1) / (kChunk * kChunks);
    if (!obc_grid_fits(((int64_t)V + 3) / 4 * chunks, 256)) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_embed_grad: too many table rows");
    const Plan p = plan_of(T, V, d);
    if (!ws || ((uintptr_t)ws & 15) != 0 || ws_bytes < p.bytes)
        return obc_fail(ctx, OBC_ERR_WORKSPACE, "obc_embed_grad: workspace of %zu bytes needed", p.bytes);
    int32_t *const start = (int32_t *)ws, *const order = (int32_t *)((char *)ws + p.order);
    const int bins = bins_of(V);
    const SortArgs sort = {ids, start, order, T, V, bins, ctx->d_status};
    embed_sort_kernel<<<(unsigned)(((int64_t)V + bins - 1) / bins), 64 * kWaves, (size_t)kWaves * bins * 4, ctx->stream>>>(sort);
    OBC_LAUNCH_CHECK(ctx, "embed_sort_kernel");
    const GradArgs a = {ids, start, order, dy, dtable, (float *)((char *)ws + p.part), T, V, d, stretch_of(T), lddy, lddt, scale, accumulate != 0};
    if (type == OBC_F32) launch_grad<OBC_F32>(ctx, a, dtable_type);
    else if (type == OBC_F16) launch_grad<OBC_F16>(ctx, a, dtable_type);
    else launch_grad<OBC_BF16>(ctx, a, dtable_type);
    OBC_LAUNCH_CHECK(ctx, "embed_grad_kernel");
    return OBC_OK;
}

}  // extern "C"
