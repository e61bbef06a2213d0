// obc_embed and obc_embed_grad: rows of an embedding table for tokens' ids, and the table's gradient.
//
//   y[t] = scale table[ids[t]];   dtable[v] = scale sum over the tokens t with ids[t] = v of dy[t], in their order
// The gradient sorts the tokens by id first, without atomics on memory: a workgroup takes a slice of ids, looks through all tokens
// for its own, counts them per id and per wave, and so knows every one's place (tokens of earlier slices are counted on the way).  Then
// waves add up the tokens of a table row, each in its columns, and write them, zeros where there is none.  Rows with more tokens than a
// stretch of the sorted ones holds are summed by stretches first, in parallel, and then over these.
//
// Memory-bound: the lookup of 16384 x 4096 in bf16 takes 31 us (188 MB, 6.1 TB/s: the table partly from the caches).  The gradient of
// 16384 x 4096 in bf16 into 32000 rows of fp32, 650 MB, takes 165 us with fresh inputs, 111 to 123 with inputs that the memory's cache holds:
// the order 9, the stretches 25, the rows 130 (4.7 TB/s; both in one launch 154, with 13 more for the long rows); of 100 x 768 in fp32
// into 5000 rows, 15 MB, 10.9 us in two dependent launches.
#include <type_traits>

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
    bool past;
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
    if (id >= 0) load8_of<TYPE>(a.table, id * a.ldt, c, a.d, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = id >= 0 ? v[j] * a.scale : 0.f;
    put8<YT>(a.y, t * a.ldy + c, left, v, a.past);
}

// ------------------------------------------------------------------------------------------------ order
constexpr int kWaves = 16, kBins = 512;
constexpr int kLoads = 8;        // of 64 tokens each, on their way at a time
constexpr int kPlaces = 16;      // 64 entries each of a wave's list

struct SortArgs {
    const int32_t *ids;
    intx2 *rows;         // V: where each id's tokens begin in `order`, and how many they are
    int32_t *order;      // tokens of an id next to one another, in their order
    int32_t *total;      // of all ids
    int T, V, slices;    // a power of two
    int *status;
};

// A token's place among those of its bin: adds the wave's tokens of each bin to that bin's counter, in the order of the lanes.
__device__ inline int place_in(int *counters, bool mine, int bin, int bins)
{
    const int lane = threadIdx.x & 63;
    const unsigned long long all = __ballot(mine);
    unsigned lo = (unsigned)all, hi = (unsigned)(all >> 32);      // the lanes with this one's bin
    for (int bit = 0; bins - 1 >> bit; ++bit) {
        const int has = (int)((unsigned)bin << (31 - bit)) >> 31;
        const unsigned long long set = __ballot(has < 0);
        lo &= ~((unsigned)set ^ has);
        hi &= ~((unsigned)(set >> 32) ^ has);
    }
    const int first = lo ? __ffs(lo) - 1 : 31 + __ffs(hi), before = __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0u));
    int place = 0;
    if (mine && lane == first) place = atomicAdd(&counters[bin], __popc(lo) + __popc(hi));
    return __shfl(place, first & 63, 64) + before;
}

// Workgroup s takes the ids s, s + slices, ... (so that frequent ids, which lie together, fall to different ones).  A wave takes a
// section of the tokens and lists its own ones first, since few are; mostly the list holds them all, and they are looked for once.
__global__ __launch_bounds__(64 * kWaves) void embed_sort_kernel(SortArgs a)
{
    __shared__ int count[kWaves][kBins];
    __shared__ unsigned listed[kWaves][64 * kPlaces];      // place in the section * kBins + bin
    __shared__ int below[kWaves], scan[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int slice = blockIdx.x, low = a.slices - 1, shift = __popc(low), bins = (a.V + low) >> shift;
    const int each = ((a.T + kWaves - 1) / kWaves + 63) / 64 * 64;
    const int64_t from = (int64_t)wave * each;
    const int64_t to = from + each < a.T ? from + each : a.T;
    int *const own = count[wave];
    unsigned *const list = listed[wave];
    int less = 0, n = 0;
    bool bad = false;
    int id[kLoads];
    auto load = [&](int64_t t0) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) id[i] = t0 + i * 64 + lane < to ? a.ids[t0 + i * 64 + lane] : -1;
    };
    // the wave's own tokens of those loaded, behind the list; the next ones' loads
    auto find = [&](int64_t t0) {
        int now[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) now[i] = id[i];
        load(t0 + 64 * kLoads);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            bad |= now[i] >= a.V;
            const bool real = (unsigned)now[i] < (unsigned)a.V;
            const int part = now[i] & low;
            less += real && part < slice;
            const unsigned long long mine = __ballot(real && part == slice);
            if (mine == 0) continue;
            const int at = n + __builtin_amdgcn_mbcnt_hi((unsigned)(mine >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mine, 0u));
            if (real && part == slice) list[at] = (unsigned)(t0 - from + i * 64 + lane) * kBins + (unsigned)(now[i] >> shift);
            n += __popcll(mine);
        }
    };
    int place[kPlaces];
    // places of the list's tokens among the wave's of their ids
    auto match = [&]() {
#pragma unroll
        for (int i = 0; i < kPlaces; ++i)
            if (i * 64 < n) {
                const bool mine = i * 64 + lane < n;
                place[i] = place_in(own, mine, mine ? (int)(list[i * 64 + lane] % kBins) : 0, bins);
            }
    };
    auto store = [&](bool kept) {
#pragma unroll
        for (int i = 0; i < kPlaces; ++i)
            if (i * 64 < n && i * 64 + lane < n) {
                const unsigned entry = list[i * 64 + lane];
                a.order[place[i] + (kept ? own[entry % kBins] : 0)] = (int)(from + entry / kBins);
            }
    };
    for (int i = lane; i < kBins; i += 64) own[i] = 0;
    bool kept = true;      // the list and the places in it are all of the wave's
    load(from);
    for (int64_t t0 = from; t0 < to; t0 += 64 * kLoads) {
        if (n > 64 * (kPlaces - kLoads)) {
            match();
            n = 0;
            kept = false;
        }
        find(t0);
    }
    match();
    if (slice == 0 && bad) obc_latch(a.status, OBC_ERR_BAD_ARG);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) less += __shfl_xor(less, off, 64);
    if (lane == 0) below[wave] = less;
    __syncthreads();
    // thread b: bin b.  Its tokens in all waves, the bins' running sum, then where each wave's begin
    int sum = 0, tokens[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        tokens[w] = tid < kBins ? count[w][tid] : 0;
        sum += tokens[w];
    }
    int run = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(run, off, 64);
        if (lane >= off) run += o;
    }
    if (lane == 63) scan[wave] = run;
    __syncthreads();
    int at = run - sum;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) at += below[w] + (w < wave ? scan[w] : 0);
    const int64_t row = ((int64_t)tid << shift) + slice;
    if (tid < bins && row < a.V) a.rows[row] = intx2{at, sum};
    if (slice == low && tid == kBins - 1) *a.total = at + sum;
    if (tid < kBins)
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            count[w][tid] = at;
            at += tokens[w];
        }
    __syncthreads();
    if (kept) return store(true);
    n = 0;
    load(from);
    for (int64_t t0 = from; t0 < to; t0 += 64 * kLoads) {
        if (n > 64 * (kPlaces - kLoads)) {
            match();
            store(false);
            n = 0;
        }
        find(t0);
    }
    match();
    store(false);
}

// ------------------------------------------------------------------------------------------------ sums
struct GradArgs {
    const int32_t *ids, *order, *total;
    const intx2 *rows;
    const void *dy;
    void *dtable;
    float *part;         // per stretch: the sum of a row's tokens that go on from before it, and of one's that go on behind it
    int T, V, d, stretch;
    int64_t lddy, lddt;
    float scale;
    bool accumulate;
    int wide;            // waves next to one another in a row: 1 << wide
    unsigned across;     // workgroups to a row
};

// Columns of a lane, 16 bytes of the wider of the two types: stores and loads of a wave's columns are whole lines
template <int TYPE, int OT>
constexpr int kCols = TYPE == OBC_F32 || OT == OBC_F32 ? 4 : 8;

// `N` columns of a row of d at column c as fp32, zeros beyond its end
template <int TYPE, int N>
__device__ inline void load_cols(const void *p, int64_t base, int c, int d, float (&v)[N])
{
    if (N == 8) {
        float w[8];
        load8_of<TYPE>(p, base, c, d, w);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = w[j];
    } else if (TYPE == OBC_F32) {
        unsigned w[4];
        load_words<OBC_F32>(p, base, c, d, 0u, w);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = __builtin_bit_cast(float, w[j & 3]);
    } else {
        const unsigned short *const row = (const unsigned short *)p + base;
        unsigned w[2] = {0u, 0u};
        if (d >= 4) {
            if (c < d) {
                const uintx2 x = *(const uintx2_at2 *)(row + (c + 4 <= d ? c : d - 4));
                w[0] = x.x;
                w[1] = x.y;
                if (c + 4 > d) move_words<true>(w, c + 4 - d, 0u);
            }
        } else {
            for (int j = 0; c + j < d; ++j) w[j >> 1] |= (unsigned)row[c + j] << (16 * (j & 1));
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const unsigned e = w[j >> 1 & 1];
            v[j] = TYPE == OBC_F16 ? (j & 1 ? half_hi(e) : half_lo(e)) : (j & 1 ? bf16_hi(e) : bf16_lo(e));
        }
    }
}

// (Past the caches: the table's gradient is not read again soon, dy is.)
template <int TYPE, int N>
__device__ inline void store_cols(void *p, int64_t at, int left, const float (&v)[N])
{
    if (left < N) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < left) store_as<TYPE>(p, at + j, v[j]);
    } else if (TYPE == OBC_F32) {
#pragma unroll
        for (int i = 0; i < N; i += 4) __builtin_nontemporal_store(floatx4{v[i], v[i + 1], v[i + 2], v[i + 3]}, (floatx4_at4 *)((float *)p + at + i));
    } else {
        unsigned w[N / 2];
#pragma unroll
        for (int j = 0; j < N / 2; ++j) w[j] = TYPE == OBC_F16 ? pair_f16(v[2 * j], v[2 * j + 1]) : pair_bf16(v[2 * j], v[2 * j + 1]);
        if (N == 8) __builtin_nontemporal_store(uintx4{w[0], w[1], w[2 % (N / 2)], w[3 % (N / 2)]}, (uintx4_at2 *)((unsigned short *)p + at));
        else __builtin_nontemporal_store(uintx2{w[0], w[1]}, (uintx2_at2 *)((unsigned short *)p + at));
    }
}

// The sum of the tokens order[from .. to) in the columns from c on, MANY tokens on their way at a time
template <int TYPE, int N, int MANY>
__device__ inline void add_tokens(const GradArgs &a, int from, int to, int c, float (&acc)[N])
{
    const int lane = threadIdx.x & 63, left = a.d - c;
    for (int n0 = from; n0 < to; n0 += 64) {
        const int mine = n0 + lane < to ? a.order[n0 + lane] : 0, n = min(64, to - n0);
        auto add = [&](int i0, auto many) {
            float v[many][N];
#pragma unroll
            for (int i = 0; i < many; ++i)
                if (left > 0) load_cols<TYPE, N>(a.dy, (int64_t)__builtin_amdgcn_readlane(mine, i0 + i) * a.lddy, c, a.d, v[i]);
#pragma unroll
            for (int i = 0; i < many; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) acc[j] += v[i][j];
        };
        int i = 0;
        for (; i + MANY <= n; i += MANY) add(i, std::integral_constant<int, MANY>());
        if (MANY > 8 && n & 8) { add(i, std::integral_constant<int, 8>()); i += 8; }
        if (n & 4) { add(i, std::integral_constant<int, 4>()); i += 4; }
        if (n & 2) { add(i, std::integral_constant<int, 2>()); i += 2; }
        if (n & 1) add(i, std::integral_constant<int, 1>());
    }
}

// The stretches' shares of rows with more than `stretch` tokens: 64 N columns of one to a wave
template <int TYPE>
__global__ __launch_bounds__(256) void embed_stretch_kernel(GradArgs a)
{
    constexpr int N = kCols<TYPE, OBC_F32>;
    const int c = (blockIdx.y * 256 + threadIdx.x) * N, left = a.d - c;
    const int total = *a.total;
    const int64_t from64 = (int64_t)(blockIdx.x >> 1) * a.stretch;
    const int half = blockIdx.x & 1;
    if (from64 >= total) return;
    const int from = (int)from64, to = (int)min((int64_t)total, from64 + a.stretch);
    const int id = a.ids[a.order[half ? to - 1 : from]];
    const intx2 own = a.rows[id];
    const int s = own.x, e = s + own.y;
    if (own.y <= a.stretch || (half && s <= from)) return;
    float acc[N] = {};
    add_tokens<TYPE, N, 8>(a, max(s, from), min(e, to), c, acc);
    if (left >= N) *(floatx4_at4 *)(a.part + (int64_t)blockIdx.x * a.d + c) = floatx4{acc[0], acc[1], acc[2], acc[3]};
    else
        for (int j = 0; j < N; ++j)
            if (j < left) a.part[(int64_t)blockIdx.x * a.d + c + j] = acc[j];
}

// 64 N columns of a table row to a wave; a workgroup's four waves lie next to one another in a row (or in two, or four, where rows are
// as short), and the workgroups of a row too: what is written at a time lies together.
template <int TYPE, int OT>
__global__ __launch_bounds__(256) void embed_grad_kernel(GradArgs a)
{
    constexpr int N = kCols<TYPE, OT>;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned group = blockIdx.x / a.across;      // of 4 >> a.wide rows
    const int c = (((blockIdx.x - group * a.across) << a.wide | (wave & ((1 << a.wide) - 1))) * 64 + (threadIdx.x & 63)) * N, left = a.d - c;
    const int64_t v = (int64_t)group * (4 >> a.wide) + (wave >> a.wide);
    if (v >= a.V || left + (int)(threadIdx.x & 63) * N <= 0) return;
    const intx2 own = a.rows[v];
    const int s = own.x, e = s + own.y;
    if (a.accumulate && s == e) return;
    float acc[N] = {};
    if (e - s <= a.stretch) {
        add_tokens<TYPE, N, 8>(a, s, e, c, acc);
    } else if (left > 0) {
        const int first = s / a.stretch, last = (e - 1) / a.stretch;
        load_cols<OBC_F32, N>(a.part, ((int64_t)first * 2 + (s > first * a.stretch)) * a.d, c, a.d, acc);
        for (int q = first + 1; q <= last; q += 8) {
            float x[8][N];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (q + i <= last) load_cols<OBC_F32, N>(a.part, (int64_t)(q + i) * 2 * a.d, c, a.d, x[i]);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (q + i <= last)
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[j] += x[i][j];
        }
    }
    if (left <= 0) return;
    float old[N] = {};
    if (a.accumulate) load_cols<OT, N>(a.dtable, v * a.lddt, c, a.d, old);
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = a.accumulate ? fmaf(acc[j], a.scale, old[j]) : s < e ? acc[j] * a.scale : 0.f;
    store_cols<OT, N>(a.dtable, v * a.lddt + c, left, acc);
}

// Workgroups that sort: one to a compute unit, or more where each would have more ids than it has counters for
inline int slices_of(int V)
{
    int n = 256;
    while ((int64_t)n * kBins < V) n *= 2;
    return n;
}

// Tokens of a stretch: rows with more are summed in two steps, in another launch, which a hundred tokens are not worth
inline int stretch_of(int T)
{
    int n = T <= 128 ? 128 : 32;
    while ((int64_t)n * 512 < T) n *= 2;
    return n;
}

struct Plan {
    size_t rows, order, part, bytes;      // (the total lies before the rows)
};

inline Plan plan_of(int T, int V, int d)
{
    Plan p;
    p.rows = 256;
    p.order = p.rows + obc_align_up((size_t)V * 8, 256);
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

struct RowGrid {
    int wide;
    unsigned across;
    int64_t blocks;
};

inline RowGrid row_grid(int V, int d, int type, int out_type)
{
    const int n = 64 * (type == OBC_F32 || out_type == OBC_F32 ? 4 : 8), waves = (d + n - 1) / n;
    RowGrid g;
    g.wide = waves > 2 ? 2 : waves > 1 ? 1 : 0;
    g.across = (unsigned)(waves + (1 << g.wide) - 1) >> g.wide;
    const int rows = 4 >> g.wide;
    g.blocks = ((int64_t)V + rows - 1) / rows * g.across;
    return g;
}

template <int TYPE>
void launch_grad(obc_ctx *ctx, GradArgs a, int out_type)
{
    if (a.T > a.stretch) {
        constexpr int N = kCols<TYPE, OBC_F32>;
        const dim3 grid((unsigned)(((int64_t)a.T + a.stretch - 1) / a.stretch * 2), (a.d + 256 * N - 1) / (256 * N));
        embed_stretch_kernel<TYPE><<<grid, 256, 0, ctx->stream>>>(a);
    }
    const RowGrid g = row_grid(a.V, a.d, TYPE, out_type);
    a.wide = g.wide;
    a.across = g.across;
    const unsigned grid = (unsigned)g.blocks;
    if (out_type == OBC_F32) embed_grad_kernel<TYPE, OBC_F32><<<grid, 256, 0, ctx->stream>>>(a);
    else if (out_type == OBC_F16) embed_grad_kernel<TYPE, OBC_F16><<<grid, 256, 0, ctx->stream>>>(a);
    else embed_grad_kernel<TYPE, OBC_BF16><<<grid, 256, 0, ctx->stream>>>(a);
}

constexpr int kMostCols = 1 << 20, kMostTokens = 1 << 26;

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
                              scale, ctx->d_status, (int64_t)T * d * (int64_t)size_of_type(y_type) > kCaches};
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
    if (!obc_grid_fits(row_grid(V, d, type, dtable_type).blocks, 256)) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_embed_grad: too many table rows");
    const Plan p = plan_of(T, V, d);
    if (!ws || ((uintptr_t)ws & 15) != 0 || ws_bytes < p.bytes)
        return obc_fail(ctx, OBC_ERR_WORKSPACE, "obc_embed_grad: workspace of %zu bytes needed", p.bytes);
    int32_t *const total = (int32_t *)ws, *const order = (int32_t *)((char *)ws + p.order);
    intx2 *const rows = (intx2 *)((char *)ws + p.rows);
    const int slices = slices_of(V);
    embed_sort_kernel<<<slices, 64 * kWaves, 0, ctx->stream>>>(SortArgs{ids, rows, order, total, T, V, slices, ctx->d_status});
    OBC_LAUNCH_CHECK(ctx, "embed_sort_kernel");
    const GradArgs a = {ids, order, total, rows, dy, dtable, (float *)((char *)ws + p.part), T, V, d, stretch_of(T), lddy, lddt, scale, accumulate != 0, 0, 1};
    if (type == OBC_F32) launch_grad<OBC_F32>(ctx, a, dtable_type);
    else if (type == OBC_F16) launch_grad<OBC_F16>(ctx, a, dtable_type);
    else launch_grad<OBC_BF16>(ctx, a, dtable_type);
    OBC_LAUNCH_CHECK(ctx, "embed_grad_kernel");
    return OBC_OK;
}

}  // extern "C"
