// obc_score: log probabilities of given tokens, entropy and the largest logits of rows of logits.
//
//   d[v] = (z[v] - max z) / tau,  S = sum exp d,  D = sum exp(d) d:  lse = max z / tau + log S,  logp = d[target] - log S,
//   entropy = log S - D / S
// A workgroup reads its part of a row once, into registers: the maximum, then S and D (kept in powers and logarithms of 2).  The k
// largest come from the same registers: the r-th largest of each wave's lanes' own maxima, r waves = k, is a bound that at least k
// logits reach and few more do; those that do go to LDS as whole numbers (logit, then index) and are sorted there.  Where too many
// reach it (equal logits, mostly), the k-th largest is found exactly, by bisection, and equal ones are taken in their order.  Rows
// of several parts are joined by a second kernel.
//
// Bound by vector issue, with memory close behind: 2048 x 131072 in bf16 with 64 alternatives, 537 MB, takes 125 us a call (4.3 TB/s; plain reads
// reach 6.0).  Traced one by one the parts take 122 (1645 instructions a wave, half of them for the two sums; vector units active three
// quarters of the time) and the join 10; with half of each row at -inf a call takes 128.  One row of 32000 in fp32 with 20 alternatives takes 8.2 us
// in one launch, 5 without alternatives.  Workgroups that stay and load the next part as they sum this one took 154 us.
#include <type_traits>

#include "row_io.h"

namespace {

typedef unsigned long long Key;      // a logit's order above its index's opposite; 0: none

constexpr int kMaxTop = 1024, kMaxCols = 1 << 30;
constexpr float kLn2 = 0.693147180559945f;

struct Stats {
    float top, sum, dot, unused;
};

struct Args {
    const void *z;
    const int32_t *target;
    float *logp, *entropy, *lse;
    int32_t *top_index;
    float *top_logit;
    int T, V, k, parts, len;      // columns of a part
    int64_t ldz;
    float tau;
    Stats *stats;                 // per part, with parts > 1
    Key *lists;                   // k per part, largest first
    int *status;
};

// Numbers in the order of floats, and back.  Bits below SHIFT are the same for all of a type's positive numbers; a bound made from
// a shifted number lies between two of the type's (or on one), which is all that comparing with it needs.
__device__ inline unsigned ordered(float f)
{
    const unsigned b = __builtin_bit_cast(unsigned, f);
    return b ^ ((int)b >> 31 | 0x80000000u);
}
__device__ inline float unordered(unsigned o) { return __builtin_bit_cast(float, o & 0x80000000u ? o ^ 0x80000000u : ~o); }

template <int TYPE>
struct Order {
    static constexpr int SHIFT = TYPE == OBC_F32 ? 0 : TYPE == OBC_F16 ? 13 : 16;
    static __device__ unsigned of(float f) { return ordered(f) >> SHIFT; }
    static __device__ float bound(unsigned o) { return unordered(o << SHIFT); }
};

// A piece's element.  (Not Piece's own access: with that the half-precision pieces would live in memory.)
template <int TYPE>
__device__ inline float element(const Piece<TYPE> &p, int j)
{
    if (TYPE == OBC_F16) return (float)half_pair(p.v[j >> 1])[j & 1];
    return p[j];
}

__device__ inline float fmaxf_of(float a, float b) { return fmaxf(a, b); }

template <int NT, int N>
__device__ inline void block_sums(float (&v)[N], float (*buf)[N])
{
    constexpr int WAVES = NT / 64;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = sum_lanes(v[i]);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) buf[threadIdx.x >> 6][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = buf[0][i];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v[i] += buf[w][i];
    }
}

template <int NT>
__device__ inline int block_count(int n, int *buf)
{
    constexpr int WAVES = NT / 64;
    n = join_lanes(n, [](int a, int b) { return a + b; });
    __syncthreads();      // buf is read by all before it is written again
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = n;
    __syncthreads();
    n = buf[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) n += buf[w];
    return __builtin_amdgcn_readfirstlane(n);
}

__device__ inline Key key_of(float z, int index) { return (Key)ordered(z + 0.f) << 32 | ~(unsigned)index; }

// keys[0 .. n) in LDS, with room for the next power of two, largest first; all threads of the workgroup.  `out` gets the first k.
template <int NT, typename OUT>
__device__ inline void sort_keys(Key *keys, int n, int k, OUT out)
{
    const int tid = threadIdx.x;
    if (n <= (NT < 512 ? NT : 512)) {
        const Key own = tid < n ? keys[tid] : 0;
        int rank = 0;
        if (tid - (tid & 63) < n)
#pragma unroll 8
            for (int j = 0; j < n; ++j) rank += keys[j] > own;
        if (tid < n && rank < k) out(rank, own);
        return;
    }
    int size = 512;
    while (size < n) size *= 2;
    for (int i = n + tid; i < size; i += NT) keys[i] = 0;
    __syncthreads();
    for (int run = 2; run <= size; run *= 2)
        for (int gap = run / 2; gap > 0; gap /= 2) {
            for (int i = tid; i < size / 2; i += NT) {
                const int lo = 2 * i - (i & (gap - 1)), hi = lo + gap;
                const Key x = keys[lo], y = keys[hi];
                if ((x < y) == ((lo & run) == 0)) {
                    keys[lo] = y;
                    keys[hi] = x;
                }
            }
            __syncthreads();
        }
    for (int i = tid; i < n && i < k; i += NT) out(i, keys[i]);
}

// (a - b) c, where a - b may be beyond fp32's end
__device__ inline float difference(float a, float b, float c) { return 2.f * ((0.5f * a - 0.5f * b) * c); }

// The results of a row; one thread
__device__ inline void finish(const Args &a, int64_t row, float top, float sum, float dot, float zt, int target)
{
    // (an empty row: sum 0, top taken as 0)
    const bool none = sum == 0.f;
    const float ln = logf(sum);
    if (a.lse) a.lse[row] = none ? -__builtin_inff() : top / a.tau + ln;
    if (a.entropy) a.entropy[row] = none ? 0.f : fmaf(-kLn2, dot / sum, ln);
    if (a.logp) a.logp[row] = target < 0 ? 0.f : none ? -__builtin_inff() : 2.f * ((0.5f * zt - 0.5f * top) / a.tau) - ln;
}

__device__ inline int target_of(const Args &a, int64_t row)
{
    int t = a.target ? a.target[row] : -1;
    if (t >= a.V) {
        obc_latch(a.status, OBC_ERR_BAD_ARG);
        t = -1;
    }
    return t;
}

// Clears the mode's IEEE bit (the ninth): a maximum of a number and a NaN is the number then, whatever NaN it is.  With the bit set, a
// signalling NaN takes the number's place.
__device__ inline void drop_nans() { __builtin_amdgcn_s_setreg(1 | 9 << 6, 0); }

// The larger halves of two dwords.  bf16 numbers lie in the order of the half-precision ones of the same bits, up to 2^121; beyond
// (infinities too) those are NaNs, signalling ones up to 2^125, which this drops after drop_nans().
__device__ inline unsigned larger_halves(unsigned a, unsigned b)
{
    unsigned r;
    asm("v_pk_max_f16 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// PIECES: room for 16-byte pieces that hold a candidate, KEYS: for candidates (0 both: none are asked for)
template <int TYPE, int NT, int CH, int PIECES, int KEYS>
__global__ __launch_bounds__(NT, NT == 1024 || PIECES <= 512 ? 4 : 3) void score_kernel(Args a)
{
    constexpr int E = Piece<TYPE>::E, WAVES = NT / 64;
    typedef Order<TYPE> O;
    if (TYPE == OBC_BF16) drop_nans();
    __shared__ float buf1[WAVES], buf2[2][WAVES][2], buf3[WAVES];
    __shared__ int buf4[WAVES], found, queued;
    __shared__ __align__(16) uintx4 queue[PIECES + 1];
    __shared__ int queue_at[PIECES + 1];
    __shared__ Key keys[KEYS + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x / a.parts;
    const int part = (int)(blockIdx.x - row * a.parts), from = part * a.len, n = max(0, min(a.len, a.V - from));
    const char *const z = (const char *)a.z + (row * a.ldz + from) * (16 / E);
    const float c2 = 1.44269504088896f / a.tau;
    // pieces 0 .. whole - 1 are whole in every thread; the part ends inside the next one, x[CH] wherever that is
    const int whole = n / (NT * E);
    const bool tail = n > whole * NT * E;
    Piece<TYPE> x[CH + 1];
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (i < whole) x[i].load(z, (i * NT + tid) * E);
    if (tail) x[CH].load_end(z, (whole * NT + tid) * E, n);
    int target = -1;
    float zt = 0.f;
    if (a.parts == 1 && tid == NT - 64) {
        target = target_of(a, row);
        if (target >= 0) zt = load_as<TYPE>(a.z, row * a.ldz + target);
    }
    if (tid == 0) found = queued = 0;
    float most[CH + 1], s[2], top, bound;      // the largest of each piece
    float own = -__builtin_inff();
#pragma unroll
    for (int i = 0; i <= CH; ++i) {
        most[i] = -__builtin_inff();
        if (i < CH ? i < whole : tail) {
            if (TYPE != OBC_F32) {
                const uintx4 w = x[i].v;
                const unsigned m = larger_halves(larger_halves(w[0], w[1]), larger_halves(w[2], w[3]));
                most[i] = TYPE == OBC_F16 ? fmaxf(half_lo(m), half_hi(m)) : fmaxf(bf16_lo(m), bf16_hi(m));
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) most[i] = fmaxf(most[i], element(x[i], j));
            }
            own = fmaxf(own, most[i]);
        }
    }
    // the largest and the least of the lanes' largest
    const float wave_top = join_lanes(own, fmaxf_of), wave_low = KEYS > 0 ? join_lanes(own, [](float a, float b) { return fminf(a, b); }) : 0.f;
    // what at least r of this wave's lanes (or of their pieces) reach, and not many more
    bound = -__builtin_inff();
    if (KEYS > 0) {
        // waves with something in every lane; the others' candidates come on top
        const int live = min(WAVES, n / (64 * E)), r = live > 0 ? (a.k + live - 1) / live : 1 << 20;
        auto count = [&](float b) {
            if (r <= 32) return (int)__popcll(__ballot(own >= b));
            int c = 0;
#pragma unroll
            for (int i = 0; i <= CH; ++i)
                if (i < CH ? i < whole : tail) c += __popcll(__ballot(most[i] >= b));
            return c;
        };
        if (r <= 4) {
            // the largest taken away a few times
            float rest = own;
            bound = wave_top;
            for (int i = 1; i < r; ++i) {
                rest = lane == __ffsll(__ballot(rest == bound)) - 1 ? -__builtin_inff() : rest;
                bound = join_lanes(rest, fmaxf_of);
            }
        }
        unsigned lo = O::of(-__builtin_inff()) + 1, hi = __builtin_amdgcn_readfirstlane(O::of(wave_top));
        if (r > 4 && r <= 64 && wave_low > -__builtin_inff()) lo = __builtin_amdgcn_readfirstlane(O::of(wave_low));
        if (r > 4 && wave_top < __builtin_inff() && count(O::bound(lo)) >= r) {
            // halves of the values' range first, of the numbers' in between where that is slow
            for (int step = 0; lo < hi; ++step) {
                unsigned mid = lo + (hi - lo + 1) / 2;
                if (step < 8) mid = min(max(__builtin_amdgcn_readfirstlane(O::of(0.5f * O::bound(lo) + 0.5f * O::bound(hi))), lo + 1), hi);
                const int c = count(O::bound(mid));
                if (c >= r) lo = mid;
                else hi = mid - 1;
                if (c >= r && c <= r + (r >> 3) + 1) break;
            }
            bound = O::bound(lo);
        }
        if (live > 0 && wave >= live) bound = __builtin_inff();
    }
    if (lane == 0) {
        buf1[wave] = wave_top;
        buf3[wave] = bound;
    }
    __syncthreads();
    top = buf1[0];
    bound = buf3[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
        top = fmaxf(top, buf1[w]);
        bound = fminf(bound, buf3[w]);
    }
    float base = top == -__builtin_inff() ? 0.f : top;
    const float off = base * c2;
    s[0] = s[1] = 0.f;
#pragma unroll
    for (int i = 0; i <= CH; ++i)
        if (i < CH ? i < whole : tail) {
            x[i].forget();
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float d = fmaf(element(x[i], j), c2, -off), e = __builtin_amdgcn_exp2f(d);
                s[0] += e;
                s[1] = fmaf(e, fmaxf(d, -1e30f), s[1]);      // (a logit of -inf adds nothing)
            }
        }
    block_sums<NT, 2>(s, buf2[0]);
    // the product base c2 was rounded: all exponents are off by this, and the sums are brought back
    const float r = fmaf(base, c2, -off);
    {
        const float f = __builtin_amdgcn_exp2f(-r);
        s[1] = fmaf(-r, s[0], s[1]) * f;
        s[0] *= f;
    }
    // Numbers that these short ways do not know: once more, from the caches.  (Loops over the registers would take some from the usual way.)
    //  - The sums of NaN and infinities, and of a maximum of 2^24 temperatures or more, where r may be no small number: they lose the digits
    //    that r takes, and from 126 on the instruction's zero for results below 2^-126 makes f or the largest logit's exponential zero.
    //  - In bf16 the maximum, where it is none of the numbers in order, or one that the maxima dropped need not have made the sum infinite, at high
    //    temperatures; and the largest, where no more than the type's lowest may reach the bound.
    const int pieces = (n + NT * E - 1) / (NT * E);
    auto all = [&](auto f) {
#pragma unroll 4
        for (int i = 0; i < pieces; ++i) {
            Piece<TYPE> p;
            p.load_end(z, (i * NT + tid) * E, n);
            f(p, from + (i * NT + tid) * E);
        }
    };
    bool nothing = false;      // bf16: -inf alone, which the maxima do not tell from the type's lowest numbers
    if (TYPE == OBC_BF16 && top == -__builtin_inff()) {
        bool other = false;
#pragma unroll
        for (int i = 0; i <= CH; ++i)
            if (i < CH ? i < whole : tail)
#pragma unroll
                for (int j = 0; j < 4; ++j) other |= x[i].v[j] != 0xff80ff80u;
        nothing = block_count<NT>(other, buf4) == 0;
    }
    // whether the maximum is right, the bound too, and the sums
    const bool sure = TYPE != OBC_BF16 ? top < __builtin_inff() : nothing || (s[0] < __builtin_inff() && c2 > 0x1p-100f && fabsf(top) < 0x1p120f);
    bool ranked = sure && (TYPE != OBC_BF16 || KEYS == 0 || nothing || bound > -0x1p120f);
    if (!sure || !(s[0] < __builtin_inff()) || !(fabsf(r) <= 1.f)) {
        if (!sure) {
            const float quick = top;
            own = -__builtin_inff();
            all([&](const Piece<TYPE> &p, int) {
#pragma unroll
                for (int j = 0; j < E; ++j) own = fmaxf(own, element(p, j));
            });
            own = join_lanes(own, fmaxf_of);
            if (lane == 0) buf1[wave] = own;
            __syncthreads();
            top = buf1[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) top = fmaxf(top, buf1[w]);
            base = top == -__builtin_inff() ? 0.f : top;
            ranked = top == quick && fabsf(top) < 0x1p120f && bound > -0x1p120f;      // (fp32 and fp16: +inf, a lost row)
        }
        s[0] = s[1] = 0.f;
        all([&](const Piece<TYPE> &p, int) {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float d = difference(element(p, j), base, c2), e = __builtin_amdgcn_exp2f(d);
                s[0] += e;
                s[1] = fmaf(e, fmaxf(d, -1e30f), s[1]);
            }
        });
        block_sums<NT, 2>(s, buf2[1]);
    }
    if (tid == NT - 64) {      // (the last wave, which has the least to do with the largest)
        if (a.parts == 1) finish(a, row, base, s[0], s[1], zt, target);
        else a.stats[blockIdx.x] = Stats{base, s[0], s[1], 0.f};
    }
    if (KEYS == 0) return;

    // The logits that reach `b`, which is above -inf, go to LDS, as far as there is room: first the pieces that hold one, of which a
    // thread has few, then, piece by piece, they themselves.  Returns whether there was room.
    auto collect = [&](float b) {
        auto slots = [&](int *counter, int many) {      // the first of `many`, for the wave
            int first = 0;
            if (lane == 0) first = atomicAdd(counter, many);
            return __builtin_amdgcn_readfirstlane(first);
        };
        auto rank = [](unsigned long long m) { return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u)); };
        int many = 0;
#pragma unroll
        for (int i = 0; i <= CH; ++i)
            if (i < CH ? i < whole : tail) many += __popcll(__ballot(most[i] >= b));
        int at = slots(&queued, many);
#pragma unroll
        for (int i = 0; i <= CH; ++i)
            if (i < CH ? i < whole : tail) {
                const unsigned long long m = __ballot(most[i] >= b);
                if (m == 0) continue;
                const int to = at + rank(m);
                if (most[i] >= b && to < PIECES) {
                    queue[to] = x[i].v;
                    queue_at[to] = from + ((i == CH ? whole : i) * NT + tid) * E;
                }
                at += __popcll(m);
            }
        __syncthreads();
        const int pieces = min(queued, PIECES);
        for (int q0 = wave * 64; q0 < pieces; q0 += NT) {
            const int q = min(q0 + lane, pieces - 1);
            Piece<TYPE> p;
            p.v = queue[q];
            const int c = queue_at[q];
            const float least = q0 + lane < pieces ? b : __builtin_inff();      // (+inf is no candidate either: its row is lost)
            many = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) many += __popcll(__ballot(element(p, j) >= least));
            at = slots(&found, many);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const unsigned long long m = __ballot(element(p, j) >= least);
                const int to = at + rank(m);
                if (element(p, j) >= least && to < KEYS) keys[to] = key_of(element(p, j), c + j);
                at += __popcll(m);
            }
        }
        __syncthreads();
        return queued <= PIECES && found <= KEYS;
    };
    const float least = O::bound(O::of(-__builtin_inff()) + 1);      // above -inf
    const bool room = ranked && collect(fmaxf(bound, least));
    int have = found;
    __syncthreads();      // (found is set again below)
    if (!room) {
        // Exactly: the largest bound that k logits reach, those above it, and of those on it the first
        auto count = [&](float b) {
            int c = 0;
            all([&](const Piece<TYPE> &p, int) {
#pragma unroll
                for (int j = 0; j < E; ++j) c += element(p, j) >= b;
            });
            return block_count<NT>(c, buf4);
        };
        unsigned lo = __builtin_amdgcn_readfirstlane(O::of(ranked ? fmaxf(bound, least) : least)), hi = __builtin_amdgcn_readfirstlane(O::of(top));
        const unsigned highest = hi;
        const int finite = count(least);
        int need = min(a.k, finite);
        while (lo < hi && finite > need) {
            const unsigned mid = lo + (hi - lo + 1) / 2;
            if (count(O::bound(mid)) >= need) lo = mid;
            else hi = mid - 1;
        }
        const float at_least = O::bound(lo), above = lo < highest ? O::bound(lo + 1) : __builtin_inff();
        if (tid == 0) found = 0;
        __syncthreads();
        all([&](const Piece<TYPE> &p, int c) {
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (element(p, j) >= above && element(p, j) < __builtin_inff()) {      // (fewer than k)
                    const int to = atomicAdd(&found, 1);
                    if (to < KEYS) keys[to] = key_of(element(p, j), c + j);
                }
        });
        __syncthreads();
        int filled = min(found, need);
        need -= filled;
        for (int i = 0; i < pieces && need > 0; ++i) {
            Piece<TYPE> p;
            p.load_end(z, (i * NT + tid) * E, n);
            auto on = [&](float v) { return v >= at_least && !(v >= above); };
            int mine = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) mine += on(element(p, j));
            int at = mine;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const int o = __shfl_up(at, off, 64);
                if (lane >= off) at += o;
            }
            __syncthreads();
            if (lane == 63) buf4[wave] = at;
            __syncthreads();
            at -= mine;
            int these = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                at += w < wave ? buf4[w] : 0;
                these += buf4[w];
            }
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (on(element(p, j))) {
                    if (at < need) keys[filled + at] = key_of(element(p, j), from + (i * NT + tid) * E + j);
                    ++at;
                }
            filled += min(these, need);
            need -= min(these, need);
        }
        __syncthreads();
        have = filled;
    }
    if (a.parts == 1) {
        const bool lost = !(s[0] == s[0]);
        sort_keys<NT>(keys, have, a.k, [&](int i, Key key) {
            a.top_index[row * a.k + i] = lost ? -1 : (int)~(unsigned)key;
            a.top_logit[row * a.k + i] = lost ? __builtin_nanf("") : unordered((unsigned)(key >> 32));
        });
        for (int i = have + tid; i < a.k; i += NT) {
            a.top_index[row * a.k + i] = -1;
            a.top_logit[row * a.k + i] = lost ? __builtin_nanf("") : -__builtin_inff();
        }
    } else {
        Key *const list = a.lists + (int64_t)blockIdx.x * a.k;
        sort_keys<NT>(keys, have, a.k, [&](int i, Key key) { list[i] = key; });
        for (int i = have + tid; i < a.k; i += NT) list[i] = 0;
    }
}

// Rows of several parts: sums brought to the largest maximum, lists joined.  At least k entries of all lists reach the least of the
// lists' entries k / parts (counted from 1, rounded up), and also the largest of their k-th ones: what reaches both is sorted.
template <int TYPE>
__global__ __launch_bounds__(256) void score_join_kernel(Args a)
{
    constexpr int NT = 256, KEYS = 2048;
    __shared__ Key keys[KEYS];
    __shared__ int found;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t row = blockIdx.x;
    const Stats *const st = a.stats + row * a.parts;
    const Key *const lists = a.lists + row * a.parts * a.k;
    const int n = a.parts * a.k;
    int target = -1;
    float zt = 0.f;
    if (tid == 0) {
        found = 0;
        target = target_of(a, row);
        if (target >= 0) zt = load_as<TYPE>(a.z, row * a.ldz + target);
    }
    const float c2 = 1.44269504088896f / a.tau;
    // every wave for itself, a part to a lane
    Key low = ~(Key)0, high = 0;
    float top = -__builtin_inff(), sum = 0.f, dot = 0.f;
    const int share = a.k > 0 ? (a.k + a.parts - 1) / a.parts : 0;
    for (int p = lane; p < a.parts; p += 64) {
        top = st[p].sum == 0.f ? top : fmaxf(top, st[p].top);
        if (a.k > 0) {
            const Key l = lists[p * a.k + share - 1], h = lists[p * a.k + a.k - 1];
            low = l < low ? l : low;
            high = h > high ? h : high;
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const Key l = __shfl_xor(low, off, 64), h = __shfl_xor(high, off, 64);
        low = l < low ? l : low;
        high = h > high ? h : high;
    }
    top = join_lanes(top, fmaxf_of);
    if (top == -__builtin_inff()) top = 0.f;
    for (int p = lane; p < a.parts; p += 64) {
        const Stats s = st[p];
        if (s.sum == 0.f) continue;
        const float d = difference(s.top, top, c2), w = __builtin_amdgcn_exp2f(d);
        sum = fmaf(s.sum, w, sum);
        dot = fmaf(fmaf(s.sum, fmaxf(d, -1e30f), s.dot), w, dot);
    }
    sum = sum_lanes(sum);
    dot = sum_lanes(dot);
    if (tid == 0) finish(a, row, top, sum, dot, zt, target);
    if (a.k == 0) return;
    const bool lost = !(sum == sum);
    auto put = [&](int i, Key key) {
        a.top_index[row * a.k + i] = lost ? -1 : (int)~(unsigned)key;
        a.top_logit[row * a.k + i] = lost ? __builtin_nanf("") : unordered((unsigned)(key >> 32));
    };
    Key bound = low > high ? low : high;
    if (bound == 0) bound = 1;      // (0: no entry)
    __syncthreads();
    for (int e0 = 0; e0 < n; e0 += NT) {
        const Key key = e0 + tid < n ? lists[e0 + tid] : 0;
        const unsigned long long m = __ballot(key >= bound);
        if (m == 0) continue;
        int at = 0;
        if (lane == 0) at = atomicAdd(&found, __popcll(m));
        at = __builtin_amdgcn_readfirstlane(at) + __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u));
        if (key >= bound && at < KEYS) keys[at] = key;
    }
    __syncthreads();
    int have = found;
    if (have <= KEYS) {
        sort_keys<NT>(keys, have, a.k, put);
    } else {
        // too many: an entry's place is its own in its list and the number of larger ones in each of the others
        have = a.k;
        for (int e = tid; e < n; e += NT) {
            const Key key = lists[e];
            if (key == 0) continue;
            const int own = e / a.k;
            int rank = e - own * a.k;
            for (int p = 0; p < a.parts && rank < a.k; ++p) {
                if (p == own) continue;
                const Key *const l = lists + p * a.k;
                int lo = 0, hi = a.k;
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (l[mid] > key) lo = mid + 1;
                    else hi = mid;
                }
                rank += lo;
            }
            if (rank < a.k) put(rank, key);
        }
    }
    for (int i = have + tid; i < a.k; i += NT) {
        a.top_index[row * a.k + i] = -1;
        a.top_logit[row * a.k + i] = lost ? __builtin_nanf("") : -__builtin_inff();
    }
}

struct Plan {
    int threads, pieces, parts, len;
    size_t lists, bytes;
};

// Threads and pieces to a part.  Many rows: 256 with 16 each, the most that leave four workgroups to a compute unit.  Few: a row that
// 1024 threads hold goes to these, for the sooner end of it and of one launch (1 x 32000 in fp32: 8.2 us against 10.9 with 256 and a join);
// longer ones to small parts, as many of them as there can be.
inline Plan plan_of(int T, int V, int type, int k)
{
    const int E = type == OBC_F32 ? 4 : 8;
    Plan p;
    const int64_t large = (int64_t)256 * 16 * E;
    const bool many = (int64_t)T * ((V + large - 1) / large) >= 512;
    if (!many && V > 256 * 4 * E && V <= 1024 * 8 * E) {
        p.threads = 1024;
        p.pieces = 8;
    } else {
        p.threads = 256;
        p.pieces = many || k > 256 ? 16 : 4;
    }
    const int64_t most = (int64_t)p.threads * p.pieces * E;
    p.parts = (int)((V + most - 1) / most);
    p.len = (int)(((int64_t)V + p.parts - 1) / p.parts);
    p.len = (p.len + E - 1) / E * E;
    p.lists = p.bytes = 0;
    if (p.parts > 1) {
        p.lists = obc_align_up((size_t)T * p.parts * sizeof(Stats), 256);
        p.bytes = p.lists + (size_t)T * p.parts * k * sizeof(Key);
    }
    return p;
}

template <int TYPE>
void launch(obc_ctx *ctx, const Args &a, const Plan &p)
{
    const unsigned blocks = (unsigned)((int64_t)a.T * a.parts);
    auto go = [&](auto nt, auto ch) {
        if (a.k == 0) score_kernel<TYPE, nt, ch, 0, 0><<<blocks, nt.value, 0, ctx->stream>>>(a);
        else if (a.k <= 256) score_kernel<TYPE, nt, ch, 512, 1024><<<blocks, nt.value, 0, ctx->stream>>>(a);
        else score_kernel<TYPE, nt, ch, 1536, 2048><<<blocks, nt.value, 0, ctx->stream>>>(a);
    };
    if (p.threads == 1024) go(std::integral_constant<int, 1024>(), std::integral_constant<int, 8>());
    else if (p.pieces == 16) go(std::integral_constant<int, 256>(), std::integral_constant<int, 16>());
    else go(std::integral_constant<int, 256>(), std::integral_constant<int, 4>());
    if (a.parts == 1) return;
    score_join_kernel<TYPE><<<a.T, 256, 0, ctx->stream>>>(a);
}

}  // namespace

extern "C" {

int obc_score_workspace_bytes(int T, int V, int type, int k, size_t *bytes)
{
    if (!bytes || T < 0 || V <= 0 || k < 0 || k > kMaxTop || !float_type(type)) return OBC_ERR_BAD_ARG;
    *bytes = plan_of(T, V, type, k).bytes;
    return OBC_OK;
}

int obc_score(obc_ctx *ctx, const void *z, int type, int T, int V, int64_t ldz, const int32_t *target, float temperature, int k, float *logp,
              float *entropy, float *lse, int32_t *top_index, float *top_logit, void *ws, size_t ws_bytes)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (T < 0 || V <= 0 || k < 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_score: bad size");
    if (k > kMaxTop || V > kMaxCols)
        return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_score: k (%d) > %d or V (%d) > %d", k, kMaxTop, V, kMaxCols);
    if (!float_type(type)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_score: type %d is not a floating type", type);
    if (!(temperature > 0.f) || !(temperature < __builtin_inff()) || !(1.44269504088896f / temperature < __builtin_inff()))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_score: temperature or its reciprocal is not positive and finite");
    if (ldz < V) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_score: leading dimension below the row's length");
    if (T == 0) return OBC_OK;
    if ((logp != nullptr) != (target != nullptr)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_score: logp goes with target");
    if ((k > 0) != (top_index != nullptr) || (k > 0) != (top_logit != nullptr))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_score: top_index and top_logit go with k > 0");
    if (!z) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_score: null z");
    if (((uintptr_t)z & (size_of_type(type) - 1)) != 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_score: z is not aligned to its elements");
    const Plan p = plan_of(T, V, type, k);
    if (!obc_grid_fits((int64_t)T * p.parts, p.threads) || (int64_t)p.parts * k >= (int64_t)1 << 30)
        return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_score: too many rows or columns");
    if (p.bytes > 0 && (!ws || ((uintptr_t)ws & 15) != 0 || ws_bytes < p.bytes))
        return obc_fail(ctx, OBC_ERR_WORKSPACE, "obc_score: workspace of %zu bytes needed", p.bytes);
    const Args a = {z, target, logp, entropy, lse, top_index, top_logit, T, V, k, p.parts, p.len, ldz, temperature, (Stats *)ws,
                    (Key *)((char *)ws + p.lists), ctx->d_status};
    if (type == OBC_F32) launch<OBC_F32>(ctx, a, p);
    else if (type == OBC_F16) launch<OBC_F16>(ctx, a, p);
    else launch<OBC_BF16>(ctx, a, p);
    OBC_LAUNCH_CHECK(ctx, "score_kernel");
    return OBC_OK;
}

}  // extern "C"
