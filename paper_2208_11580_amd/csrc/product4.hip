// obc_product4: y = x W^T with W in 4-bit codes and a step and an offset per row and group of columns.
//
//   y[t, r] = sum_g ( delta[r, g] S - (16 delta[r, g] - offset[r, g]) s ),   S = sum_{c in g} x[t, c] (16 + code[r, c]),
//                                                                           s = sum_{c in g} x[t, c]
// The codes enter the matrix instructions as the 16-bit numbers 16 + code, exactly (8-bit inputs: as bytes, without
// the 16), so their products with 16-bit inputs are exact in fp32 and the only roundings are those of the fp32 sums; a
// group's sums start from zero and are scaled when it ends.  fp32 inputs go in as three bf16 terms, against 2 code - 15, which also
// 16-bit inputs meet where the output is fp32.
//
// Up to 16 tokens: bound by the weights' bytes (product4_rows_kernel).  One token through 8192 x 8192 takes 9.2 us in half
// precision, 35.7 MB at 3.9 TB/s (plain reads of 64 MB and more: 6.0 to 6.3); through 768 x 768 3.3 us, of which about 2 are a
// launch.  More tokens (product4_tiles_kernel): the matrix cores and the unpacking, neither of which fills the time.  2048 tokens through
// 4096 x 4096 in bf16 take 80 us, 860 TFLOP/s (a dense library product of that size: 61 us, 1120); in the tiles' 73 us the matrix cores are
// busy 41 % of the time and the vector instructions issue 38 % of it, 3.7 to a matrix instruction.  8-bit inputs: 1000 tokens through 4096
// x 8192 in groups of 64 take 84 us in the tiles, 800 TOP/s, 19 % and 48 %, 10 vector instructions to a matrix instruction.  (Medians, captured in a graph.)
#include "product4.h"

namespace {

struct Args {
    const uintx4 *codes;
    const unsigned *scales;
    const void *x;
    const float *xs;
    void *y;
    int T, R, d, RB, KT, NG, tpg;
    unsigned tpg_inv, tpg_one;      // floor(2^32 / tpg) + 1 and 0; for tpg = 1, 0 and all ones; for one group, 0 and 0
    int64_t ldx, ldy;

    // kt / tpg: exact while kt tpg < 2^32, beyond which a call with several groups is refused (rows of 8 million columns and more)
    __device__ int group_of(int kt) const { return (int)(__umulhi((unsigned)kt, tpg_inv) + ((unsigned)kt & tpg_one)); }
};

template <int V>
struct Type {
    static constexpr int value = V;
};

constexpr bool is_16_bit(int type) { return type == OBC_F16 || type == OBC_BF16; }

// f(Type<y_type>()), for the types that XT and CENTRED come with: 16-bit inputs are centred where the output is fp32
template <int XT, bool CENTRED, class F>
__device__ inline void with_output_type(int y_type, F f)
{
    if constexpr (is_16_bit(XT) && CENTRED) {
        f(Type<OBC_F32>());
    } else {
        if (!is_16_bit(XT) && y_type == OBC_F32) f(Type<OBC_F32>());
        else if (y_type == OBC_F16) f(Type<OBC_F16>());
        else f(Type<OBC_BF16>());
    }
}

// One 16x16x32 operand of token rows: the lane's eight columns from `c` on of row `row`, zeros from d on.
template <int XT>
struct Operand;

template <>
struct Operand<OBC_BF16> {
    uintx4 v;
    __device__ void load(const void *x, int64_t at, int left)
    {
        const unsigned short *p = (const unsigned short *)x + at;
        if (left >= 8) {
            v = *(const uintx4_at2 *)p;
        } else {
            unsigned short e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = j < left ? p[j] : (unsigned short)0;
            v = uintx4{e[0] | (unsigned)e[1] << 16, e[2] | (unsigned)e[3] << 16, e[4] | (unsigned)e[5] << 16, e[6] | (unsigned)e[7] << 16};
        }
    }
};

template <>
struct Operand<OBC_F16> : Operand<OBC_BF16> {
};

template <>
struct Operand<OBC_F32> {
    uintx4 v[3];
    __device__ void load(const void *x, int64_t at, int left)
    {
        const float *p = (const float *)x + at;
        float e[8];
        if (left >= 8) {
            const floatx4 a = *(const floatx4_at4 *)p, b = *(const floatx4_at4 *)(p + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) { e[j] = a[j]; e[4 + j] = b[j]; }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = j < left ? p[j] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float h0, m0, l0, h1, m1, l1;
            split3(e[2 * j], h0, m0, l0);
            split3(e[2 * j + 1], h1, m1, l1);
            v[0][j] = pair_bf16(h0, h1);
            v[1][j] = pair_bf16(m0, m1);
            v[2][j] = pair_bf16(l0, l1);
        }
    }
};

template <>
struct Operand<OBC_I8> {
    uintx2 v;
    __device__ void load(const void *x, int64_t at, int left)
    {
        const uint8_t *p = (const uint8_t *)x + at;
        uintx2 r;
        if (left >= 8) {
            r = *(const uintx2_at1 *)p;
        } else {
            unsigned e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = j < left ? p[j] : 0u;
            r = uintx2{e[0] | e[1] << 8 | e[2] << 16 | e[3] << 24, e[4] | e[5] << 8 | e[6] << 16 | e[7] << 24};
        }
        v = bytes_like_codes(r);
    }
};

// What stands for a code q in XT's operands is q / unit + base.  CENTRED, for fp32 inputs and fp32 outputs: 2 q - 15, which costs the
// unpacking three times the instructions (22 for eight codes, 8 for 16 + q): the matrix cores' sums are not rounded to nearest, and their
// error grows with the sums' size, five times as large with 16 + q.  (fp32 inputs, 100 tokens through 300 x 128: 1.1e-6 off with 16 + q,
// 1.1e-7 with 2 q - 15; 40 through 512 x 16384 3.4e-6 and 1.6e-7; 500 through 4096 x 4096 take 75 us, 67 with 16 + q.  fp16
// inputs, fp32 outputs, 40 through 512 x 16384: 1.0e-7 off, with 16 + q six times as much; one token through 8192 x 8192 takes 11.3 us,
// with 16 + q 9.4, 2048 through 4096 x 4096 90 and 77.)  16-bit outputs hide either.
template <int XT, bool CENTRED>
constexpr float kUnit = CENTRED ? 0.5f : 1.f;
template <int XT, bool CENTRED>
constexpr float kBase = CENTRED ? -7.5f : XT == OBC_I8 ? 0.f : kCodeBase;      // base times unit

template <int XT, bool CENTRED>
__device__ inline uintx4 codes_of(unsigned w)
{
    return CENTRED ? codes_centred<XT == OBC_F16>(w) : XT == OBC_F16 ? codes_f16(w) : codes_bf16(w);
}

// Codes of one instruction and ones, as the operand that meets XT's.
template <int XT, bool CENTRED>
struct Codes {
    uintx4 v;
    __device__ explicit Codes(unsigned w) : v(codes_of<XT, CENTRED>(w)) {}
    static __device__ Codes ones()
    {
        Codes c(0);
        const unsigned one = XT == OBC_F16 ? 0x3c003c00u : 0x3f803f80u;
        c.v = uintx4{one, one, one, one};
        return c;
    }
};

template <>
struct Codes<OBC_I8, false> {
    uintx2 v;
    __device__ explicit Codes(unsigned w) : v(codes_i8(w)) {}
    static __device__ Codes ones()
    {
        Codes c(0);
        c.v = uintx2{0x01010101u, 0x01010101u};
        return c;
    }
};

template <int XT>
struct Sum {
    floatx4 s = {0.f, 0.f, 0.f, 0.f};
    template <bool CENTRED>
    __device__ void add(const Operand<XT> &a, const Codes<XT, CENTRED> &b)
    {
        if constexpr (XT == OBC_F32) {
            s = mfma_bf16(a.v[2], b.v, s);
            s = mfma_bf16(a.v[1], b.v, s);
            s = mfma_bf16(a.v[0], b.v, s);
        } else if constexpr (XT == OBC_F16) {
            s = mfma_f16(a.v, b.v, s);
        } else {
            s = mfma_bf16(a.v, b.v, s);
        }
    }
    __device__ float operator[](int i) const { return s[i]; }
};

template <>
struct Sum<OBC_I8> {
    intx4 s = {0, 0, 0, 0};
    __device__ void add(const Operand<OBC_I8> &a, const Codes<OBC_I8, false> &b) { s = mfma_i8(a.v, b.v, s); }
    __device__ float operator[](int i) const { return (float)s[i]; }
};

// What a token's pieces are exchanged by in LDS, so that the 16 tokens of an operand lie in different banks: rows of 16 pieces
// are as long as the 64 banks, rows of 8 (8-bit inputs) half as long.
template <int ROW>
__device__ inline int turned(int t)
{
    return ROW == 16 ? t & 15 : (t >> 1) & 7;
}

// ---- few tokens ------------------------------------------------------------------------------
constexpr int kRowsTokens = 16;
constexpr int kRowsLds = 147456;     // of a compute unit, for its workgroups' tokens
// waves of a workgroup at most, as registers allow: an fp32 operand is three
constexpr int rows_waves(int XT) { return XT == OBC_F32 ? 8 : 16; }

// Bytes of a token's tile of 128 columns in LDS
constexpr int tile_bytes(int XT) { return XT == OBC_F32 ? 768 : XT == OBC_I8 ? 128 : 256; }

// 16 NF rows of W and up to 16 tokens to a workgroup, whose waves take turns along the columns' tiles and sum in LDS.  The
// weights' bytes bound it: a wave has its next tile's codes on their way (two or three ahead measured slower, 9.9 and 11.3 us against
// 9.2 for one token through 8192 x 8192: 16 waves to a compute unit cover the rest, and the copies cost instructions).  Loads come back
// in order, so the tokens must not be among them: they go through LDS, `chunk` tiles at a time.
template <int XT, bool CENTRED, int SUB, int NF>
__global__ __launch_bounds__(rows_waves(XT) * 64) void product4_rows_kernel(Args a, int y_type, int chunk)
{
    constexpr int P = XT == OBC_F32 ? 3 : 1, OPS = XT == OBC_I8 ? 8 : 16;      // planes; 16-byte places of a token's tile
    extern __shared__ uintx4 lds[];
    // (the wave's number is the same in all its lanes, which the compiler does not see by itself)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int n = lane & 15, quad = lane >> 4;
    const int rb0 = blockIdx.x * NF;
    int64_t rb[NF];
#pragma unroll
    for (int j = 0; j < NF; ++j) rb[j] = rb0 + j < a.RB ? rb0 + j : a.RB - 1;
    float acc[NF][4];
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    const auto ones = Codes<XT, CENTRED>::ones();
    struct Weights {
        uintx4 w[NF];
        unsigned sc[NF][SUB];
    };
    auto fetch = [&](Weights &g, int kt) {
        if (kt >= a.KT) kt = a.KT - 1;
#pragma unroll
        for (int j = 0; j < NF; ++j) {
            g.w[j] = a.codes[(rb[j] * a.KT + kt) * 64 + lane];
            if constexpr (SUB == 4) {
                const uintx4 v = *((const uintx4 *)a.scales + (rb[j] * a.KT + kt) * 16 + n);
#pragma unroll
                for (int u = 0; u < 4; ++u) g.sc[j][u] = v[u];
            } else if constexpr (SUB == 2) {
                const uintx2 v = *((const uintx2 *)a.scales + (rb[j] * a.KT + kt) * 16 + n);
                g.sc[j][0] = v.x;
                g.sc[j][1] = v.y;
            } else {
                g.sc[j][0] = a.scales[(rb[j] * a.NG + a.group_of(kt)) * 16 + n];
            }
        }
    };
    // Operand o (step k, quad) of token t and tile i of the chunk; 8-bit inputs: 8 bytes
    auto place = [&](int i, int p, int t, int o) { return ((i * P + p) * a.T + t) * OPS + ((XT == OBC_I8 ? o >> 1 : o) ^ turned<OPS>(t)); };
    auto put = [&](const Operand<XT> &x, int i, int t, int o) {
        if constexpr (XT == OBC_F32) {
#pragma unroll
            for (int p = 0; p < 3; ++p) lds[place(i, p, t, o)] = x.v[p];
        } else if constexpr (XT == OBC_I8) {
            ((uintx2 *)&lds[place(i, 0, t, o)])[o & 1] = x.v;
        } else {
            lds[place(i, 0, t, o)] = x.v;
        }
    };
    auto stage = [&](int kt0, int tiles) {
        // tiles that are whole: 64 operands of a token to a wave, several loads on their way at a time; the tile that d ends
        // in: element by element
        const int full = (a.d >> 7) - kt0 < tiles ? (a.d >> 7) - kt0 : tiles;
        const int ops = full * 16, blocks = (ops + 63) >> 6;
        constexpr int N = XT == OBC_F32 ? 2 : 8;
        int t = 0, b = wave;
        while (t < a.T && blocks > 0) {
            Operand<XT> x[N];
            int ts[N], bs[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                while (b >= blocks && t < a.T) {
                    b -= blocks;
                    ++t;
                }
                ts[i] = t;
                bs[i] = b;
                if (t < a.T) {
                    int e = b * 64 + lane;
                    e = e < ops ? e : ops - 1;
                    x[i].load(a.x, t * a.ldx + kt0 * 128 + 8 * e, 8);
                }
                b += waves;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int e = bs[i] * 64 + lane;
                if (ts[i] < a.T && e < ops) put(x[i], e >> 4, ts[i], e & 15);
            }
        }
        if (full < tiles)
            for (int e = threadIdx.x; e < a.T * 16; e += blockDim.x) {
                const int o = e & 15, c = (kt0 + full) * 128 + 8 * o;
                Operand<XT> x;
                x.load(a.x, (e >> 4) * a.ldx + c, a.d - c);
                put(x, full, e >> 4, o);
            }
    };
    const int t = n < a.T ? n : a.T - 1;      // rows beyond the last token: not stored
    auto compute = [&](const Weights &g, int i) {
        Operand<XT> x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (XT == OBC_F32) {
#pragma unroll
                for (int p = 0; p < 3; ++p) x[k].v[p] = lds[place(i, p, t, 4 * k + quad)];
            } else if constexpr (XT == OBC_I8) {
                x[k].v = ((const uintx2 *)&lds[place(i, 0, t, 4 * k + quad)])[quad & 1];
            } else {
                x[k].v = lds[place(i, 0, t, 4 * k + quad)];
            }
        }
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            Sum<XT> s, S[NF];
#pragma unroll
            for (int k = u * 4 / SUB; k < (u + 1) * 4 / SUB; ++k) {
                s.add(x[k], ones);
#pragma unroll
                for (int j = 0; j < NF; ++j) S[j].add(x[k], Codes<XT, CENTRED>(g.w[j][k]));
            }
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                const float step = half_lo(g.sc[j][u]), off = half_hi(g.sc[j][u]) - kBase<XT, CENTRED> * step;
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[j][v] = fmaf(step * kUnit<XT, CENTRED>, S[j][v], fmaf(off, s[v], acc[j][v]));
            }
        }
    };
    Weights next;
    fetch(next, wave);
    for (int kt0 = 0; kt0 < a.KT; kt0 += chunk) {      // chunks are multiples of the waves, but for the last
        const int tiles = kt0 + chunk < a.KT ? chunk : a.KT - kt0;
        if (kt0) __syncthreads();
        stage(kt0, tiles);
        __syncthreads();
        for (int i = wave; i < tiles; i += waves) {
            const Weights now = next;
            fetch(next, kt0 + i + waves);
            compute(now, i);
        }
    }
    __syncthreads();
    float *const part = (float *)lds;      // waves x NF x 4 x 64
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[((wave * NF + j) * 4 + i) * 64 + lane] = acc[j][i];
    __syncthreads();
    for (int e = threadIdx.x; e < NF * 256; e += blockDim.x) {
        const int l = e & 63, i = (e >> 6) & 3, j = e >> 8;
        const int to = 4 * (l >> 4) + i, r = (rb0 + j) * 16 + (l & 15);
        if (to >= a.T || r >= a.R) continue;
        float v = 0.f;
        for (int w = 0; w < waves; ++w) v += part[w * (NF * 256) + e];
        if (XT == OBC_I8) v *= a.xs[to];
        const int64_t at = (int64_t)to * a.ldy + r;
        with_output_type<XT, CENTRED>(y_type, [&](auto type) { store_as<decltype(type)::value>(a.y, at, v); });
    }
}

// ---- many tokens ------------------------------------------------------------------------------
// What the tiles' kernel needs beside x: the sums of every token's groups, as three planes of bf16 terms (T x NGP each, zeros
// from NG on); and, where x is not laid out like that already, the tokens' rows at multiples of 16 bytes with zeros up to a multiple
// of 128 columns -- fp32 as three planes of bf16 terms, 8-bit ones in the order of the operands (i8_place).  A team of TEAM lanes to a
// token and group.
struct Lay {
    unsigned short *sums;
    uintx4 *rows;      // null: x as it lies
    int NGP, G;        // groups of a row, padded to 32; columns of a group
    int64_t jobs;      // T x NG
};

// Where piece p of eight columns of a laid-out 8-bit token lies: the two that a lane of quad q takes for one instruction of 64
// columns, 8 q and 32 + 8 q on, side by side, bytes in the codes' order.
__device__ inline int i8_place(int p)
{
    return (p & ~7) | (p & 3) << 1 | (p >> 2 & 1);
}

template <int XT, int TEAM>
__global__ __launch_bounds__(256) void product4_lay_kernel(Args a, Lay lay)
{
    const int64_t job = ((int64_t)blockIdx.x * 256 + threadIdx.x) / TEAM;
    const int lane = threadIdx.x % TEAM;
    if (job >= lay.jobs) return;
    const int64_t t = job / a.NG;
    const int g = (int)(job - t * a.NG);
    const int pieces = a.KT * 16, first = g * (lay.G / 8), end = g == a.NG - 1 ? pieces : first + lay.G / 8;
    const int64_t plane = (int64_t)a.T * pieces;
    float sum = 0.f;
    for (int p = first + lane; p < end; p += TEAM) {
        const int c = p * 8;
        Operand<XT> o;
        o.load(a.x, t * a.ldx + c, a.d - c);
        if constexpr (XT == OBC_F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sum += (bf16_lo(o.v[0][j]) + bf16_lo(o.v[1][j]) + bf16_lo(o.v[2][j])) + (bf16_hi(o.v[0][j]) + bf16_hi(o.v[1][j]) + bf16_hi(o.v[2][j]));
            }
            if (lay.rows)
#pragma unroll
                for (int q = 0; q < 3; ++q) lay.rows[q * plane + t * pieces + p] = o.v[q];
        } else if constexpr (XT == OBC_I8) {
            int s = __builtin_amdgcn_sdot4((int)o.v.x, 0x01010101, 0, false);
            s = __builtin_amdgcn_sdot4((int)o.v.y, 0x01010101, s, false);
            sum += (float)s;
            ((uintx2 *)lay.rows)[t * pieces + i8_place(p)] = o.v;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned w = o.v[j];
                sum += XT == OBC_F16 ? half_lo(w) + half_hi(w) : bf16_lo(w) + bf16_hi(w);
            }
            if (lay.rows) lay.rows[t * pieces + p] = o.v;
        }
    }
#pragma unroll
    for (int off = TEAM / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off, TEAM);
    float term[3];
    split3(sum, term[0], term[1], term[2]);
    unsigned short *const at = lay.sums + t * lay.NGP;
    const int64_t splane = (int64_t)a.T * lay.NGP;
    if (lane == 0)
#pragma unroll
        for (int q = 0; q < 3; ++q) at[q * splane + g] = (unsigned short)pair_bf16(term[q], 0.f);
    if (g == a.NG - 1)
        for (int z = a.NG + lane; z < lay.NGP; z += TEAM)
#pragma unroll
            for (int q = 0; q < 3; ++q) at[q * splane + z] = 0;
}

struct Tokens {
    const char *x;           // first plane
    int64_t ld, plane;       // bytes between rows, between planes
    const unsigned short *sums;
    int NGP;
    int mtiles, tiles;       // blocks of BM tokens, of those x BN rows
    int per;                 // column tiles of a slice
    float *part;             // slices x T x R sums, where there are several
};

// BM tokens x BN rows of W to a workgroup of WM x WN waves.  Tokens, codes and steps of STAGES column tiles go through LDS in
// turn, so that loads have STAGES - 1 tiles' time to arrive; a wave waits for all but its newest ones and then for the others.
//
// 128 x 256 with eight waves of 64 x 64 where that fills the chip: a wave's unpacked codes serve 64 tokens, its tokens 64 rows.  Waves
// of 128 x 64, which unpack half as much, are one to a SIMD and slower (2048 tokens through 4096 x 4096: 106 us, when this one took
// 84); more stages or operands read a step earlier changed nothing.
constexpr int tile_waves(int BN) { return BN / 32; }

template <int XT, int SUB, int BM, int BN, int WM, int STAGES>
struct Tile {
    static constexpr int WAVES = tile_waves(BN);
    static constexpr int WN = WAVES / WM;
    static constexpr int P = XT == OBC_F32 ? 3 : 1, MF = BM / WM / 16, NF = BN / WN / 16;
    static constexpr int ROW = XT == OBC_I8 ? 8 : 16;      // 16-byte pieces of a token's 128 columns
    static constexpr int XN = P * BM * ROW, WN16 = BN * 4;      // 16-byte places of a stage: tokens, codes
    // loads of a wave for a stage: 64 places each, and 64 steps -- 32 of them twice where a wave has only 32 to load: what the
    // compiler makes of waits depends on every path having the same loads
    static constexpr int XL = XN / 64 / WAVES, WL = WN16 / 64 / WAVES, SL = BN * SUB / 64 / WAVES > 0 ? BN * SUB / 64 / WAVES : 1;
    static constexpr int SLANES = BN * SUB / WAVES < 64 ? BN * SUB / WAVES : 64;
    static constexpr int LOADS = XL + WL + SL;
    static constexpr int PLACES = XN + WN16 + SL * WAVES * 16;
    static __device__ int step_at(int e) { return e / SLANES * 64 + e % SLANES; }
    static_assert(XN % (64 * WAVES) == 0 && WN16 % (64 * WAVES) == 0, "whole loads");
};

template <int XT, bool CENTRED, int SUB, int BM, int BN, int WM, int STAGES>
__global__ __launch_bounds__(tile_waves(BN) * 64, 2) void product4_tiles_kernel(Args a, Tokens tok, int y_type)
{
    using C = Tile<XT, SUB, BM, BN, WM, STAGES>;
    constexpr int P = C::P, MF = C::MF, NF = C::NF, ROW = C::ROW;
    // separate arrays: the compiler then knows that reading one does not wait for loads to another
    __shared__ uintx4 lds0[C::PLACES], lds1[C::PLACES], lds2[STAGES > 2 ? C::PLACES : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, quad = lane >> 4;
    const int wm = wave % WM, wn = wave / WM;
    const int slice = blockIdx.x / tok.tiles, tile = tile_of(blockIdx.x % tok.tiles, tok.tiles);
    const int t0 = (tile % tok.mtiles) * BM, rb0 = (tile / tok.mtiles) * (BN / 16);
    const int kt0 = slice * tok.per, kt1 = kt0 + tok.per < a.KT ? kt0 + tok.per : a.KT;
    auto row_block = [&](int j) { return (int64_t)(rb0 + j < a.RB ? rb0 + j : a.RB - 1); };      // beyond the last: not stored

    // where this lane's loads come from, at the slice's first tile
    const char *xsrc[C::XL], *wsrc[C::WL], *ssrc[C::SL];
    // Piece o of token t lies at place o ^ turned(t) of its row.  The lanes of a load to LDS write 64 places in a row: each
    // fetches the piece that belongs to its place.
#pragma unroll
    for (int i = 0; i < C::XL; ++i) {
        const int first = (i * C::WAVES + wave) * (64 / ROW);      // row of the planes, one below the other
        const int p = P > 1 ? first / BM : 0, t = first - p * BM + lane / ROW;
        const int row = t0 + t < a.T ? t0 + t : a.T - 1;
        xsrc[i] = tok.x + p * tok.plane + row * tok.ld + (int64_t)kt0 * (ROW * 16) + ((lane % ROW) ^ turned<ROW>(t)) * 16;
    }
#pragma unroll
    for (int i = 0; i < C::WL; ++i) wsrc[i] = (const char *)a.codes + (row_block(i * C::WAVES + wave) * a.KT + kt0) * 1024 + lane * 16;
    // steps: row r of the tile, group u of its SUB is the step r SUB + u
    int64_t srow[C::SL];
#pragma unroll
    for (int i = 0; i < C::SL; ++i) {
        const int e = (i * C::WAVES + wave) * C::SLANES + lane % C::SLANES, r = e / SUB;
        srow[i] = SUB > 1 ? ((row_block(r >> 4) * a.KT) * 16 + (r & 15)) * SUB + e % SUB : row_block(r >> 4) * a.NG * 16 + (r & 15);
        ssrc[i] = (const char *)a.scales + srow[i] * 4;
    }
    auto fetch = [&](int kt, uintx4 *lds) __attribute__((always_inline)) {
        const int k = (kt < kt1 ? kt : kt1 - 1) - kt0;      // (behind the last: its tile again, for the count of loads)
#pragma unroll
        for (int i = 0; i < C::XL; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(xsrc[i] + (int64_t)k * (ROW * 16)), (lds_ptr)(lds + (i * C::WAVES + wave) * 64), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < C::WL; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(wsrc[i] + (int64_t)k * 1024), (lds_ptr)(lds + C::XN + (i * C::WAVES + wave) * 64), 16, 0, 0);
        const int64_t s = SUB > 1 ? (int64_t)(k + kt0) * 64 * SUB : (int64_t)a.group_of(k + kt0) * 64;
#pragma unroll
        for (int i = 0; i < C::SL; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(ssrc[i] + s), (lds_ptr)((unsigned *)(lds + C::XN + C::WN16) + (i * C::WAVES + wave) * 64), 4, 0, 0);
    };
    fetch(kt0, lds0);
    if (STAGES > 2) fetch(kt0 + 1, lds1);

    floatx4 acc[MF][NF];
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[m][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    // the groups' sums times what codes leave out of the weights, offset - 16 step: six of the nine products of terms (the
    // first slice's work)
    if (slice == 0) {
        for (int g0 = 0; g0 < a.NG; g0 += 32) {
            uintx4 B[3][NF];
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                const int64_t rb = row_block(wn * NF + j);
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int g = g0 + 8 * quad + e;
                    unsigned sc = 0;
                    if (g < a.NG) sc = SUB > 1 ? a.scales[((rb * a.KT + g / SUB) * 16 + n) * SUB + g % SUB] : a.scales[(rb * a.NG + g) * 16 + n];
                    v[e] = half_hi(sc) - kBase<XT, CENTRED> * half_lo(sc);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float h0, m0, l0, h1, m1, l1;
                    split3(v[2 * e], h0, m0, l0);
                    split3(v[2 * e + 1], h1, m1, l1);
                    B[0][j][e] = pair_bf16(h0, h1);
                    B[1][j][e] = pair_bf16(m0, m1);
                    B[2][j][e] = pair_bf16(l0, l1);
                }
            }
#pragma unroll
            for (int m = 0; m < MF; ++m) {
                const int t = t0 + (wm * MF + m) * 16 + n;
                const unsigned short *src = tok.sums + (int64_t)(t < a.T ? t : a.T - 1) * tok.NGP + g0 + 8 * quad;
                uintx4 A[3];
#pragma unroll
                for (int p = 0; p < 3; ++p) A[p] = *(const uintx4 *)(src + p * (int64_t)a.T * tok.NGP);
#pragma unroll
                for (int o = 2; o >= 0; --o)
#pragma unroll
                    for (int p = 0; p <= o; ++p)
#pragma unroll
                        for (int j = 0; j < NF; ++j) acc[m][j] = mfma_bf16(A[p], B[o - p][j], acc[m][j]);
            }
        }
    }
    __builtin_amdgcn_s_waitcnt(wait_loads(0));
    stage_barrier();

    auto turn = [&](const int kt, const uintx4 *lds, uintx4 *lds_next) __attribute__((always_inline)) {
        fetch(kt + STAGES - 1, lds_next);
        uintx4 w[NF];
        float step[NF][SUB];
#pragma unroll
        for (int j = 0; j < NF; ++j) {
            w[j] = lds[C::XN + (wn * NF + j) * 64 + lane];
#pragma unroll
            for (int u = 0; u < SUB; ++u)
                step[j][u] = kUnit<XT, CENTRED> * half_lo(((const unsigned *)(lds + C::XN + C::WN16))[C::step_at(((wn * NF + j) * 16 + n) * SUB + u)]);
        }
        if constexpr (XT == OBC_I8) {
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                intx4 S[MF][NF];
#pragma unroll
                for (int m = 0; m < MF; ++m)
#pragma unroll
                    for (int j = 0; j < NF; ++j) S[m][j] = intx4{0, 0, 0, 0};
                // the lane's columns of 64 (i8_place)
                auto place = [&](int m, int k) { return (16 * (wm * MF + m) + n) * ROW + ((4 * k + quad) ^ turned<ROW>(n)); };
                if constexpr (SUB == 4) {
                    uintx2 B[NF];
#pragma unroll
                    for (int j = 0; j < NF; ++j) B[j] = codes_i8(w[j][u]);
#pragma unroll
                    for (int m = 0; m < MF; ++m) {
                        const uintx2 A = ((const uintx2 *)lds)[2 * place(m, u >> 1) + (u & 1)];
#pragma unroll
                        for (int j = 0; j < NF; ++j) S[m][j] = mfma_i8(A, B[j], S[m][j]);
                    }
                } else {
#pragma unroll
                    for (int k = u * 2 / SUB; k < (u + 1) * 2 / SUB; ++k) {
                        intx4 B[NF];
#pragma unroll
                        for (int j = 0; j < NF; ++j) {
                            const uintx2 lo = codes_i8(w[j][2 * k]), hi = codes_i8(w[j][2 * k + 1]);
                            B[j] = intx4{(int)lo.x, (int)lo.y, (int)hi.x, (int)hi.y};
                        }
#pragma unroll
                        for (int m = 0; m < MF; ++m) {
                            const intx4 A = ((const intx4 *)lds)[place(m, k)];
#pragma unroll
                            for (int j = 0; j < NF; ++j) S[m][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(A, B[j], S[m][j], 0, 0, 0);
                        }
                    }
                }
#pragma unroll
                for (int m = 0; m < MF; ++m)
#pragma unroll
                    for (int j = 0; j < NF; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[m][j][i] = fmaf(step[j][u], (float)S[m][j][i], acc[m][j][i]);
            }
        } else {
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                floatx4 S[MF][NF];
#pragma unroll
                for (int m = 0; m < MF; ++m)
#pragma unroll
                    for (int j = 0; j < NF; ++j) S[m][j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = u * 4 / SUB; k < (u + 1) * 4 / SUB; ++k) {
                    uintx4 B[NF];
#pragma unroll
                    for (int j = 0; j < NF; ++j) B[j] = codes_of<XT, CENTRED>(w[j][k]);
#pragma unroll
                    for (int m = 0; m < MF; ++m)
#pragma unroll
                        for (int p = P - 1; p >= 0; --p) {
                            const uintx4 A = lds[(p * BM + 16 * (wm * MF + m) + n) * ROW + ((4 * k + quad) ^ turned<ROW>(n))];
#pragma unroll
                            for (int j = 0; j < NF; ++j) S[m][j] = XT == OBC_F16 ? mfma_f16(A, B[j], S[m][j]) : mfma_bf16(A, B[j], S[m][j]);
                        }
                }
#pragma unroll
                for (int m = 0; m < MF; ++m)
#pragma unroll
                    for (int j = 0; j < NF; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[m][j][i] = fmaf(step[j][u], S[m][j][i], acc[m][j][i]);
            }
        }
        __builtin_amdgcn_s_waitcnt(wait_loads(STAGES > 2 ? C::LOADS : 0));      // the next tile is in LDS
        stage_barrier();
    };
    for (int kt = kt0;;) {
        turn(kt, lds0, STAGES > 2 ? lds2 : lds1);
        if (++kt >= kt1) break;
        turn(kt, lds1, lds0);
        if (++kt >= kt1) break;
        if (STAGES > 2) {
            turn(kt, lds2, lds1);
            if (++kt >= kt1) break;
        }
    }
    // (loads behind the last tile still write to LDS: they are waited for before it can be another workgroup's)
    __builtin_amdgcn_s_waitcnt(wait_loads(0));
    const bool sliced = tok.part != nullptr;
    auto put = [&](auto type) {
        constexpr int YT = decltype(type)::value;
#pragma unroll
        for (int m = 0; m < MF; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = t0 + (wm * MF + m) * 16 + 4 * quad + i;
                if (t >= a.T) continue;
                const float xs = XT == OBC_I8 && !sliced ? a.xs[t] : 1.f;
#pragma unroll
                for (int j = 0; j < NF; ++j) {
                    const int r = (rb0 + wn * NF + j) * 16 + n;
                    const float v = XT == OBC_I8 ? acc[m][j][i] * xs : acc[m][j][i];
                    if (r >= a.R) continue;
                    if (sliced) tok.part[((int64_t)slice * a.T + t) * a.R + r] = v;
                    else store_as<YT>(a.y, (int64_t)t * a.ldy + r, v);
                }
            }
    };
    with_output_type<XT, CENTRED>(y_type, put);
}

// The slices' sums, in their order.
__global__ __launch_bounds__(256) void product4_add_kernel(Args a, const float *__restrict__ part, int slices, int y_type)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)a.T * a.R;
    if (i >= n) return;
    float v = add_slices(part + i, n, slices);
    const int64_t t = i / a.R;
    if (a.xs) v *= a.xs[t];
    const int64_t at = t * a.ldy + (i - t * a.R);
    if (y_type == OBC_F32) store_as<OBC_F32>(a.y, at, v);
    else if (y_type == OBC_F16) store_as<OBC_F16>(a.y, at, v);
    else store_as<OBC_BF16>(a.y, at, v);
}

// True where the tiles' kernel can read x as it lies.
inline bool laid_out(const void *x, int x_type, int64_t ldx, int d)
{
    return (x_type == OBC_F16 || x_type == OBC_BF16) && d % 128 == 0 && ((uintptr_t)x & 15) == 0 && (ldx * (int64_t)size_of_type(x_type)) % 16 == 0;
}

// What a product with more tokens than the rows' kernel takes is cut into, and its workspace.
struct Plan {
    int BM, BN, mtiles, ntiles, slices, per, NGP;
    size_t sums, laid, part, bytes;      // the groups' sums, tokens laid out (where x is not like that already), the slices' sums
};

Plan plan_of(const pack4_layout &L, int T, int x_type)
{
    Plan p;
    auto cut = [&](int BM, int BN) {
        p.BM = BM;
        p.BN = BN;
        p.mtiles = T / BM + (T % BM != 0);
        p.ntiles = (L.RB * 16 + BN - 1) / BN;
        return (int64_t)p.mtiles * p.ntiles;
    };
    int64_t tiles = 0;
    if (x_type == OBC_F32) tiles = T > 32 ? cut(64, 128) : cut(32, 128);
    else if (T <= 32) tiles = cut(32, 128);
    // 128 x 256 for three quarters of the compute units and more (2048 x 4096 x 4096 in bf16, 256 tiles: 82 us, in tiles of 64 x 128
    // 101; 500 x 4096 x 4096, 64 tiles: 63 us and 34; 8 bits, 1000 x 4096 x 8192, 128 tiles: 145 us and 102)
    else if (T <= 64 || (tiles = cut(128, 256)) < 192) tiles = cut(64, 128);
    // few tokens leave too few tiles for the chip: slices of the columns, two workgroups to a compute unit (fp32 in tiles of 64: one),
    // two tiles at least to a slice (4096 x 4096 in bf16, 17 tokens: 12.8 us, with one slice 20.9; 64 tokens: 19.0 and 31.1)
    int64_t s = p.BM < 128 && tiles > 0 ? (x_type == OBC_F32 && p.BM == 64 ? 256 : 512) / tiles : 1;
    if (s > 16) s = 16;
    if (s > L.KT / 2) s = L.KT / 2;
    if (s < 1) s = 1;
    p.per = (int)((L.KT + s - 1) / s);
    p.slices = (L.KT + p.per - 1) / p.per;
    p.NGP = (L.NG + 31) / 32 * 32;
    size_t at = 0;
    auto take = [&](size_t n) { const size_t b = at; at += obc_align_up(n, 256); return b; };
    p.sums = take((size_t)T * p.NGP * 6);
    p.part = take(p.slices > 1 ? (size_t)p.slices * T * L.R * 4 : 0);
    p.laid = take((size_t)T * L.KT * 128 * (x_type == OBC_F32 ? 6 : x_type == OBC_I8 ? 1 : 2));
    p.bytes = at;
    return p;
}

// The rows' kernel: up to 16 tokens, if they fit in LDS at once or there are rows for every compute unit.  (16 tokens through
// 768 x 16384: 62 us in fp32 and 24 in half precision with 16 and 3 fillings of LDS in 48 workgroups, in tiles 27 and 21;
// through 4096 x 4096 in half precision 9 us, in tiles 16.)
struct Rows {
    int NF, blocks, waves, chunk;
};

bool takes_rows(const pack4_layout &L, int T, int x_type, Rows *r)
{
    if (T > kRowsTokens) return false;
    const bool wide = x_type == OBC_F32;
    // 32 rows to a workgroup, which share the tokens in LDS, where 16 would be more than a workgroup to a compute unit (8 bits, 8 x 16384 x
    // 4096: 14.9 us, with 16 rows 17.2; 13 x 5000 x 4999: 9.9 and 13.7; the other way round 1 x 4096 x 4096: 5.1 us with 16, 6.1 with 32)
    r->NF = L.RB > 256 ? 2 : 1;
    r->blocks = (L.RB + r->NF - 1) / r->NF;
    // sixteen waves to a compute unit, in one workgroup or two; no more than there are tiles
    int waves = r->blocks > 256 || wide ? 8 : 16;
    const int room = kRowsLds / (r->blocks > 256 ? 2 : 1) / (T * (wide ? 768 : x_type == OBC_I8 ? 128 : 256));
    while (waves > 1 && (waves / 2 >= L.KT || (room < L.KT && room < waves))) waves /= 2;
    r->waves = waves;
    r->chunk = room >= L.KT ? L.KT : room / waves * waves;
    return room >= L.KT || r->blocks >= 200;
}

template <int XT>
void launch_lay(obc_ctx *ctx, const Args &a, const Lay &lay)
{
    auto blocks = [&](int team) { return (unsigned)((lay.jobs * team + 255) / 256); };
    if (lay.G <= 32) product4_lay_kernel<XT, 4><<<blocks(4), 256, 0, ctx->stream>>>(a, lay);
    else if (lay.G <= 64) product4_lay_kernel<XT, 8><<<blocks(8), 256, 0, ctx->stream>>>(a, lay);
    else if (lay.G <= 128) product4_lay_kernel<XT, 16><<<blocks(16), 256, 0, ctx->stream>>>(a, lay);
    else product4_lay_kernel<XT, 64><<<blocks(64), 256, 0, ctx->stream>>>(a, lay);
}

template <int XT, bool CENTRED, int SUB, int BM, int BN, int WM, int STAGES>
void launch_tiles(obc_ctx *ctx, const Args &a, const Tokens &tok, int y_type, int slices)
{
    product4_tiles_kernel<XT, CENTRED, SUB, BM, BN, WM, STAGES>
        <<<(unsigned)(tok.tiles * slices), tile_waves(BN) * 64, 0, ctx->stream>>>(a, tok, y_type);
}

template <int XT, bool CENTRED, int SUB, int NF>
void launch_rows(obc_ctx *ctx, const Args &a, int y_type, int waves, int chunk)
{
    const size_t tokens = (size_t)chunk * a.T * tile_bytes(XT), sums = (size_t)waves * NF * 1024;
    product4_rows_kernel<XT, CENTRED, SUB, NF><<<(a.RB + NF - 1) / NF, waves * 64, tokens > sums ? tokens : sums, ctx->stream>>>(a, y_type, chunk);
}

template <int XT, bool CENTRED, int SUB>
int launch(obc_ctx *ctx, const Args &a, int y_type, const Rows *rows, const Plan &p, void *ws)
{
    if (rows) {
        if (rows->NF == 2) launch_rows<XT, CENTRED, SUB, 2>(ctx, a, y_type, rows->waves, rows->chunk);
        else launch_rows<XT, CENTRED, SUB, 1>(ctx, a, y_type, rows->waves, rows->chunk);
        OBC_LAUNCH_CHECK(ctx, "product4_rows_kernel");
        return OBC_OK;
    }
    const int64_t blocks = (int64_t)p.mtiles * p.ntiles * p.slices, adds = ((int64_t)a.T * a.R + 255) / 256;
    const bool as_it_lies = laid_out(a.x, XT, a.ldx, a.d);
    Lay lay;
    lay.sums = (unsigned short *)((char *)ws + p.sums);
    lay.rows = as_it_lies ? nullptr : (uintx4 *)((char *)ws + p.laid);
    lay.NGP = p.NGP;
    lay.G = SUB > 1 ? 128 / SUB : a.tpg * 128;
    lay.jobs = (int64_t)a.T * a.NG;
    if (!obc_grid_fits(blocks, tile_waves(p.BN) * 64) || (p.slices > 1 && !obc_grid_fits(adds, 256)) || !obc_grid_fits(lay.jobs, 64))
        return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_product4: too many tiles");
    launch_lay<XT>(ctx, a, lay);
    OBC_LAUNCH_CHECK(ctx, "product4_lay_kernel");
    Tokens tok;
    tok.x = as_it_lies ? (const char *)a.x : (const char *)lay.rows;
    tok.ld = as_it_lies ? a.ldx * (int64_t)size_of_type(XT) : (int64_t)a.KT * (XT == OBC_I8 ? 128 : 256);
    tok.plane = a.T * tok.ld;
    tok.sums = lay.sums;
    tok.NGP = p.NGP;
    tok.mtiles = p.mtiles;
    tok.tiles = p.mtiles * p.ntiles;
    tok.per = p.per;
    tok.part = p.slices > 1 ? (float *)((char *)ws + p.part) : nullptr;
    if constexpr (XT == OBC_F32) {
        if (p.BM == 32) launch_tiles<XT, CENTRED, SUB, 32, 128, 1, 2>(ctx, a, tok, y_type, p.slices);
        else launch_tiles<XT, CENTRED, SUB, 64, 128, 1, 2>(ctx, a, tok, y_type, p.slices);
    } else {
        if (p.BM == 32) launch_tiles<XT, CENTRED, SUB, 32, 128, 1, 3>(ctx, a, tok, y_type, p.slices);
        else if (p.BM == 64) launch_tiles<XT, CENTRED, SUB, 64, 128, 1, 3>(ctx, a, tok, y_type, p.slices);
        else launch_tiles<XT, CENTRED, SUB, 128, 256, 2, 3>(ctx, a, tok, y_type, p.slices);
    }
    OBC_LAUNCH_CHECK(ctx, "product4_tiles_kernel");
    if (p.slices > 1) {
        product4_add_kernel<<<(unsigned)adds, 256, 0, ctx->stream>>>(a, tok.part, p.slices, y_type);
        OBC_LAUNCH_CHECK(ctx, "product4_add_kernel");
    }
    return OBC_OK;
}

template <int XT, bool CENTRED>
int launch_sub(obc_ctx *ctx, const Args &a, int sub, int y_type, const Rows *rows, const Plan &p, void *ws)
{
    return sub == 1   ? launch<XT, CENTRED, 1>(ctx, a, y_type, rows, p, ws)
           : sub == 2 ? launch<XT, CENTRED, 2>(ctx, a, y_type, rows, p, ws)
                      : launch<XT, CENTRED, 4>(ctx, a, y_type, rows, p, ws);
}

}  // namespace

extern "C" {

int obc_product4_workspace_bytes(int T, int R, int d, int group, int x_type, size_t *bytes)
{
    pack4_layout L;
    if (!bytes || T < 0 || R < 0 || d <= 0 || !(float_type(x_type) || x_type == OBC_I8) || !pack4_layout_of(R, d, group, &L))
        return OBC_ERR_BAD_ARG;
    Rows r;
    *bytes = T > 0 && R > 0 && !takes_rows(L, T, x_type, &r) ? plan_of(L, T, x_type).bytes : 0;
    return OBC_OK;
}

int obc_product4(obc_ctx *ctx, const void *packed, int R, int d, int group, const void *x, int x_type, const float *x_scale,
                 int T, int64_t ldx, void *y, int y_type, int64_t ldy, void *ws, size_t ws_bytes)
{
    if (!ctx) return OBC_ERR_BAD_ARG;
    if (T < 0 || R < 0 || d <= 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: bad size");
    if (!float_type(x_type) && x_type != OBC_I8) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: unknown x_type %d", x_type);
    if (!float_type(y_type)) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: y_type %d is not a floating type", y_type);
    pack4_layout L;
    if (!pack4_layout_of(R, d, group, &L))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: group (%d) is not 0, 32, 64 or a multiple of 128", group);
    if (L.NG > 1 && (int64_t)L.KT * L.tpg >= (int64_t)1 << 32)
        return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_product4: groups of %d columns in rows of %d", group, d);
    if (ldx < d || ldy < R) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_product4: leading dimension below the row's length");
    if (T == 0 || R == 0) return OBC_OK;
    if (!packed || !x || !y) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: null argument");
    if ((x_type == OBC_I8) != (x_scale != nullptr))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: x_scale goes with 8-bit inputs");
    if (((uintptr_t)packed & 15) != 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: packed is not aligned to 16 bytes");
    if (((uintptr_t)x & (size_of_type(x_type) - 1)) != 0 || ((uintptr_t)y & (size_of_type(y_type) - 1)) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: x or y is not aligned to its elements");
    Rows r;
    const Rows *const rows = takes_rows(L, T, x_type, &r) ? &r : nullptr;
    const Plan p = rows ? Plan() : plan_of(L, T, x_type);
    if (!rows) {
        // (tokens that lie as the kernel wants them need no room)
        const size_t need = laid_out(x, x_type, ldx, d) ? p.laid : p.bytes;
        if (need > 0 && (!ws || ((uintptr_t)ws & 15) != 0 || ws_bytes < need))
            return obc_fail(ctx, OBC_ERR_WORKSPACE, "obc_product4: workspace of %zu bytes needed", need);
    }
    Args a;
    a.codes = (const uintx4 *)packed;
    a.scales = (const unsigned *)((const char *)packed + L.scales);
    a.x = x; a.xs = x_scale; a.y = y;
    a.T = T; a.R = R; a.d = d; a.RB = L.RB; a.KT = L.KT; a.NG = L.NG; a.tpg = L.tpg;
    a.tpg_inv = L.tpg > 1 && L.NG > 1 ? (unsigned)(0x100000000ull / (unsigned)L.tpg) + 1u : 0u;
    a.tpg_one = L.tpg > 1 || L.NG == 1 ? 0u : ~0u;
    a.ldx = ldx; a.ldy = ldy;
    const bool fp32 = y_type == OBC_F32;
    switch (x_type) {
    case OBC_F32: return launch_sub<OBC_F32, true>(ctx, a, L.SUB, y_type, rows, p, ws);
    case OBC_F16: return fp32 ? launch_sub<OBC_F16, true>(ctx, a, L.SUB, y_type, rows, p, ws) : launch_sub<OBC_F16, false>(ctx, a, L.SUB, y_type, rows, p, ws);
    case OBC_BF16: return fp32 ? launch_sub<OBC_BF16, true>(ctx, a, L.SUB, y_type, rows, p, ws) : launch_sub<OBC_BF16, false>(ctx, a, L.SUB, y_type, rows, p, ws);
    default: return launch_sub<OBC_I8, false>(ctx, a, L.SUB, y_type, rows, p, ws);
    }
}

}  // extern "C"
