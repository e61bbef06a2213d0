// obc_product4: y = x W^T with W in 4-bit codes and a step and an offset per row and group of columns.
//
//   y[t, r] = sum_g ( delta[r, g] S - (16 delta[r, g] - offset[r, g]) s ),   S = sum_{c in g} x[t, c] (16 + code[r, c]),
//                                                                           s = sum_{c in g} x[t, c]
// The codes enter the matrix instructions as the 16-bit numbers 16 + code, exactly (8-bit inputs: as bytes, without
// the 16), so their products with 16-bit inputs are exact in fp32 and the only roundings are those of the fp32 sums; a
// group's sums start from zero and are scaled when it ends.  fp32 inputs go in as three bf16 terms.  s comes from one
// more instruction, against ones, in the very lanes that need it.
#include "product4.h"

namespace {

struct Args {
    const uintx4 *codes;
    const unsigned *scales;
    const void *x;
    const float *xs;
    void *y;
    int T, R, d, RB, KT, NG, tpg;
    int64_t ldx, ldy;
};

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

// Codes of one instruction and ones, as the operand that meets XT's.
template <int XT>
struct Codes {
    uintx4 v;
    __device__ explicit Codes(unsigned w) : v(XT == OBC_F16 ? codes_f16(w) : codes_bf16(w)) {}
    static __device__ Codes ones()
    {
        Codes c(0);
        const unsigned one = XT == OBC_F16 ? 0x3c003c00u : 0x3f803f80u;
        c.v = uintx4{one, one, one, one};
        return c;
    }
};

template <>
struct Codes<OBC_I8> {
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
    __device__ void add(const Operand<XT> &a, const Codes<XT> &b)
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
    __device__ void add(const Operand<OBC_I8> &a, const Codes<OBC_I8> &b) { s = mfma_i8(a.v, b.v, s); }
    __device__ float operator[](int i) const { return (float)s[i]; }
};

// 16 rows of W and 16 MF tokens to a workgroup whose WAVES waves take turns along the columns' tiles and sum in LDS.
template <int XT, int SUB, int MF, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void product4_rows_kernel(Args a, int y_type)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = lane & 15, quad = lane >> 4;
    const int rb = blockIdx.x;
    const int t0 = blockIdx.y * 16 * MF;
    int64_t row_at[MF];
#pragma unroll
    for (int m = 0; m < MF; ++m) {
        const int t = t0 + 16 * m + n;
        row_at[m] = (int64_t)(t < a.T ? t : a.T - 1) * a.ldx;      // rows beyond the last: their sums are not stored
    }
    float acc[MF][4];
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][i] = 0.f;
    constexpr float base = XT == OBC_I8 ? 0.f : kCodeBase;
    const Codes<XT> ones = Codes<XT>::ones();
    for (int kt = wave; kt < a.KT; kt += WAVES) {
        const uintx4 w = a.codes[((int64_t)rb * a.KT + kt) * 64 + lane];
        unsigned sc[SUB];
#pragma unroll
        for (int u = 0; u < SUB; ++u)
            sc[u] = SUB > 1 ? a.scales[(((int64_t)rb * a.KT + kt) * 16 + n) * SUB + u]
                            : a.scales[((int64_t)rb * a.NG + kt / a.tpg) * 16 + n];
#pragma unroll
        for (int m = 0; m < MF; ++m) {
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                Sum<XT> S, s;
#pragma unroll
                for (int k = u * 4 / SUB; k < (u + 1) * 4 / SUB; ++k) {
                    Operand<XT> x;
                    const int c = kt * 128 + 32 * k + 8 * quad;
                    x.load(a.x, row_at[m] + c, a.d - c);
                    S.add(x, Codes<XT>(w[k]));
                    s.add(x, ones);
                }
                const float step = half_lo(sc[u]), off = half_hi(sc[u]) - base * step;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][i] = fmaf(step, S[i], fmaf(off, s[i], acc[m][i]));
            }
        }
    }
    __shared__ float part[WAVES][MF][64][4];
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[wave][m][lane][i] = acc[m][i];
    __syncthreads();
    for (int e = threadIdx.x; e < MF * 256; e += WAVES * 64) {
        const int m = e >> 8, i = (e >> 6) & 3, l = e & 63;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += part[w][m][l][i];
        const int t = t0 + 16 * m + 4 * (l >> 4) + i, r = rb * 16 + (l & 15);
        if (t >= a.T || r >= a.R) continue;
        if (XT == OBC_I8) v *= a.xs[t];
        const int64_t at = (int64_t)t * a.ldy + r;
        if (y_type == OBC_F32) store_as<OBC_F32>(a.y, at, v);
        else if (y_type == OBC_F16) store_as<OBC_F16>(a.y, at, v);
        else store_as<OBC_BF16>(a.y, at, v);
    }
}


// ---- many tokens ------------------------------------------------------------------------------
// The tokens as product4_tiles_kernel takes them: rows at multiples of 16 bytes, columns up to a multiple of 128, zeros
// from d on; fp32 as three planes of bf16 terms.  Only where x is not like that already.
template <int XT>
__global__ __launch_bounds__(256) void product4_lay_kernel(const void *x, int64_t ldx, int d, int pieces, int64_t jobs, int64_t plane,
                                                           uintx4 *out)
{
    constexpr int E = XT == OBC_I8 ? 16 : 8;
    const int64_t job = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (job >= jobs) return;
    const int64_t t = job / pieces;
    const int c = (int)(job - t * pieces) * E;
    const int64_t at = t * ldx + c;
    if constexpr (XT == OBC_I8) {
        uintx4 v = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (c + j < d) v[j >> 2] |= (unsigned)((const uint8_t *)x)[at + j] << (8 * (j & 3));
        out[job] = v;
    } else {
        Operand<XT> o;
        o.load(x, at, d - c);
        if constexpr (XT == OBC_F32) {
            out[job] = o.v[0];
            out[job + plane] = o.v[1];
            out[job + 2 * plane] = o.v[2];
        } else {
            out[job] = o.v;
        }
    }
}

template <int V>
struct Type {
    static constexpr int value = V;
};

struct Tokens {
    const char *x;           // first plane
    int64_t ld, plane;       // bytes between rows, between planes
};

typedef __attribute__((address_space(1))) const void *global_ptr;
typedef __attribute__((address_space(3))) void *lds_ptr;

// BM tokens x 128 rows of W to a workgroup of 2 x 2 waves, BM / 2 x 64 each.  The tokens go through LDS, two tiles
// in turn; a wave's codes come straight from memory in operand order and are unpacked once for its BM / 2 tokens.
// The inputs' sums of every group are kept in LDS and meet the offsets in one fp32 product of matrices at the end.
constexpr int kWaitVm0 = 0x0f70;    // s_waitcnt vmcnt(0), the other counters not waited for
constexpr int kSumGroups = 32;      // groups whose sums LDS holds; more are worked off in between

template <int XT, int SUB, int BM>
__global__ __launch_bounds__(256, 2) void product4_tiles_kernel(Args a, Tokens tok, int y_type, int mtiles)
{
    constexpr int P = XT == OBC_F32 ? 3 : 1, MF = BM / 32;
    constexpr int ROW = XT == OBC_I8 ? 8 : 16;      // 16-byte pieces of a token's 128 columns
    // two arrays, not one of two: the compiler then knows that reading one does not wait for loads to the other
    __shared__ uintx4 even[P * BM * ROW], odd[P * BM * ROW];
    __shared__ float sums[kSumGroups][BM];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = lane & 15, quad = lane >> 4;
    const int wm = wave & 1, wn = wave >> 1;
    // consecutive workgroups go to different dies: give each die a run of tiles
    const int tiles = gridDim.x, per = tiles >> 3, left = tiles & 7, die = blockIdx.x & 7;
    const int tile = die * per + (die < left ? die : left) + (blockIdx.x >> 3);
    const int t0 = (tile % mtiles) * BM, rb0 = (tile / mtiles) * 8 + wn * 4;
    constexpr float base = XT == OBC_I8 ? 0.f : kCodeBase;
    floatx4 acc[MF][4];
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[m][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    int64_t rb[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) rb[j] = rb0 + j < a.RB ? rb0 + j : a.RB - 1;      // beyond the last: not stored
    // Piece o of token t lies at place o ^ (t mod ROW) of its row, so that the 16 tokens of an operand lie in different
    // banks.  The lanes of a load to LDS write 64 places in a row: each fetches the piece that belongs to its place.
    auto fetch = [&](int kt, uintx4 *lds) {
        constexpr int TOK = 64 / ROW;      // tokens of one load
#pragma unroll
        for (int i = 0; i < P * BM / TOK / 4; ++i) {
            const int first = (i * 4 + wave) * TOK;                  // row of the planes, one below the other
            const int p = P > 1 ? first / BM : 0, t = first - p * BM + lane / ROW;
            const int row = t0 + t < a.T ? t0 + t : a.T - 1;
            const char *src = tok.x + p * tok.plane + row * tok.ld + (int64_t)kt * (ROW * 16) + ((lane % ROW) ^ (t % ROW)) * 16;
            __builtin_amdgcn_global_load_lds((global_ptr)src, (lds_ptr)(lds + first * ROW), 16, 0, 0);
        }
    };
    auto operand = [&](const uintx4 *lds, int p, int m, int o) {
        return lds[(p * BM + 16 * m + n) * ROW + (o ^ (n & (ROW - 1)))];
    };
    // 8-bit inputs: the eight columns of step k, in the codes' order
    auto operand8 = [&](const uintx4 *lds, int m, int k) {
        const int e = 4 * k + quad;
        return bytes_like_codes(((const uintx2 *)lds)[((16 * m + n) * ROW + ((e >> 1) ^ (n & (ROW - 1)))) * 2 + (e & 1)]);
    };
    // sums x offsets of the groups [g0, g0 + count): four groups to an instruction
    auto offsets = [&](int g0, int count) {
        for (int g = 0; g < count; g += 4) {
            const bool in = g + quad < count;
            float b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                unsigned sc = 0;
                if (in) {
                    const int at = g0 + g + quad;
                    sc = SUB > 1 ? a.scales[((rb[j] * a.KT + at / SUB) * 16 + n) * SUB + at % SUB]
                                 : a.scales[(rb[j] * a.NG + at / a.tpg) * 16 + n];
                }
                b[j] = half_hi(sc) - base * half_lo(sc);
            }
#pragma unroll
            for (int m = 0; m < MF; ++m) {
                const float s = in ? sums[g + quad][wm * (BM / 2) + 16 * m + n] : 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[m][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(s, b[j], acc[m][j], 0, 0, 0);
            }
        }
    };
    uintx4 codes[4];
    unsigned scale[4][SUB];
    auto fetch_codes = [&](int kt) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            codes[j] = a.codes[(rb[j] * a.KT + kt) * 64 + lane];
#pragma unroll
            for (int u = 0; u < SUB; ++u)
                scale[j][u] = SUB > 1 ? a.scales[((rb[j] * a.KT + kt) * 16 + n) * SUB + u] : a.scales[(rb[j] * a.NG + kt / a.tpg) * 16 + n];
        }
    };
    fetch(0, even);
    fetch_codes(0);
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __syncthreads();
    int done = 0;      // tiles whose offsets are in
    auto turn = [&](const int kt, const uintx4 *lds, uintx4 *lds_next) __attribute__((always_inline)) {
        uintx4 w[4];
        float step[4][SUB];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = codes[j];
#pragma unroll
            for (int u = 0; u < SUB; ++u) step[j][u] = half_lo(scale[j][u]);
        }
        // (the last tile again after the last: a branch here would make the compiler wait for all of it at once)
        const int ahead = kt + 1 < a.KT ? kt + 1 : kt;
        fetch(ahead, lds_next);
        fetch_codes(ahead);
        // the tile's sums, a quarter of the tokens to each wave
        for (int m = wave; m < BM / 16; m += 4) {
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                Sum<XT> s;
#pragma unroll
                for (int k = u * 4 / SUB; k < (u + 1) * 4 / SUB; ++k) {
                    Operand<XT> x;
                    if constexpr (XT == OBC_F32) {
#pragma unroll
                        for (int p = 0; p < 3; ++p) x.v[p] = operand(lds, p, m, 4 * k + quad);
                    } else if constexpr (XT == OBC_I8) {
                        x.v = operand8(lds, m, k);
                    } else {
                        x.v = operand(lds, 0, m, 4 * k + quad);
                    }
                    s.add(x, Codes<XT>::ones());
                }
                if (n == 0)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sums[(kt - done) * SUB + u][16 * m + 4 * quad + i] = s[i];
            }
        }
        uintx4 B[4][XT == OBC_I8 ? 2 : 4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (XT == OBC_I8) {
                    const uintx2 c = codes_i8(w[j][k]);
                    B[j][k >> 1][2 * (k & 1)] = c.x;
                    B[j][k >> 1][2 * (k & 1) + 1] = c.y;
                } else {
                    B[j][k] = XT == OBC_F16 ? codes_f16(w[j][k]) : codes_bf16(w[j][k]);
                }
            }
#pragma unroll
        for (int m = 0; m < MF; ++m) {
            const int mm = wm * MF + m;
            if constexpr (XT == OBC_I8) {
                uintx4 A[2];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uintx2 x = operand8(lds, mm, k);
                    A[k >> 1][2 * (k & 1)] = x.x;
                    A[k >> 1][2 * (k & 1) + 1] = x.y;
                }
#pragma unroll
                for (int u = 0; u < SUB; ++u) {
                    intx4 S[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        S[j] = intx4{0, 0, 0, 0};
                        if constexpr (SUB == 4) {
                            const uintx4 x = A[u >> 1], b = B[j][u >> 1];
                            S[j] = u & 1 ? mfma_i8(uintx2{x.z, x.w}, uintx2{b.z, b.w}, S[j]) : mfma_i8(uintx2{x.x, x.y}, uintx2{b.x, b.y}, S[j]);
                        } else {
#pragma unroll
                            for (int k = u * 2 / SUB; k < (u + 1) * 2 / SUB; ++k)
                                S[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(intx4, A[k]), __builtin_bit_cast(intx4, B[j][k]), S[j], 0, 0, 0);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[m][j][i] = fmaf(step[j][u], (float)S[j][i], acc[m][j][i]);
                }
            } else {
#pragma unroll
                for (int u = 0; u < SUB; ++u) {
                    floatx4 S[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) S[j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = u * 4 / SUB; k < (u + 1) * 4 / SUB; ++k) {
#pragma unroll
                        for (int p = P - 1; p >= 0; --p) {
                            const uintx4 A = operand(lds, p, mm, 4 * k + quad);
#pragma unroll
                            for (int j = 0; j < 4; ++j) S[j] = XT == OBC_F16 ? mfma_f16(A, B[j][k], S[j]) : mfma_bf16(A, B[j][k], S[j]);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[m][j][i] = fmaf(step[j][u], S[j][i], acc[m][j][i]);
                }
            }
        }
        __builtin_amdgcn_s_waitcnt(kWaitVm0);      // the next tile is in LDS
        __syncthreads();
        if ((kt + 1 - done + 1) * SUB > kSumGroups || kt + 1 == a.KT) {
            offsets(done * SUB, (kt + 1 - done) * SUB);
            done = kt + 1;
            __syncthreads();
        }
    };
    for (int kt = 0;; kt += 2) {
        turn(kt, even, odd);
        if (kt + 1 >= a.KT) break;
        turn(kt + 1, odd, even);
        if (kt + 2 >= a.KT) break;
    }
    auto put = [&](auto type) {
        constexpr int YT = decltype(type)::value;
#pragma unroll
        for (int m = 0; m < MF; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = t0 + wm * (BM / 2) + 16 * m + 4 * quad + i;
                if (t >= a.T) continue;
                const float xs = XT == OBC_I8 ? a.xs[t] : 1.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = (rb0 + j) * 16 + n;
                    if (r < a.R) store_as<YT>(a.y, (int64_t)t * a.ldy + r, XT == OBC_I8 ? acc[m][j][i] * xs : acc[m][j][i]);
                }
            }
    };
    if (y_type == OBC_F32) put(Type<OBC_F32>());
    else if (y_type == OBC_F16) put(Type<OBC_F16>());
    else put(Type<OBC_BF16>());
}

// True where the tiles' kernel can read x as it lies.
inline bool laid_out(const void *x, int x_type, int64_t ldx, int d)
{
    return x_type != OBC_F32 && d % 128 == 0 && ((uintptr_t)x & 15) == 0 && (ldx * (int64_t)size_of_type(x_type)) % 16 == 0;
}

inline size_t laid_bytes(int T, int KT, int x_type)
{
    return (size_t)T * KT * 128 * (x_type == OBC_F32 ? 6 : x_type == OBC_I8 ? 1 : 2);
}

template <int XT, int SUB>
int launch(obc_ctx *ctx, const Args &a, int y_type, void *ws)
{
    if (a.T <= 16) {
        product4_rows_kernel<XT, SUB, 1, 8><<<dim3(a.RB, 1), 512, 0, ctx->stream>>>(a, y_type);
    } else if (a.T > 64) {
        constexpr int BM = XT == OBC_F32 ? 64 : 128;
        const int mtiles = a.T / BM + (a.T % BM != 0), ntiles = (a.RB + 7) / 8;
        if ((int64_t)mtiles * ntiles > 0x7fffffff) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_product4: too many tiles");
        Tokens tok = {(const char *)a.x, a.ldx * (int64_t)size_of_type(XT), 0};
        if (!laid_out(a.x, XT, a.ldx, a.d)) {
            const int pieces = a.KT * (XT == OBC_I8 ? 8 : 16);
            const int64_t jobs = (int64_t)a.T * pieces;
            if ((jobs + 255) / 256 > 0x7fffffff) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_product4: too many inputs");
            product4_lay_kernel<XT><<<(unsigned)((jobs + 255) / 256), 256, 0, ctx->stream>>>(a.x, a.ldx, a.d, pieces, jobs, jobs, (uintx4 *)ws);
            OBC_LAUNCH_CHECK(ctx, "product4_lay_kernel");
            tok = Tokens{(const char *)ws, (int64_t)pieces * 16, jobs * 16};
        }
        product4_tiles_kernel<XT, SUB, BM><<<mtiles * ntiles, 256, 0, ctx->stream>>>(a, tok, y_type, mtiles);
    } else {
        const int per = 64, blocks = (a.T + per - 1) / per;
        for (int b0 = 0; b0 < blocks; b0 += 65535) {
            Args c = a;
            const int64_t t0 = (int64_t)b0 * per;
            c.x = (const char *)a.x + t0 * a.ldx * (int64_t)size_of_type(XT);
            c.y = (char *)a.y + t0 * a.ldy * (int64_t)size_of_type(y_type);
            if (a.xs) c.xs = a.xs + t0;
            c.T = a.T - (int)t0;
            const int nb = blocks - b0 < 65535 ? blocks - b0 : 65535;
            product4_rows_kernel<XT, SUB, 4, 4><<<dim3(a.RB, nb), 256, 0, ctx->stream>>>(c, y_type);
        }
    }
    OBC_LAUNCH_CHECK(ctx, "product4_rows_kernel");
    return OBC_OK;
}

template <int XT>
int launch_sub(obc_ctx *ctx, const Args &a, int sub, int y_type, void *ws)
{
    return sub == 1 ? launch<XT, 1>(ctx, a, y_type, ws) : sub == 2 ? launch<XT, 2>(ctx, a, y_type, ws) : launch<XT, 4>(ctx, a, y_type, ws);
}

}  // namespace

extern "C" {

int obc_product4_workspace_bytes(int T, int R, int d, int group, int x_type, size_t *bytes)
{
    pack4_layout L;
    if (!bytes || T < 0 || R < 0 || d <= 0 || !(float_type(x_type) || x_type == OBC_I8) || !pack4_layout_of(R, d, group, &L))
        return OBC_ERR_BAD_ARG;
    // rows that are not laid out for the tiles' kernel; a workspace for T tokens serves fewer
    *bytes = T > 64 ? laid_bytes(T, L.KT, x_type) : 0;
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
    if (ldx < d || ldy < R) return obc_fail(ctx, OBC_ERR_BAD_SHAPE, "obc_product4: leading dimension below the row's length");
    if (T == 0 || R == 0) return OBC_OK;
    if (!packed || !x || !y) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: null argument");
    if ((x_type == OBC_I8) != (x_scale != nullptr))
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: x_scale goes with 8-bit inputs");
    if (((uintptr_t)packed & 15) != 0) return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: packed is not aligned to 16 bytes");
    if (((uintptr_t)x & (size_of_type(x_type) - 1)) != 0 || ((uintptr_t)y & (size_of_type(y_type) - 1)) != 0)
        return obc_fail(ctx, OBC_ERR_BAD_ARG, "obc_product4: x or y is not aligned to its elements");
    if (T > 64 && !laid_out(x, x_type, ldx, d) && (!ws || ((uintptr_t)ws & 15) != 0 || ws_bytes < laid_bytes(T, L.KT, x_type)))
        return obc_fail(ctx, OBC_ERR_WORKSPACE, "obc_product4: workspace of %zu bytes needed", laid_bytes(T, L.KT, x_type));
    Args a;
    a.codes = (const uintx4 *)packed;
    a.scales = (const unsigned *)((const char *)packed + L.scales);
    a.x = x; a.xs = x_scale; a.y = y;
    a.T = T; a.R = R; a.d = d; a.RB = L.RB; a.KT = L.KT; a.NG = L.NG; a.tpg = L.tpg;
    a.ldx = ldx; a.ldy = ldy;
    switch (x_type) {
    case OBC_F32: return launch_sub<OBC_F32>(ctx, a, L.SUB, y_type, ws);
    case OBC_F16: return launch_sub<OBC_F16>(ctx, a, L.SUB, y_type, ws);
    case OBC_BF16: return launch_sub<OBC_BF16>(ctx, a, L.SUB, y_type, ws);
    default: return launch_sub<OBC_I8>(ctx, a, L.SUB, y_type, ws);
    }
}

}  // extern "C"
