// The gated feed-forward block: both projections, the activation and the product
// in one kernel, with its backward pass (gfx950).
//
//   a = x W_g^T,  b = x W_u^T,  h = act(a) * b                       x [M][D], W [F][D]
//   da = dh * b * act'(a),  db = dh * act(a)                         (a and b computed again)
//   dx = da W_g + db W_u,   dW_g = da^T x,   dW_u = db^T x
//
// Four M D F flops forward; backward twelve, as a and b are not kept.
//
// One matrix product serves all of it.  An operand's tile is brought to LDS by
// direct loads, 128 bytes along the sum for each of its rows or columns, and is
// stored as it lies in memory: along the sum (x and the weights of the forward
// products), or across it (the weights in dx, and both operands of the weight
// gradients), where the fragments are read transposed; nothing is transposed in
// memory.  Within a tile the 16-byte pieces (across: 32-byte) are permuted by their
// row, so that the fragments' reads spread over the LDS banks.  A workgroup's tile
// of the projections holds W_g's and W_u's rows of the same inner values, dealt to the waves so that a lane ends
// up with both sums of a value: the activation needs no exchange.
//
// The product's rows (16 a fragment, four consecutive in a lane) are the inner
// values, or x's columns, and its columns the tokens, so that a lane stores four
// consecutive values of a token.
//
// What bounds it: the matrix units and the LDS reads that feed them.  16 384 x 2048 -> 2 x 5632, bf16: 608 to 617 us, 1225 to 1243 TFLOP/s
// (a library product of 8192 cubed reaches 1363), no LDS bank conflicts, 58 % of the cycles with a matrix instruction under way.
// Backward at 5003 x 1032 -> 2731, GELU: 92 us for the projections and their gradients, 77 and 75 for the two products, which
// fill 360 and 387 of the 512 places for small tiles.  da and db are rounded to the tensors' type, as their products' operands are:
// in 16-bit types dx and the weights' gradients are off by 1.4 times the rounding at the store (bf16, two-norms: 2.3e-3 for
// 1.7e-3).  In two parts each they would not be, and the two products would take twice as long, the call about 380 us for 226.
//
// Few tokens (up to 64): reading the weights bounds it.  tf_gated_rows_kernel
// streams them once, straight to registers, the sum dealt out to a workgroup's
// waves (13 tokens, 1024 -> 2 x 4096: 17 MB in 5.7 us, 3 TB/s).
#include "dma.h"
#include "ops.h"

#include <cmath>

namespace {

typedef __attribute__((ext_vector_type(4))) short g_s16x4;
typedef __attribute__((address_space(3))) g_s16x4 lds_g_s16x4;
typedef __attribute__((ext_vector_type(8))) __bf16 g_bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 g_f16x8;

// 16 bytes a lane that are not in the arrays: they read zeros from here.
__device__ __attribute__((aligned(16))) unsigned g_zeros[4];

template <class T> struct Mma;
template <> struct Mma<ElemBF16> {
    typedef g_bf16x8 F;
    static constexpr int KS = 64, KM = 32;  // values of the sum in 128 bytes; in a fragment
    static __device__ __forceinline__ o_f32x4 mma(F a, F b, o_f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Mma<ElemF16> {
    typedef g_f16x8 F;
    static constexpr int KS = 64, KM = 32;
    static __device__ __forceinline__ o_f32x4 mma(F a, F b, o_f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};
template <> struct Mma<ElemF32> {
    typedef o_f32x4 F;
    static constexpr int KS = 32, KM = 16;
    static __device__ __forceinline__ o_f32x4 mma(F a, F b, o_f32x4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

// The wave's loads into LDS have arrived and its reads are done; then the workgroup's.
__device__ __forceinline__ void stage_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// act and act'.  The 16-bit types round the result to 2^-8 or 2^-11 of itself: the hardware's exp2 and reciprocal (2^-22) do.  GELU's
// Phi(-x) = exp(-x^2 / 2) R(x), x >= 0, shares its exponential with the derivative; R, which falls from 1/2 as 0.4 / x, is a
// polynomial in 1 / (1 + 0.305 x), fitted to erfcx(x / sqrt 2) / 2 over 0 .. 14 for the smallest relative error (1e-7, in fp32's
// arithmetic 4e-7), so that the negative tail is good to its own size.
template <class T, bool GELU> __device__ __forceinline__ void act_of(float a, float &v, float &d) {
    if constexpr (GELU && sizeof(typename T::E) == 2) {
        const float t = __builtin_amdgcn_rcpf(1.0f + 0.305f * fabsf(a));
        const float e = __builtin_amdgcn_exp2f(-0.72134752044448170f * a * a);  // exp(-a^2 / 2)
        const float r = t * (0.12163974f + t * (0.122466765f + t * (0.10342119f + t * (0.12102058f + t * (-0.03797468f +
                        t * (0.18571450f + t * (-0.15298687f + t * 0.036698833f)))))));
        const float half = r * e;  // Phi(-|a|)
        const float p = a < 0.0f ? half : 1.0f - half;
        v = a * p;
        d = p + a * (0.3989422804014327f * e);
    } else if constexpr (GELU) {
        const float p = 0.5f * erfcf(a * -0.70710678118654752f);  // (1 + erf would lose the negative tail's digits)
        v = a * p;
        d = p + a * (0.3989422804014327f * expf(-0.5f * a * a));
    } else {
        float s;
        if constexpr (sizeof(typename T::E) == 4) s = 1.0f / (1.0f + expf(-a));
        else s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * a));
        v = a * s;
        d = s * (1.0f + a * (1.0f - s));
    }
}

// An operand: `rows` rows of `width` values, ld apart.  ALONG the sum: the rows are the product's rows or
// columns and the sum runs along them.  Across: the sum runs over the rows.
struct Operand {
    const void *p, *p2;  // p2: W_u where p is W_g
    long long ld;
    int rows, width;
};
struct GatedArgs {
    Operand m, n;       // tokens' side (the product's columns), inner side (its rows)
    int K, k_per;       // length of the sum; of one part of it, where it is split
    int F, Fp;          // inner values; padded
    void *out, *out2;   // h, dx, dW_g; dW_u
    long long os;
    const void *dh;
    long long ds;
    float *part;        // partial products of a split sum: [parts][M][N] fp32
    long long M, N;     // extents of the product
    int tiles_m, tiles_n;
};

enum { GATED_H = 0, GATED_D = 1, GATED_DX = 2, GATED_DW = 3 };

// The column (across: row) mapping of the tiles is that of the four products:
//   H, D:  m = x along, n = W_g and W_u along (interleaved by wave)
//   DX:    m = [da db] along, n = W_g, then W_u, across
//   DW:    m = [da db] across, n = x across
template <class T, int ROLE, int BM, int BN, int WM, int WN, bool GELU, bool SPLIT>
__global__ __launch_bounds__(64 * WM * WN, 2) void tf_gated_kernel(GatedArgs A) {
    typedef typename T::E E;
    typedef typename Mma<T>::F F;
    constexpr int NT = 64 * WM * WN, KS = Mma<T>::KS, SUBS = KS / Mma<T>::KM, ES = sizeof(E);
    constexpr bool MA = ROLE != GATED_DW, NA = ROLE == GATED_H || ROLE == GATED_D;  // along
    constexpr int WTM = BM / WM / 16, WTN = BN / WN / 16;  // a wave's tiles
    constexpr int LM = BM * 8 / NT, LN = BN * 8 / NT;      // 16-byte pieces a thread brings of each operand
    static_assert(LM * NT == BM * 8 && LN * NT == BN * 8, "pieces");
    constexpr int STAGE = (BM + BN) * 128;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int wm = wave / WN, wn = wave % WN, n = lane % 16, q = lane / 16;

    // Tiles are dealt to the XCDs (workgroup i runs on XCD i % 8) in runs, and within a run eight token tiles go through
    // the inner tiles together, so that an XCD's L2 is asked for the same operands.
    const int tiles = A.tiles_m * A.tiles_n;
    int tile = blockIdx.x;
    {
        const int per = tiles / 8, more = tiles % 8, x = tile % 8;
        tile = x * per + (x < more ? x : more) + tile / 8;
        constexpr int G = 8;
        const int group = tile / (G * A.tiles_n), first = group * G;
        const int size = A.tiles_m - first < G ? A.tiles_m - first : G, in = tile - group * G * A.tiles_n;
        tile = (in / size) * A.tiles_m + first + in % size;
    }
    const int tm = tile % A.tiles_m, tn = tile / A.tiles_m;
    const long long m0 = (long long)tm * BM;
    const int k_begin = SPLIT ? blockIdx.y * A.k_per : 0;
    const int k_end = SPLIT ? (A.K - k_begin < A.k_per ? A.K : k_begin + A.k_per) : A.K;
    const int steps = (k_end - k_begin + KS - 1) / KS;

    // Where each piece comes from: a scalar that moves along the sum, and an offset of the lane's own (32 bits: at most 256
    // rows of 2^20 values).  Rows and columns past the end are read as the last ones; what they give is not stored.
    unsigned mo[LM], no[LN];
    int mk[LM], nk[LN];  // the piece's first place along the sum within a step
    auto across_of = [&](int piece, int cols, int &row, int &col) {
        const int per = cols * ES / 16, slot = piece % per;
        row = piece / per;
        if constexpr (ES == 2) {
            const int g = (row & 3) | ((row >> 3) & 1) << 2;
            col = ((((slot >> 1) ^ g) << 1) | (slot & 1)) * 8;
        } else {
            const int g = (row >> 2) & 3;
            col = ((((slot >> 2) ^ g) << 2) | (slot & 3)) * 4;
        }
    };
    const long long n0 = (long long)tn * BN;
    const int f0 = tn * (BN / 2) < A.F ? tn * (BN / 2) : A.F - 1;  // (the padding's tiles read the last inner value)
#pragma unroll
    for (int i = 0; i < LM; ++i) {
        const int piece = i * NT + tid;
        if constexpr (MA) {
            const int row = piece / 8, chunk = (piece % 8) ^ (row & 7);
            const int r = m0 + row < A.m.rows ? row : (int)(A.m.rows - 1 - m0);
            mk[i] = chunk * (16 / ES);
            mo[i] = (unsigned)r * (unsigned)A.m.ld * ES + chunk * 16;
        } else {
            int row, col;
            across_of(piece, BM, row, col);
            const long long last = A.m.width - 16 / ES - m0;
            mk[i] = row;
            mo[i] = (unsigned)row * (unsigned)A.m.ld * ES + (unsigned)(col < last ? col : (int)last) * ES;
        }
    }
#pragma unroll
    for (int i = 0; i < LN; ++i) {
        const int piece = i * NT + tid;
        if constexpr (NA) {
            constexpr int per = BN / WN, half = per / 2;
            const int row = piece / 8, chunk = (piece % 8) ^ (row & 7), in = row % per;
            const int f = row / per * half + in % half, r = f0 + f < A.F ? f : A.F - 1 - f0;
            nk[i] = chunk * (16 / ES);
            no[i] = (unsigned)r * (unsigned)A.n.ld * ES + chunk * 16;
        } else {
            int row, col;
            across_of(piece, BN, row, col);
            const long long last = A.n.width - 16 / ES - n0;
            nk[i] = row;
            no[i] = (unsigned)row * (unsigned)A.n.ld * ES + (unsigned)(col < last ? col : (int)last) * ES;
        }
    }
    const char *mb = (const char *)A.m.p + (MA ? m0 * A.m.ld : m0) * ES;
    const long long m_step = MA ? ES : A.m.ld * ES, n_step = NA ? ES : A.n.ld * ES;  // bytes from one place along the sum to the next
    const char *nb = (const char *)A.n.p + (NA ? (long long)f0 * A.n.ld : n0) * ES, *nb2 = nullptr;
    if (ROLE != GATED_DW) nb2 = (const char *)A.n.p2 + (NA ? (long long)f0 * A.n.ld : n0) * ES;
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char *)smem;
    auto bring = [&](int step, int slot) {
        const int k0 = k_begin + step * KS;
        const unsigned to = lds0 + slot * STAGE + wave * 1024;
        const char *m = mb + k0 * m_step, *n = nb + k0 * n_step, *n2 = nb2;
        int f = k0;  // DX: the inner value (its sum runs over W_g's, then W_u's; both are padded to whole steps)
        if constexpr (NA) n2 += k0 * n_step;
        if constexpr (ROLE == GATED_DX) {
            if (k0 >= A.Fp) f = k0 - A.Fp, n = nb2 + f * n_step;
        }
        const bool whole = k0 + KS <= k_end && (ROLE != GATED_DX || f + KS <= A.F);
        if (whole) {
#pragma unroll
            for (int i = 0; i < LM; ++i) lds_dma16(m, mo[i], to + i * NT * 16);
#pragma unroll
            for (int i = 0; i < LN; ++i) {
                // (which weight a piece is of is the same for the whole wave: 8 rows of 16, 32 or 64)
                const bool up = NA && __builtin_amdgcn_readfirstlane((i * NT + tid) / 8 % (BN / WN)) >= BN / WN / 2;
                lds_dma16(up ? n2 : n, no[i], to + BM * 128 + i * NT * 16);
            }
        } else {
#pragma unroll
            for (int i = 0; i < LM; ++i) {
                const void *src = m + mo[i];
                if (k0 + mk[i] >= k_end) src = g_zeros;
                lds_dma16(src, to + i * NT * 16);
            }
#pragma unroll
            for (int i = 0; i < LN; ++i) {
                const bool up = NA && (i * NT + tid) / 8 % (BN / WN) >= BN / WN / 2;
                const void *src = (up ? n2 : n) + no[i];
                if (k0 + nk[i] >= k_end || (ROLE == GATED_DX && f + nk[i] >= A.F)) src = g_zeros;
                lds_dma16(src, to + BM * 128 + i * NT * 16);
            }
        }
    };
    auto frag = [&](const char *tile, bool along, int cols, int t, int sub) -> F {
        if (along) return *(const F *)(tile + (16 * t + n) * 128 + (((4 * sub + q) ^ (n & 7)) << 4));
        if constexpr (ES == 2) {
            const int g = (n >> 2) | (q & 1) << 2;
            const char *p = tile + (32 * sub + 8 * q + (n >> 2)) * cols * 2 + ((t ^ g) << 5) + (n & 3) * 8;
            const g_s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_g_s16x4 *)p);
            const g_s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_g_s16x4 *)(p + 4 * cols * 2));
            return __builtin_bit_cast(F, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            F f;
            const char *p = tile + (16 * sub + 4 * q) * cols * 4 + ((t ^ q) << 6) + n * 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = *(const float *)(p + i * cols * 4);
            return f;
        }
    };

    o_f32x4 acc[WTN][WTM];
#pragma unroll
    for (int i = 0; i < WTN; ++i)
#pragma unroll
        for (int j = 0; j < WTM; ++j) acc[i][j] = o_f32x4{0.f, 0.f, 0.f, 0.f};
    if (steps > 0) bring(0, 0);
    for (int s = 0; s < steps; ++s) {
        stage_barrier();
        if (s + 1 < steps) bring(s + 1, (s + 1) & 1);
        const char *tm_ = smem + (s & 1) * STAGE, *tn_ = tm_ + BM * 128;
        F fn[SUBS][WTN];
#pragma unroll
        for (int i = 0; i < SUBS * WTN; ++i) fn[i / WTN][i % WTN] = frag(tn_, NA, BN, wn * WTN + i % WTN, i / WTN);
        in_turn<SUBS * WTM, 4>([&](int i) { return frag(tm_, MA, BM, wm * WTM + i % WTM, i / WTM); },
                               [&](int i, F fm) {
#pragma unroll
                                   for (int e = 0; e < WTN; ++e)
                                       acc[e][i % WTM] = Mma<T>::mma(fn[i / WTM][e], fm, acc[e][i % WTM]);
                               });
    }

    typedef __attribute__((ext_vector_type(4))) E E4;
    // Four values at any element's address: one access, whether it is aligned or not (rows of odd length: dh read value by
    // value, or through LDS, cost a product of 5003 x 1032 -> 2731 36 us).
    typedef E4 __attribute__((aligned(sizeof(E)))) E4u;
    auto put = [&](E *p, int left, o_f32x4 v) {  // up to `left` of them
        const E4 e = __builtin_convertvector(v, E4);
        if (left >= 4) *(E4u *)p = e;
        else
            for (int i = 0; i < 4; ++i)
                if (i < left) p[i] = e[i];
    };
    if constexpr (NA) {
        constexpr int HT = WTN / 2;
        struct Row {
            E4 g[HT];
        };
        // all of dh's tile is on its way before the first of it is used
        auto read = [&](int j) {
            Row r = {};
            if constexpr (ROLE == GATED_D) {
                long long m = m0 + 16 * (wm * WTM + j) + n;
                if (m >= A.M) m = A.M - 1;
#pragma unroll
                for (int i = 0; i < HT; ++i) {
                    const int f = tn * (BN / 2) + 16 * (wn * HT + i) + 4 * q;
                    const E *p = (const E *)A.dh + m * A.ds;
                    if (f + 4 <= A.F) r.g[i] = *(const E4u *)(p + f);
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e) r.g[i][e] = p[f + e < A.F ? f + e : A.F - 1];
                }
            }
            return r;
        };
        in_turn<WTM, WTM + 1>(read, [&](int j, const Row &row) {
            const long long m = m0 + 16 * (wm * WTM + j) + n;
            if (m >= A.M) return;
#pragma unroll
            for (int i = 0; i < HT; ++i) {
                const int f = tn * (BN / 2) + 16 * (wn * HT + i) + 4 * q, left = A.F - f;
                const o_f32x4 a = acc[i][j], b = acc[i + HT][j];
                o_f32x4 v, d;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x, y;
                    act_of<T, GELU>(a[e], x, y);
                    v[e] = x, d[e] = y;
                }
                if constexpr (ROLE == GATED_H) {
                    if (left > 0) put((E *)A.out + m * A.os + f, left, v * b);
                } else {
                    if (f >= A.Fp) continue;
                    const o_f32x4 g = __builtin_convertvector(row.g[i], o_f32x4);
                    o_f32x4 da = g * b * d, db = g * v;
#pragma unroll
                    for (int e = 0; e < 4; ++e)  // the padding is zeros whatever the sums of the clamped rows are
                        if (e >= left) da[e] = db[e] = 0.0f;
                    E *o = (E *)A.out + m * A.os + f;
                    put(o, 4, da);
                    put(o + A.Fp, 4, db);
                }
            }
        });
    } else {
#pragma unroll
        for (int j = 0; j < WTM; ++j) {
            const long long m = m0 + 16 * (wm * WTM + j) + n;
            if (m >= A.M) continue;
#pragma unroll
            for (int i = 0; i < WTN; ++i) {
                const long long c = (long long)tn * BN + 16 * (wn * WTN + i) + 4 * q;
                const int left = (int)(A.N - c);
                if (left <= 0) continue;
                if constexpr (SPLIT) {  // N is a multiple of 8
                    *(o_f32x4 *)(A.part + ((long long)blockIdx.y * A.M + m) * A.N + c) = acc[i][j];
                } else if constexpr (ROLE == GATED_DX) {
                    put((E *)A.out + m * A.os + c, left, acc[i][j]);
                } else {
                    const int f = m < A.Fp ? (int)m : (int)m - A.Fp;
                    if (f < A.F) put((E *)(m < A.Fp ? A.out : A.out2) + f * A.os + c, left, acc[i][j]);
                }
            }
        }
    }
}

// The parts of a split sum, added in order, to dx (or dW_g and dW_u).
template <class T>
__global__ __launch_bounds__(256) void tf_gated_join_kernel(const float *__restrict__ part, int parts, long long M, long long N, int F, int Fp,
                                                            bool weights, void *out, void *out2, long long os) {
    typedef typename T::E E;
    const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= M * N) return;
    const long long m = i / N, c = i - m * N;
    E *p;
    if (weights) {
        const int f = m < Fp ? (int)m : (int)m - Fp;
        if (f >= F) return;
        p = (E *)(m < Fp ? out : out2) + f * os + c;
    } else {
        p = (E *)out + m * os + c;
    }
    o_f32x4 v = *(const o_f32x4 *)(part + i);
    for (int s = 1; s < parts; ++s) v += *(const o_f32x4 *)(part + (long long)s * M * N + i);
    typedef __attribute__((ext_vector_type(4))) E E4;
    *(E4 *)p = __builtin_convertvector(v, E4);
}

// Up to 16 MT tokens.  A workgroup has 16 inner values, its waves a part of the sum each.
constexpr int kRowWaves = 8;
template <class T, int MT, bool BACK, bool GELU>
__global__ __launch_bounds__(64 * kRowWaves) void tf_gated_rows_kernel(GatedArgs A) {
    typedef typename T::E E;
    typedef typename Mma<T>::F F;
    constexpr int KM = Mma<T>::KM, VEC = 16 / sizeof(E);
    __shared__ o_f32x4 sums[kRowWaves][2][MT][64];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, n = lane % 16, q = lane / 16;
    const int f0 = blockIdx.x * 16;
    const int fr = f0 + n < A.F ? f0 + n : A.F - 1;
    const E *wg = (const E *)A.n.p + (long long)fr * A.n.ld, *wu = (const E *)A.n.p2 + (long long)fr * A.n.ld;
    const E *xp[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) {
        const int r = 16 * j + n < A.m.rows ? 16 * j + n : A.m.rows - 1;
        xp[j] = (const E *)A.m.p + (long long)r * A.m.ld;
    }
    o_f32x4 acc[2][MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[0][j] = acc[1][j] = o_f32x4{0.f, 0.f, 0.f, 0.f};
    const F zero = {};
#pragma unroll 4
    for (int k0 = wave * KM; k0 < A.K; k0 += kRowWaves * KM) {
        const int k = k0 + VEC * q;
        const bool in = k < A.K;
        const F a = in ? *(const F *)(wg + k) : zero, b = in ? *(const F *)(wu + k) : zero;
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            const F x = in ? *(const F *)(xp[j] + k) : zero;
            acc[0][j] = Mma<T>::mma(a, x, acc[0][j]);
            acc[1][j] = Mma<T>::mma(b, x, acc[1][j]);
        }
    }
#pragma unroll
    for (int j = 0; j < MT; ++j) sums[wave][0][j][lane] = acc[0][j], sums[wave][1][j][lane] = acc[1][j];
    __syncthreads();
    for (int i = wave; i < MT; i += kRowWaves) {
        o_f32x4 a = sums[0][0][i][lane], b = sums[0][1][i][lane];
        for (int w = 1; w < kRowWaves; ++w) a += sums[w][0][i][lane], b += sums[w][1][i][lane];
        const int m = 16 * i + n;
        if (m >= A.M) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int f = f0 + 4 * q + e;
            float v, d;
            act_of<T, GELU>(a[e], v, d);
            if (!BACK) {
                if (f < A.F) ((E *)A.out)[m * A.os + f] = (E)(v * b[e]);
            } else if (f < A.Fp) {
                const float g = f < A.F ? (float)((const E *)A.dh)[m * A.ds + f] : 0.0f;
                E *o = (E *)A.out + m * A.os + f;
                o[0] = f < A.F ? (E)(g * b[e] * d) : (E)0.0f;
                o[A.Fp] = f < A.F ? (E)(g * v) : (E)0.0f;
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------------

constexpr int kFewRows = 64;

tf_status gated_check(const tf_gated_config *c, int64_t n_rows) {
    if (!c || !elem_ok(c->elem) || c->width < 1 || c->inner < 1 || n_rows < 0) return TF_EINVAL;
    if (c->activation != TF_ACT_SILU && c->activation != TF_ACT_GELU) return TF_EINVAL;
    if (c->width % 8 || c->width > (1 << 20) || c->inner > (1 << 20) || n_rows > (1 << 28)) return TF_EUNSUPPORTED;
    return TF_OK;
}
// A tile's rows are addressed by 32-bit offsets, its workgroups by 31-bit numbers.
bool gated_fits(const tf_gated_config *c, int64_t n_rows, std::initializer_list<int64_t> strides) {
    if (!strides_fit(strides, 1 << 22)) return false;
    const int64_t inner = (c->inner + 63) / 64, rows = (n_rows + 127) / 128, width = (c->width + 127) / 128;
    return inner * rows <= INT32_MAX && 2 * inner * width <= INT32_MAX && rows * width <= INT32_MAX;
}
int64_t gated_pad(const tf_gated_config *c) { return ((int64_t)c->inner + 63) / 64 * 64; }

// The tiles of a product of m x n: 256 x 256, one workgroup of eight waves a compute unit, or 128 x 128, two of four waves,
// each with a ring of two stages (and 64 x 64 for few tiles, below).  16-bit types: whole rounds of the compute units' tiles are
// paid for; a round of pairs of small tiles takes 0.62 of one of large ones, for half its products.  5003 x 1032 with sums of 5504:
// 77 us in small tiles, 126 in large ones; 256 x 128 with three stages and 128 x 128 with four, one workgroup a compute unit: 88
// and 124.  Forward and backward at 43 shapes of 1500 to 14 000 rows, 512 to 2048 -> 1024 to 5600, the rule is level with the
// better of the two on average and 10 % over it at worst, where small tiles alone lose up to 16 and large ones alone up to 57 %.
// fp32, whose products take sixteen times as long: small tiles, as fast or faster at all of 28 shapes (700 x 1024 -> 2 x 5600
// forward: 193 us for 242).
constexpr int kShapes[3] = {256, 128, 64};
constexpr double kRound[2] = {1.0, 0.62};
// Tiles of 128 x 128 up to which the projections, whose sums are not split, take 64 x 64 (up to five workgroups a compute unit):
// 1024 -> 2 x 4096, bf16, 128 rows (64 tiles) 7.8 us for 12.6, 300 rows (192) 12.0 for 13.5, 400 rows (256) 14.6 for 14.1; fp32,
// whose products take sixteen times as long, 128 rows 26 us for 72, 600 (320) 98 for 123, 800 (448) 119 for 124.
template <class T> constexpr int64_t kFewTiles = sizeof(typename T::E) == 4 ? 512 : 192;
int64_t gated_tiles(int64_t m, int64_t n, int shape) {
    const int b = kShapes[shape];
    return ((m + b - 1) / b) * ((n + b - 1) / b);
}
int gated_shape(int64_t m, int64_t n) {
    const int64_t large = gated_tiles(m, n, 0), small = gated_tiles(m, n, 1);
    return (double)((large + 255) / 256) * kRound[0] <= (double)((small + 511) / 512) * kRound[1] ? 0 : 1;
}
// Parts of a sum of length k over `tiles` tiles of 128 x 128: as many as give every compute unit two workgroups,
// each so long that its products take longer than its fp32 part's way out and back: 512, of fp32's slower ones 64.  Backward
// in fp32, 192 -> 2 x 512, 200 rows: 38 us with 64, 68 with 512; in bf16, 1024 -> 2 x 4096, 200 rows: 43 us with 512, 49 with 256.
int gated_parts(int64_t tiles, int64_t k, int elem) {
    const int64_t least = elem == TF_ELEM_FP32 ? 64 : 512;
    int64_t p = 512 / (tiles < 1 ? 1 : tiles);
    if (p > k / least) p = k / least;
    if (p > 32) p = 32;
    return p < 1 ? 1 : (int)p;
}

struct GatedPlan {
    int64_t fp, dx_parts, dw_parts;
    size_t dgu, part, bytes;
};
GatedPlan gated_plan(const tf_gated_config *c, int64_t m) {
    GatedPlan p = {};
    p.fp = gated_pad(c);
    p.dx_parts = gated_parts(gated_tiles(m, c->width, 1), 2 * p.fp, c->elem);
    p.dw_parts = gated_parts(gated_tiles(2 * p.fp, c->width, 1), m, c->elem);
    p.dgu = ((size_t)m * 2 * p.fp * elem_bytes(c->elem) + 255) / 256 * 256;
    const size_t a = p.dx_parts > 1 ? (size_t)p.dx_parts * m * c->width * 4 : 0;
    const size_t b = p.dw_parts > 1 ? (size_t)p.dw_parts * 2 * p.fp * c->width * 4 : 0;
    p.part = a > b ? a : b;
    p.bytes = p.dgu + p.part;
    return p;
}

template <class T, int ROLE, int SHAPE, bool GELU, bool SPLIT> void gated_tile(GatedArgs A, int parts, hipStream_t s) {
    constexpr int BM = kShapes[SHAPE], BN = BM, WM = 2, WN = SHAPE == 0 ? 4 : 2, LDS = 2 * (BM + BN) * 128;
    constexpr int inner = ROLE == GATED_H || ROLE == GATED_D ? BN / 2 : BN;  // inner values of a tile
    A.tiles_m = (int)((A.M + BM - 1) / BM);
    A.tiles_n = (int)((A.N + inner - 1) / inner);
    auto kernel = tf_gated_kernel<T, ROLE, BM, BN, WM, WN, GELU, SPLIT>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)A.tiles_m * A.tiles_n), SPLIT ? parts : 1), dim3(64 * WM * WN), LDS, s, A);
}
template <class T, int ROLE, bool GELU> void gated_product(const GatedArgs &A, int parts, hipStream_t s) {
    if constexpr (ROLE == GATED_DX || ROLE == GATED_DW) {
        if (parts > 1) {
            gated_tile<T, ROLE, 1, GELU, true>(A, parts, s);
            const int64_t blocks = (A.M * A.N / 4 + 255) / 256;
            hipLaunchKernelGGL((tf_gated_join_kernel<T>), dim3((unsigned)blocks), dim3(256), 0, s, A.part, parts, A.M, A.N, A.F, A.Fp,
                               ROLE == GATED_DW, A.out, A.out2, A.os);
            return;
        }
    }
    const int64_t n = ROLE == GATED_H || ROLE == GATED_D ? 2 * A.N : A.N;
    if constexpr (ROLE == GATED_H || ROLE == GATED_D) {
        if (gated_tiles(A.M, n, 1) <= kFewTiles<T>) {
            gated_tile<T, ROLE, 2, GELU, false>(A, 1, s);
            return;
        }
    }
    if constexpr (sizeof(typename T::E) == 2) {
        if (gated_shape(A.M, n) == 0) {
            gated_tile<T, ROLE, 0, GELU, false>(A, 1, s);
            return;
        }
    }
    gated_tile<T, ROLE, 1, GELU, false>(A, 1, s);
}
template <class T, bool BACK, bool GELU> void gated_project(const GatedArgs &A, hipStream_t s) {
    if (A.M <= kFewRows) {
        const dim3 grid((unsigned)(((BACK ? A.Fp : A.F) + 15) / 16)), block(64 * kRowWaves);
        if (A.M <= 16) hipLaunchKernelGGL((tf_gated_rows_kernel<T, 1, BACK, GELU>), grid, block, 0, s, A);
        else if (A.M <= 32) hipLaunchKernelGGL((tf_gated_rows_kernel<T, 2, BACK, GELU>), grid, block, 0, s, A);
        else hipLaunchKernelGGL((tf_gated_rows_kernel<T, 4, BACK, GELU>), grid, block, 0, s, A);
        return;
    }
    gated_product<T, BACK ? GATED_D : GATED_H, GELU>(A, 1, s);
}
template <class T> void gated_forward(const tf_gated_config *c, const GatedArgs &A, hipStream_t s) {
    if (c->activation == TF_ACT_GELU) gated_project<T, false, true>(A, s);
    else gated_project<T, false, false>(A, s);
}
template <class T> void gated_backward(const tf_gated_config *c, const GatedArgs &P, const GatedArgs &X, const GatedArgs &W, const GatedPlan &p, hipStream_t s) {
    if (c->activation == TF_ACT_GELU) gated_project<T, true, true>(P, s);
    else gated_project<T, true, false>(P, s);
    gated_product<T, GATED_DX, false>(X, (int)p.dx_parts, s);
    gated_product<T, GATED_DW, false>(W, (int)p.dw_parts, s);
}

}  // namespace

extern "C" tf_status tf_gated_ffn(const tf_gated_config *c, const void *x, int64_t x_stride, int64_t n_rows, const void *w_gate,
                                  const void *w_up, int64_t w_stride, void *out, int64_t out_stride, hipStream_t stream) {
    const tf_status st = gated_check(c, n_rows);
    if (st != TF_OK) return st;
    if (!stride_ok(x_stride, c->width, c->elem) || !stride_ok(w_stride, c->width, c->elem) || out_stride < c->inner) return TF_EINVAL;
    if (!gated_fits(c, n_rows, {x_stride, w_stride})) return TF_EUNSUPPORTED;
    if (n_rows == 0) return TF_OK;
    if (!x || !w_gate || !w_up || !out) return TF_EINVAL;
    if (!aligned16(x) || !aligned16(w_gate) || !aligned16(w_up) || ((uintptr_t)out & (elem_bytes(c->elem) - 1))) return TF_EINVAL;
    if (over_inputs({out}, {x, w_gate, w_up})) return TF_EINVAL;
    GatedArgs A = {};
    A.m = {x, nullptr, x_stride, (int)n_rows, c->width};
    A.n = {w_gate, w_up, w_stride, c->inner, c->width};
    A.K = c->width, A.F = c->inner, A.Fp = (int)gated_pad(c), A.out = out, A.os = out_stride, A.M = n_rows, A.N = c->inner;
    if (c->elem == TF_ELEM_BF16) gated_forward<ElemBF16>(c, A, stream);
    else if (c->elem == TF_ELEM_FP32) gated_forward<ElemF32>(c, A, stream);
    else gated_forward<ElemF16>(c, A, stream);
    return hipGetLastError() == hipSuccess ? TF_OK : TF_EHIP;
}

extern "C" size_t tf_gated_ffn_workspace_size(const tf_gated_config *c, int64_t n_rows) {
    if (gated_check(c, n_rows) != TF_OK) return 0;
    const size_t b = gated_plan(c, n_rows).bytes;
    return b ? b : 256;
}

extern "C" tf_status tf_gated_ffn_backward(const tf_gated_config *c, const void *d_out, int64_t d_out_stride, const void *x,
                                           int64_t x_stride, int64_t n_rows, const void *w_gate, const void *w_up, int64_t w_stride,
                                           void *workspace, size_t workspace_bytes, void *dx, int64_t dx_stride, void *dw_gate,
                                           void *dw_up, int64_t dw_stride, hipStream_t stream) {
    const tf_status st = gated_check(c, n_rows);
    if (st != TF_OK) return st;
    if (!stride_ok(x_stride, c->width, c->elem) || !stride_ok(w_stride, c->width, c->elem) || !stride_ok(dx_stride, c->width, c->elem) ||
        !stride_ok(dw_stride, c->width, c->elem) || d_out_stride < c->inner)
        return TF_EINVAL;
    if (!gated_fits(c, n_rows, {x_stride, w_stride, dx_stride, dw_stride})) return TF_EUNSUPPORTED;
    if (!w_gate || !w_up || !dw_gate || !dw_up || !workspace) return TF_EINVAL;
    if (n_rows > 0 && (!d_out || !x || !dx)) return TF_EINVAL;
    if (!aligned16(x) || !aligned16(w_gate) || !aligned16(w_up) || !aligned16(dx) || !aligned16(dw_gate) || !aligned16(dw_up) ||
        !aligned16(workspace) || ((uintptr_t)d_out & (elem_bytes(c->elem) - 1)))
        return TF_EINVAL;
    if ((n_rows > 0 && over_inputs({dx, dw_gate, dw_up, workspace}, {d_out, x})) ||
        over_inputs({dx, dw_gate, dw_up, workspace}, {w_gate, w_up}) || twice({dx, dw_gate, dw_up, workspace}))
        return TF_EINVAL;
    const GatedPlan p = gated_plan(c, n_rows);
    if (workspace_bytes < p.bytes) return TF_EINVAL;
    float *part = (float *)((char *)workspace + p.dgu);
    GatedArgs P = {};  // [da db], rows of 2 Fp
    P.m = {x, nullptr, x_stride, (int)n_rows, c->width};
    P.n = {w_gate, w_up, w_stride, c->inner, c->width};
    P.K = c->width, P.F = c->inner, P.Fp = (int)p.fp, P.out = workspace, P.os = 2 * p.fp, P.dh = d_out, P.ds = d_out_stride;
    P.M = n_rows, P.N = p.fp;
    GatedArgs X = {};
    X.m = {workspace, nullptr, 2 * p.fp, (int)n_rows, (int)(2 * p.fp)};
    X.n = {w_gate, w_up, w_stride, c->inner, c->width};
    X.K = (int)(2 * p.fp), X.F = c->inner, X.Fp = (int)p.fp, X.out = dx, X.os = dx_stride, X.M = n_rows, X.N = c->width, X.part = part;
    X.k_per = (int)((X.K / 64 + p.dx_parts - 1) / p.dx_parts * 64);
    GatedArgs W = {};
    W.m = {workspace, nullptr, 2 * p.fp, (int)n_rows, (int)(2 * p.fp)};
    W.n = {x, nullptr, x_stride, (int)n_rows, c->width};
    W.K = (int)n_rows, W.F = c->inner, W.Fp = (int)p.fp, W.out = dw_gate, W.out2 = dw_up, W.os = dw_stride;
    W.M = 2 * p.fp, W.N = c->width, W.part = part;
    W.k_per = (int)(((n_rows + 63) / 64 + p.dw_parts - 1) / p.dw_parts * 64);
    if (n_rows == 0) {
        // no tokens: the weights' gradients are zeros (a product over an empty sum)
        if (c->elem == TF_ELEM_BF16) gated_product<ElemBF16, GATED_DW, false>(W, 1, stream);
        else if (c->elem == TF_ELEM_FP32) gated_product<ElemF32, GATED_DW, false>(W, 1, stream);
        else gated_product<ElemF16, GATED_DW, false>(W, 1, stream);
    } else if (c->elem == TF_ELEM_BF16) gated_backward<ElemBF16>(c, P, X, W, p, stream);
    else if (c->elem == TF_ELEM_FP32) gated_backward<ElemF32>(c, P, X, W, p, stream);
    else gated_backward<ElemF16>(c, P, X, W, p, stream);
    return hipGetLastError() == hipSuccess ? TF_OK : TF_EHIP;
}
