// Linear attention with a decay for each head over packed sequences (gfx950):
//
//   S_t = exp(g_t) S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t            (each sequence and head)
//
// with its backward pass and its form for single tokens.  In chunks of 64 rows,
// with b the running sum of g,
//
//   o_t = scale (sum over s <= t of exp(b_t - b_s) (q_t k_s) v_s  +  exp(b_t) S_in^T q_t)
//   S_out = exp(b_end) S_in + sum over s of exp(b_end - b_s) k_s v_s^T
//
// so that all of it is matrix products.  Only differences b_t - b_s within one
// sequence are ever exponentiated; with g <= 0 none of them overflows.
//
// The gradients are the same function of other arguments: with U_t the gradient
// of S_t, which runs the other way,
//
//   dq_t = scale S_t do_t                                 q, k, v <- do, v, k    (S transposed)
//   dv_s = U_s^T k_s                                      q, k, v <- k, q, do    (from the last row)
//   dk_s = U_s v_s                                        q, k, v <- v, do, q    (from the last row)
//   U_s = scale q_s do_s^T + exp(g_{s+1}) U_{s+1}
//
// (in that direction a row's decay is its predecessor's: `shift`), and with
// db_t = q_t dq_t - k_t dk_t the gradient of g_t is the sum of db over the
// sequence's rows from t on, plus <dS_last, S_last>.  What both terms of db have
// of the same pair of rows, or of the same row and dS_last, is one number, taken
// away in fp64, so that a head that forgets at once keeps its digits.
//
// How the rows are split.  Sequences may be a handful of rows or tens of
// thousands, and the host does not know their lengths.  So the packed rows are cut
// into spans of equal length, whatever sequences they hold: chunks of a span hold
// rows of several sequences, whose products are masked apart.  A span border within
// 64 rows of an end of its sequence moves there; only the others cut a sequence, and
// for these a first launch computes each span's own contribution to the state at its
// end, and a second joins them in order.  With tracks of up to 64 hits no border
// cuts a sequence and these two launches end at once.
//
// Numbers.  bf16 tensors: the products q k^T, and the states' products, take bf16
// operands that are the tensors themselves, or fp32 values as bf16 parts: three in
// states and in everything that reaches the decays' gradient (all 24 bits), two
// (2^-17 of them is lost) where the result is only rounded to bf16, the states and the
// weights exp(b_t - b_s) (q_t k_s) of the outputs.  (Weights of one part: 65 536 tracks
// 344 us for 358, but outputs off by a quarter to two fifths more than their rounding.)
// fp32 and fp16 tensors are multiplied by the fp32 instruction.
#include "ops.h"

#include <cmath>
#include <initializer_list>

namespace {

constexpr int kChunk = 64;
constexpr int span_threads(int dv) { return dv == 128 ? 512 : 256; }
constexpr int kMinSpan = 2 * kChunk;  // borders move by less than a chunk: their order stays
constexpr float kForget = -200.0f;    // exp of this and less is 0: smaller log decays, -inf too, count as it
typedef __attribute__((ext_vector_type(4))) short o_s16x4;
typedef __attribute__((ext_vector_type(4))) __bf16 o_bf16x4;
typedef __attribute__((ext_vector_type(8))) __bf16 o_bf16x8;
typedef __attribute__((ext_vector_type(4))) _Float16 o_f16x4;
typedef __attribute__((address_space(3))) o_s16x4 lds_s16x4;

// The matrix-core side.  A fragment of an operand is 16 bytes a lane: row (or column) lane % 16,
// and 8 (bf16) or 4 (fp32) of KM values along the sum for the lane group lane / 16.
struct MatBF16 {
    typedef __bf16 E;
    typedef o_bf16x8 F;
    static constexpr int KM = 32, PAD = 8;
    static __device__ __forceinline__ o_f32x4 mma(F a, F b, o_f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    // the sum runs along x's rows: x[row][k0 ..]
    static __device__ __forceinline__ F along(const E *x, int ld, int row, int k0, int q) {
        return *(const F *)(x + row * ld + k0 + 8 * q);
    }
    // the sum runs down x's columns: x[k0 ..][c0 + lane % 16], read transposed
    static __device__ __forceinline__ F down(const E *x, int ld, int k0, int c0, int n, int q) {
        const E *p = x + (k0 + 8 * q + n / 4) * ld + c0 + 4 * (n % 4);
        const o_s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
        const o_s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 4 * ld));
        return __builtin_bit_cast(F, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // x[row][k0 ..] in the order in which the accumulators of a state hold those rows
    static __device__ __forceinline__ F along_state(const E *x, int ld, int row, int k0, int q) {
        const o_bf16x4 a = *(const o_bf16x4 *)(x + row * ld + k0 + 4 * q);
        const o_bf16x4 b = *(const o_bf16x4 *)(x + row * ld + k0 + 16 + 4 * q);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static constexpr int TILES = 2;  // state tiles of 16 rows in a fragment
    // fp32 values as N bf16 parts, each the rest rounded: three hold all 24 bits, two 16 (and sign).  WILD: values may be infinite,
    // which have no rest
    template <int N, bool WILD> static __device__ __forceinline__ void split(const float *x, F (&p)[N]) {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        o_u32x4 w[N];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f2 r = {x[2 * i], x[2 * i + 1]};
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const unsigned u = __builtin_bit_cast(unsigned, __builtin_convertvector(r, b2));
                w[j][i] = u;
                if (j + 1 < N) r = f2{r[0] - __uint_as_float(u << 16), r[1] - __uint_as_float(u & 0xffff0000u)};
                if (WILD && j == 0)
#pragma unroll
                    for (int h = 0; h < 2; ++h) r[h] = __builtin_amdgcn_fmed3f(r[h], 0.0f, r[h]);  // NaN: the other operand
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) p[j] = __builtin_bit_cast(F, w[j]);
    }
};
struct MatF32 {
    typedef float E;
    typedef o_f32x4 F;
    static constexpr int KM = 16, PAD = 4;
    static __device__ __forceinline__ o_f32x4 mma(F a, F b, o_f32x4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ F along(const E *x, int ld, int row, int k0, int q) {
        return *(const F *)(x + row * ld + k0 + 4 * q);
    }
    static __device__ __forceinline__ F down(const E *x, int ld, int k0, int c0, int n, int q) {
        F f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = x[(k0 + 4 * q + i) * ld + c0 + n];
        return f;
    }
    static __device__ __forceinline__ F along_state(const E *x, int ld, int row, int k0, int q) {
        return along(x, ld, row, k0, q);
    }
    static constexpr int TILES = 1;
    template <int N, bool WILD> static __device__ __forceinline__ void split(const float *x, F (&p)[N]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[0][i] = x[i];
    }
};
// How many parts an fp32 operand needs for `n` bf16 parts' worth of digits.
template <class M> constexpr int parts_of(int n) { return M::KM == 32 ? n : 1; }
template <class T> struct MatOf { typedef MatF32 M; };
template <> struct MatOf<ElemBF16> { typedef MatBF16 M; };

// Rows of a workgroup of the index; workgroups that check the offsets, each with a word of its own for what it finds.
constexpr int kIndexRows = 1024, kCheckers = 16;
__device__ __forceinline__ bool any_bad(const int *__restrict__ bad) {
    int b = 0;
#pragma unroll
    for (int i = 0; i < kCheckers; ++i) b |= bad[i];
    return b;
}

// Where the spans' borders are.
struct Spans {
    const int2 *info;  // first and past-the-last row of each row's sequence, (-1, -1) outside of all
    int n_rows, span, n;
    struct Border {
        int row;
        bool cuts;  // rows row - 1 and row are of one sequence
    };
    __device__ __forceinline__ Border border(int p) const {
        if (p <= 0) return {0, false};
        const long long b = (long long)p * span;
        if (p >= n || b >= n_rows) return {n_rows, false};
        const int r = (int)b;
        const int2 s = info[r];
        if (s.x < 0 || s.x == r) return {r, false};
        if (r - s.x < kChunk) return {s.x, false};
        if (s.y - r < kChunk) return {s.y, false};
        return {r, true};
    }
};

struct DecayRun {
    const void *q, *k, *v, *x;           // x: what the part from the state is multiplied with for db
    long long qs, ks, vs, xs;            // row strides, elements
    int group, qg, kg, vg, xg;           // heads that share a query's and key's; whether q, k, v, x are one
    void *out;
    long long os;
    int out_f32;                         // out holds fp32 rows of all heads (summed over sharing heads later)
    const float *g;
    long long gs;                        // 0: one decay a head
    int shift;
    const float *s0;                     // [n_seqs][heads][state], or null
    float *sf;
    int turned;                          // states in memory are the transposed of this run's
    int sf_decay;                        // the last state is multiplied by the last row's own decay
    int sf_before;                       // the state kept is that from before the last chunk, decayed to the last row
    float *local;                        // [spans][heads][state]: the state at the spans' ends
    float *mult;                         // [spans][heads]: decay over a span that is all one sequence's
    int *kind;                           // [spans]: 0 its end cuts no sequence, 1 it does, 2 and its start cuts the same
    double *db;                          // [n_rows][heads]
    int pairs;                           // db has the chunks' pairs of rows too
    float out_scale, kv_scale;
    const int32_t *offsets;
    int n_seqs, heads, dir;
    const int *bad;
    Spans spans;
};

// A launch's runs: one, or up to three of the same shapes side by side (blockIdx.y).
struct DecayRuns {
    DecayRun run[3];
};

enum { DECAY_STATE = 0, DECAY_OUT = 1, DECAY_DOT = 2 };

__device__ __forceinline__ float log_decay_of(const DecayRun &A, int r, int h) {
    const float g = A.gs ? A.g[(long long)r * A.gs + h] : A.g[h];
    return g < kForget ? kForget : g;  // (NaN stays)
}

// The 16-byte pieces of a [64][D] tile that a thread brings from memory to LDS.  Rows are counted from the chunk's
// first in memory: a thread's are p, p + NT / PIECES, ...; in LDS they lie in the recurrence's order.
template <class T, class M, int D, int NT> struct Tile {
    typedef typename T::E E;
    typedef typename M::E ME;
    static constexpr int VEC = 16 / sizeof(E), PIECES = D / VEC, STEP = NT / PIECES, N = (kChunk + STEP - 1) / STEP;
    o_u32x4 raw[N];
    // (through a descriptor that ends behind the chunk's last row, so that rows past it come as zeros: a load under a condition
    // is waited for where its register meets the other value, four memory latencies a chunk)
    __device__ __forceinline__ void load(const void *base, long long stride, int rows, int tid) {
        const unsigned row = (unsigned)stride * (unsigned)sizeof(E);
        const auto all = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)((rows - 1) * row + D * (unsigned)sizeof(E)), 0x00020000);
        const unsigned at = tid / PIECES * row + tid % PIECES * 16u;
#pragma unroll
        for (int j = 0; j < N; ++j) raw[j] = __builtin_amdgcn_raw_buffer_load_b128(all, (int)(at + j * STEP * row), 0, 0);
    }
    __device__ __forceinline__ void store(ME *lds, int rows, int dir, int tid) const {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int p = tid / PIECES + j * STEP;
            if (N * STEP > kChunk && p >= kChunk) break;
            const int i = dir < 0 && p < rows ? rows - 1 - p : p;
            ME *q = lds + i * (D + M::PAD) + tid % PIECES * VEC;
            if constexpr (sizeof(ME) == sizeof(E)) {
                *(o_u32x4 *)q = raw[j];
            } else {  // fp16 to fp32
                typedef __attribute__((ext_vector_type(8))) _Float16 H8;
                *(o_f32x8 *)q = __builtin_convertvector(__builtin_bit_cast(H8, raw[j]), o_f32x8);
            }
        }
    }
    __device__ __forceinline__ bool infinite() const {  // or NaN: the largest exponent there is
        if constexpr (sizeof(E) == 4) {
            unsigned most = 0;
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const unsigned u = raw[j][w] & 0x7fffffffu;
                    most = most > u ? most : u;
                }
            return most >= 0x7f800000u;
        } else {
            typedef __attribute__((ext_vector_type(2))) unsigned short H2;
            H2 most = {0, 0};
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    most = __builtin_elementwise_max(most, __builtin_bit_cast(H2, raw[j][w] & 0x7fff7fffu));
            constexpr unsigned short top = sizeof(ME) == 2 ? 0x7f80 : 0x7c00;
            return most[0] >= top || most[1] >= top;
        }
    }
};

template <class T> __device__ __forceinline__ void store4(typename T::E *p, o_f32x4 v) {
    typedef __attribute__((ext_vector_type(4))) typename T::E V;
    *(V *)p = __builtin_convertvector(v, V);
}

// v of another lane of the same 16 (DPP; 0 where there is none).
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
template <int CTRL> __device__ __forceinline__ double dpp(double v) {
    const long long b = __builtin_bit_cast(long long, v);
    const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xf, 0xf, false);
    const unsigned hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xf, 0xf, false);
    return __builtin_bit_cast(double, (long long)((unsigned long long)hi << 32 | lo));
}
__device__ __forceinline__ double lane_of(double v, int lane) {
    const long long b = __builtin_bit_cast(long long, v);
    const unsigned lo = __builtin_amdgcn_readlane((int)b, lane), hi = __builtin_amdgcn_readlane((int)(b >> 32), lane);
    return __builtin_bit_cast(double, (long long)((unsigned long long)hi << 32 | lo));
}
// The sum over the four lanes n, n + 16, n + 32, n + 48, in all of them: halves, then rows of 16, swapped.
__device__ __forceinline__ float sum_rows(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// Four fp64 values summed over the 16 lanes of a row: lane n has the sum of value 2 (n & 1) + (n >> 1 & 1).  Neighbours, then
// pairs, each keep one half of the values that they add; quads and halves, rotated, are added whole.
__device__ __forceinline__ double sum16_of_4(const double (&v)[4], int n) {
    const bool odd = n & 1, high = n & 2;
    const double a = (odd ? v[2] : v[0]) + dpp<0xb1>(odd ? v[0] : v[2]);  // quad_perm 1 0 3 2
    const double b = (odd ? v[3] : v[1]) + dpp<0xb1>(odd ? v[1] : v[3]);
    double s = (high ? b : a) + dpp<0x4e>(high ? a : b);  // quad_perm 2 3 0 1
    s += dpp<0x128>(s);  // row_ror 8
    return s + dpp<0x124>(s);
}
// The sum over the four lanes n, n + 16, n + 32, n + 48 of an fp64 value.
__device__ __forceinline__ double sum_rows(double v) {
    auto pair = [](unsigned lo, unsigned hi) { return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo); };
    auto words = [&] { return __builtin_bit_cast(unsigned long long, v); };
    const auto al = __builtin_amdgcn_permlane32_swap((unsigned)words(), (unsigned)words(), false, false);
    const auto ah = __builtin_amdgcn_permlane32_swap((unsigned)(words() >> 32), (unsigned)(words() >> 32), false, false);
    v = pair(al[0], ah[0]) + pair(al[1], ah[1]);
    const auto bl = __builtin_amdgcn_permlane16_swap((unsigned)words(), (unsigned)words(), false, false);
    const auto bh = __builtin_amdgcn_permlane16_swap((unsigned)(words() >> 32), (unsigned)(words() >> 32), false, false);
    return pair(bl[0], bh[0]) + pair(bl[1], bh[1]);
}
// v summed over the lanes from `from` (this lane's own, at most this lane) to this one.
__device__ __forceinline__ double sum_from(double v, int from, int lane) {
    const int in = lane & 15;
    auto step = [&](double o, int d) {
        if (in >= d && lane - d >= from) v += o;
    };
    step(dpp<0x111>(v), 1);  // row_shr
    step(dpp<0x112>(v), 2);
    step(dpp<0x114>(v), 4);
    step(dpp<0x118>(v), 8);
#pragma unroll
    for (int r = 16; r < 64; r += 16) {  // the rows of 16 before: their last lane's sum is of the same run
        const double o = lane_of(v, r - 1);
        if (lane >= r && lane < r + 16 && from < r) v += o;
    }
    return v;
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
// 2^x of an fp64 x, to fp32's precision
__device__ __forceinline__ float exp2_of(double x) {
    const float h = (float)x;
    const float e = exp2_hw(h), l = (float)(x - (double)h);
    return l == l ? fmaf(e, l * 0.693147180559945f, e) : e;  // (h infinite: no rest)
}

// What the products need to know of a chunk's rows, in the recurrence's order.
struct ChunkRows {
    float bh[kChunk], bl[kChunk];  // sum of the log2 decays from the chunk's first row, or the sequence's, to the row: high and low part
    float to[kChunk];              // 2^(b_end - b) times kv_scale: what the row brings to the state after
    float decay[kChunk];           // 2^b (times out_scale: what the state before brings to the row)
    int seg[kChunk];               // the sequence: its first row in the chunk + 1 (0: before the chunk), its last + 1 << 8, 1 << 16 if it ends there
};
__device__ __forceinline__ int seg_first(int s) { return (s & 255) - 1; }
__device__ __forceinline__ int seg_past(int s) { return (s >> 8) & 255; }
__device__ __forceinline__ bool seg_ends(int s) { return s >> 16; }

// The tiles of a chunk's weights on or below the diagonal, two bits each, in the order in which they are dealt to four
// waves: the last wave, which has the next chunk's rows to prepare, gets two of the far ones, which short sequences skip.
constexpr int tile_list(int a, int b, int c, int d, int e, int f, int g, int h, int i, int j) {
    return a | b << 2 | c << 4 | d << 6 | e << 8 | f << 10 | g << 12 | h << 14 | i << 16 | j << 18;
}
constexpr int kTileT = tile_list(3, 2, 1, 3, 0, 3, 2, 2, 1, 3), kTileS = tile_list(3, 2, 1, 0, 0, 2, 1, 0, 0, 1);
__device__ __forceinline__ int tile_of(int list, int w) { return list >> (2 * w) & 3; }
__device__ __forceinline__ int tile_at(int mt, int ms) { return mt * (mt + 1) / 2 + ms; }  // row by row
// Values of a chunk's weights in LDS: a row tile has columns up to its diagonal, in whole fragments, padded.
template <class M> constexpr int weights_size() { return 16 * (4 * M::PAD + (M::KM == 32 ? 192 : 160)); }

// Waves a SIMD that the registers are to allow.  Not more than workgroups fit in a compute unit's LDS: asked for those, the
// compiler gives the limit up and goes past 256 registers, which leaves one workgroup (fp32 64 x 64, 16 384 tracks of 4 heads:
// 402 us, 272 with two; bf16 128 x 32 300 and 188).  fp32 states of d_k 128 take more registers than three or four waves leave
// (128 x 128, one sequence of 16 384 rows: spilled 141 us, in two waves 135).  Others spill a little and are faster all the
// same: 28 bytes or less in the 16-bit types' states of 128 x 128 (120 us, without 125), 24 in the fp32 products' outputs of 32 x 64
// (195 us, without 208), 8 in bf16's outputs of 64 x 64.
template <class T, int DK, int DV, int MODE> constexpr int span_waves() {
    typedef typename MatOf<T>::M M;
    constexpr int per = span_threads(DV) / 256, es = sizeof(typename M::E), lk = DK + M::PAD, lv = DV + M::PAD;
    constexpr int tiles = MODE == DECAY_STATE ? lk + lv : MODE == DECAY_OUT ? 2 * lk + lv : 2 * (lk + lv);
    constexpr int weights = MODE == DECAY_STATE ? 0 : weights_size<M>() * parts_of<M>(2);
    constexpr int sums = MODE == DECAY_DOT ? 2 * 10 * 16 * 8 + kChunk * 4 * (DV == 32 ? 2 : DV / 16) : 0;
    constexpr int fit = 160 * 1024 / ((kChunk * tiles + weights) * es + 2 * (int)sizeof(ChunkRows) + sums + 128) * per;
    constexpr int want = MODE == DECAY_STATE ? (sizeof(typename T::E) == 4 && DK == 128 ? 2 : DK <= DV ? 4 : 3)
                                             : DK * DV <= 32 * 32 || (MODE == DECAY_OUT && DK * DV <= 64 * 64) ? 3 : 2;
    return want < fit ? want : fit;
}

// One span of one head.  A wave (four of them, eight for d_v 128) owns 16 of the state's and the output's columns (d_v 32: 16
// of them too, and of the outputs every second row tile; its pair holds the same state); the state stays in its accumulators
// over the span.  The 64 x 64 weights of a chunk are computed once, 16 x 16 tiles on or below the diagonal dealt out to the
// waves, and pass through LDS; the last wave prepares the next chunk's row sums meanwhile.  The next chunk's rows of the
// tensors are on their way to registers.
//
// Chunks of 64 rows: a chunk's weights cost 64 (d_k + d_v) products a row and its state 2 d_k d_v, equal at 64 columns, and
// tracks of up to 20 hits are whole within one or two.  What bounds it: with many spans, memory.  918 161 rows of 65 536 tracks,
// 3 heads of 64 x 64, bf16: 1.42 GB in 357 us, 4.0 TB/s of the 5.1 that a copy reaches, the vector units half busy.  With few,
// the latency of a chunk's phases, each behind a barrier: one sequence of 32 768 rows, 8 heads of 128 x 128, 512 workgroups of
// eight chunks, 161 us.  The states, two workgroups a compute unit, take 47 us, 6 a chunk; the outputs, whose registers leave one
// workgroup a compute unit and so two rounds, 109 us, 7 a chunk; the matrix units a fifth and the vector units two fifths busy.
// fp32: the fp32 instruction (16 times slower than bf16's) and LDS: gradients of 115 thousand rows, 4 heads of 32 x 32, 280 us.
template <class T, int DK, int DV, int MODE>
__global__ __launch_bounds__(span_threads(DV), (span_waves<T, DK, DV, MODE>())) void tf_decay_span_kernel(DecayRuns R) {
    typedef typename MatOf<T>::M M;
    typedef typename M::E ME;
    typedef typename M::F F;
    constexpr bool OUT = MODE >= DECAY_OUT, DOT = MODE >= DECAY_DOT;
    constexpr int NT = span_threads(DV), NW = NT / 64, KM = M::KM, ES = sizeof(typename T::E);
    constexpr int LK = DK + M::PAD, LV = DV + M::PAD;
    // a row tile of the weights has columns up to its diagonal, in whole fragments
    auto p_ld = [](int mt) { return (16 * mt + 16 + KM - 1) / KM * KM + M::PAD; };
    auto p_at = [&](int mt) { return 16 * ((mt > 0 ? p_ld(0) : 0) + (mt > 1 ? p_ld(1) : 0) + (mt > 2 ? p_ld(2) : 0)); };
    constexpr int PSIZE = weights_size<M>();
    constexpr int RG = DV == 32 ? 2 : 1, TM = 4 / RG;  // waves that share a column tile, and their row tiles
    constexpr int ST = DK / 16;                    // state tiles of a wave's column tile
    constexpr int NB = kChunk / KM;                // fragments along a chunk's rows
    constexpr int NS = parts_of<M>(DOT ? 3 : 2);   // parts of the state in its product with q
    constexpr int NU = parts_of<M>(3);             // parts of the weighted v in the state's update
    constexpr int NP = parts_of<M>(2);             // parts of the weights
    __shared__ __attribute__((aligned(16))) ME Qs[OUT ? kChunk * LK : 8], Ks[kChunk * LK], Vs[kChunk * LV],
        Xs[DOT ? kChunk * LV : 8], Ps[OUT ? NP * PSIZE : 8];
    __shared__ ChunkRows rows_of[2];
    __shared__ int wild[2];
    __shared__ double rowp[DOT ? 10 : 1][16], colp[DOT ? 10 : 1][16];  // of the weights' tiles, by tile_at
    __shared__ float dots[DOT ? NW / RG : 1][kChunk];

    const DecayRun &A = R.run[blockIdx.y];
    const bool dot = DOT && A.x, pairs = DOT && A.pairs;
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int n = lane % 16, q = lane / 16, group = wave / RG, rg = wave % RG, c0 = 16 * group;
    auto row_tile = [&](int m) { return RG == 1 ? m : rg ? 1 + m : 3 * m; };  // (pairs of tiles with equally long sums)
    const int p = blockIdx.x / A.heads, h = blockIdx.x % A.heads, dir = A.dir;
    const int bad = any_bad(A.bad), olo = A.offsets[0], ohi = A.offsets[A.n_seqs];
    const Spans::Border b0 = A.spans.border(p), b1 = A.spans.border(p + 1);
    if (bad) {
        if (OUT) {  // offsets that make no sequences: every row of the array is NaN
            const long long lo = (long long)p * A.spans.span;
            const long long hi = lo + A.spans.span < A.spans.n_rows ? lo + A.spans.span : A.spans.n_rows;
            const float nan = __builtin_nanf("");
            for (long long r = lo; r < hi; ++r)
                for (int i = tid; i < DV; i += NT) {
                    if (A.out_f32) ((float *)A.out)[r * A.os + h * DV + i] = nan;
                    else ((typename T::E *)A.out)[r * A.os + h * DV + i] = (typename T::E)nan;
                }
            if (A.sf)
                for (long long s = p; s < A.n_seqs; s += A.spans.n)
                    for (int i = tid; i < DK * DV; i += NT) A.sf[(s * A.heads + h) * (DK * DV) + i] = nan;
        }
        return;
    }
    int lo = b0.row, hi = b1.row;
    const bool cut_in = dir > 0 ? b0.cuts : b1.cuts, cut_out = dir > 0 ? b1.cuts : b0.cuts;
    bool whole = false;
    if (!OUT) {
        // only the sequence that the span's end cuts has a state there
        int kind = 0;
        if (cut_out) {
            const int2 s = A.spans.info[dir > 0 ? hi - 1 : lo];
            whole = cut_in && (dir > 0 ? s.x < lo : s.y > hi);
            kind = whole ? 2 : 1;
            if (dir > 0) lo = s.x > lo ? s.x : lo;
            else hi = s.y < hi ? s.y : hi;
        }
        if (h == 0 && tid == 0) A.kind[p] = kind;
        if (!cut_out) return;
    } else {
        // rows outside of all sequences are before the first and behind the last
        lo = lo > olo ? lo : olo;
        hi = hi < ohi ? hi : ohi;
    }
    if (hi <= lo) return;
    // Chunks are counted from the span's first row in memory whichever way they are run through, so that the runs of
    // both directions have the same ones (db's two halves are split by chunks).
    const int chunks = (hi - lo + kChunk - 1) / kChunk;

    o_f32x4 S[ST];
    auto clear_state = [&] {
#pragma unroll
        for (int m = 0; m < ST; ++m) S[m] = o_f32x4{0.f, 0.f, 0.f, 0.f};
    };
    clear_state();
    bool have = false;  // the state is that of the sequence that goes on
    auto load_state = [&](const float *s) {
        const int step = A.turned ? 1 : DV;
        const float *e = s + (A.turned ? (c0 + n) * DK + 4 * q : 4 * q * DV + c0 + n);
#pragma unroll
        for (int m = 0; m < ST; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) S[m][i] = e[(16 * m + i) * step];
    };
    auto save_state = [&](float *s, bool turned, float d) {
        const int step = turned ? 1 : DV;
        float *e = s + (turned ? (c0 + n) * DK + 4 * q : 4 * q * DV + c0 + n);
        if (rg == 0) {
#pragma unroll
            for (int m = 0; m < ST; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) e[(16 * m + i) * step] = S[m][i] * d;
        }
    };
    if (OUT && cut_in) {
        load_state(A.local + ((long long)(p - dir) * A.heads + h) * (DK * DV));
        have = true;
    }

    Tile<T, M, DK, NT> tq, tk;
    Tile<T, M, DV, NT> tv, tx;
    // the head's columns, at the span's first row
    const char *bq = nullptr, *bx = nullptr;
    const int hs = h / A.group;
    if (OUT) bq = (const char *)A.q + ((long long)lo * A.qs + (A.qg ? hs : h) * DK) * ES;
    const char *bk = (const char *)A.k + ((long long)lo * A.ks + (A.kg ? hs : h) * DK) * ES;
    const char *bv = (const char *)A.v + ((long long)lo * A.vs + (A.vg ? hs : h) * DV) * ES;
    if (dot) bx = (const char *)A.x + ((long long)lo * A.xs + (A.xg ? hs : h) * DV) * ES;
    auto chunk_rows = [&](int at) { return hi - lo - at < kChunk ? hi - lo - at : kChunk; };
    auto chunk_at = [&](int c) { return (dir > 0 ? c : chunks - 1 - c) * kChunk; };  // the c-th on the way: its first row in memory, from lo
    auto fetch = [&](int c) {
        const int at = chunk_at(c), rows = chunk_rows(at);
        if (OUT) tq.load(bq + (long long)at * A.qs * ES, A.qs, rows, tid);
        tk.load(bk + (long long)at * A.ks * ES, A.ks, rows, tid);
        tv.load(bv + (long long)at * A.vs * ES, A.vs, rows, tid);
        if (dot) tx.load(bx + (long long)at * A.xs * ES, A.xs, rows, tid);
    };
    // The last wave's: a chunk's sequences and decays, one row a lane.
    int2 next_seq = {0, 0};
    float next_g = 0.0f;
    double total = 0.0;
    auto fetch_rows = [&](int c) {
        const int at = chunk_at(c), rows = chunk_rows(at), i = lane < rows ? lane : 0;
        const int r = lo + at + (dir > 0 ? i : rows - 1 - i);
        next_seq = A.spans.info[r];
        int rg = A.shift ? r - dir : r;  // (where that is another sequence's it is not used)
        rg = rg < olo ? olo : rg >= ohi ? ohi - 1 : rg;
        next_g = A.gs ? A.g[(long long)rg * A.gs + h] : A.g[h];
    };
    auto put_rows = [&](ChunkRows &W, int c) {
        const int at = chunk_at(c), rows = chunk_rows(at), i = lane;
        const int r = lo + at + (dir > 0 ? i : rows - 1 - i);
        int f = dir > 0 ? next_seq.x - (r - i) : (r + i) - (next_seq.y - 1), l = dir > 0 ? next_seq.y - 1 - (r - i) : (r + i) - next_seq.x;
        if (i >= rows) f = l = i;  // behind the last row: on its own
        const float g = next_g < kForget ? kForget : next_g;  // (NaN stays)
        double b = i >= rows || (A.shift && f == i) ? 0.0 : (double)g * 1.4426950408889634;
        b = sum_from(b, f > 0 ? f : 0, i);
        const int e = l < rows - 1 ? l : rows - 1;
        const double be = __shfl(b, e & 63);
        const float bf = (float)b, de = exp2_of(b);
        W.bh[i] = bf, W.bl[i] = (float)(b - (double)bf);
        W.decay[i] = de, W.to[i] = A.kv_scale * exp2_of(be - b);
        W.seg[i] = (f < 0 ? 0 : f + 1) | (i < rows ? e + 1 : i + 1) << 8 | (l <= rows - 1 ? 1 << 16 : 0);
        if (!OUT) total += lane_of(b, rows - 1);
    };
    // What a chunk's loads bring goes to LDS when the chunk before is done with it.  The registers in between are this
    // chunk's own (carried around the loop they would be copied at its end, and waited for there).
    auto put = [&](int c) {
        const int rows = chunk_rows(chunk_at(c));
        if (OUT) tq.store(Qs, rows, dir, tid);
        tk.store(Ks, rows, dir, tid);
        tv.store(Vs, rows, dir, tid);
        if (dot) tx.store(Xs, rows, dir, tid);
        if (tk.infinite() || tv.infinite()) wild[c & 1] = 1;
    };
    fetch(0);
    if (tid < 2) wild[tid] = 0;
    if (wave == NW - 1) {
        fetch_rows(0);
        put_rows(rows_of[0], 0);
        if (chunks > 1) fetch_rows(1);
    }
    if (OUT)  // the weights above the diagonal that share a fragment with some below
        for (int i = tid; i < NP * PSIZE * (int)sizeof(ME) / 4; i += NT) ((unsigned *)Ps)[i] = 0;
    __syncthreads();
    put(0);
    __syncthreads();

    for (int c = 0; c < chunks; ++c) {
        const int at = chunk_at(c), rows = chunk_rows(at);
        const ChunkRows &W = rows_of[c & 1];
        const bool slow = __builtin_amdgcn_readfirstlane(wild[c & 1]);
        // (Behind the last chunk that chunk again: under a branch the loads are waited for where it ends.  One sequence of 32 768
        // rows, 8 heads of 128 x 128: 171 us with a branch, 157 without; 65 536 tracks 360 and 342.)
        fetch(c + 1 < chunks ? c + 1 : c);
        F vf[NB];  // the wave's columns of v, for the state and for the output
        auto read_v = [&](int k) { vf[k] = M::down(Vs, LV, k * KM, c0, n, q); };
        if (OUT) {
#pragma unroll
            for (int k = 0; k < NB; ++k) read_v(k);
        }
        // the last wave prepares the next chunk's rows while the others compute the weights
        if (wave == NW - 1 && c + 1 < chunks) {
            put_rows(rows_of[(c + 1) & 1], c + 1);
            if (c + 2 < chunks) fetch_rows(c + 2);
        }
        if (OUT) {
            // weights: tile (s tile ms, t tile mt), transposed, so that four consecutive s of a row t land in a lane
            const float sc = A.out_scale * A.kv_scale;
#pragma unroll 1
            for (int w = NW == 4 || wave < NW - 1 ? wave : 10; w < 10; w += NW == 4 ? NW : NW - 1) {
                const int mt = tile_of(kTileT, w), ms = tile_of(kTileS, w);
                const int t = 16 * mt + n, s = 16 * ms + 4 * q, f = seg_first(W.seg[t]);
                const bool apart = seg_first(__builtin_amdgcn_readfirstlane(W.seg[16 * mt])) >= 16 * ms + 16;  // all of the tile's rows are of later sequences
                typedef __attribute__((ext_vector_type(4))) ME V4;
                o_f32x4 a = {0.f, 0.f, 0.f, 0.f}, z = {0.f, 0.f, 0.f, 0.f};
                if (!apart) {
                    struct Two { F k, q; };
                    in_turn<DK / KM, (DK / KM < 4 ? DK / KM + 1 : 4)>(
                        [&](int i) { return Two{M::along(Ks, LK, 16 * ms + n, i * KM, q), M::along(Qs, LK, 16 * mt + n, i * KM, q)}; },
                        [&](int, Two f) { a = M::mma(f.k, f.q, a); });
                    if (pairs) {
#pragma unroll
                        for (int k0 = 0; k0 < DV; k0 += KM)
                            z = M::mma(M::along(Vs, LV, 16 * ms + n, k0, q), M::along(Xs, LV, 16 * mt + n, k0, q), z);
                    }
                    const float th = W.bh[t], tl = W.bl[t];
                    const o_f32x4 sh = *(const o_f32x4 *)&W.bh[s], sl = *(const o_f32x4 *)&W.bl[s];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float e = exp2_hw((th - sh[i]) + (tl - sl[i]));
                        a[i] = s + i <= t && s + i >= f ? a[i] * (e * sc) : 0.0f;
                    }
                }
                const V4 high = __builtin_convertvector(a, V4);
                *(V4 *)(Ps + p_at(mt) + n * p_ld(mt) + s) = high;
                if constexpr (NP == 2) {
                    o_f32x4 low = a - __builtin_convertvector(high, o_f32x4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) low[i] = __builtin_amdgcn_fmed3f(low[i], 0.0f, low[i]);
                    *(V4 *)(Ps + PSIZE + p_at(mt) + n * p_ld(mt) + s) = __builtin_convertvector(low, V4);
                }
                if (pairs) {
                    // products of dq's weights with q k: their sums by t and by s are what q dq and k dk have of them.  In fp64: the
                    // decays' gradient is a sum of these over a span, in which all pairs but the few around a row cancel
                    double row = 0.0, four = 0.0;
                    if (!apart) {
                        double col[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            col[i] = s + i <= t && s + i >= f ? (double)(a[i] * z[i]) : 0.0;
                            row += col[i];
                        }
                        row = sum_rows(row);
                        four = sum16_of_4(col, n);
                    }
                    if (q == 0) rowp[tile_at(mt, ms)][n] = row;
                    if (n < 4) colp[tile_at(mt, ms)][4 * q + 2 * (n & 1) + (n >> 1)] = four;
                }
            }
            __syncthreads();
        }

        o_f32x4 o[TM];
#pragma unroll
        for (int m = 0; m < TM; ++m) o[m] = o_f32x4{0.f, 0.f, 0.f, 0.f};
        // The chunk's sequences, one after the other: what their state adds to their rows, and the state after them.  Those
        // that are whole in the chunk have none, unless states come in or go out.
#pragma unroll 1
        for (int a = 0; a < rows;) {
            const int seg = __builtin_amdgcn_readfirstlane(W.seg[a]), b = seg_past(seg);
            const bool starts = seg_first(seg) >= 0, ends = seg_ends(seg);
            int seq = -1;
            if ((starts && A.s0) || (ends && A.sf))
                seq = seq_of_row(A.offsets, A.n_seqs, lo + at + (dir > 0 ? a : rows - 1 - a));
            if (starts) {
                have = A.s0 != nullptr;
                if (have) load_state(A.s0 + ((long long)seq * A.heads + h) * (DK * DV));
            }
            if (OUT && have) {
                o_f32x4 z[TM];
#pragma unroll
                for (int m = 0; m < TM; ++m) z[m] = o_f32x4{0.f, 0.f, 0.f, 0.f};
                F sp[NS];
                in_turn<DK / KM * TM, 4>([&](int i) { return M::along_state(Qs, LK, 16 * row_tile(i % TM) + n, i / TM * KM, q); },
                                         [&](int i, F f) {
                                             const int k = i / TM, m = i % TM;
                                             if (m == 0) {
                                                 float x[4 * M::TILES];
#pragma unroll
                                                 for (int e = 0; e < 4 * M::TILES; ++e) x[e] = S[k * M::TILES + e / 4][e % 4];
                                                 M::template split<NS, true>(x, sp);
                                             }
                                             // (a branch costs more than the bf16 products of rows that are not the sequence's)
                                             const int t = 16 * row_tile(m);
                                             if (KM == 16 && (t + 16 <= a || t >= b)) return;
#pragma unroll
                                             for (int e = NS - 1; e >= 0; --e) z[m] = M::mma(sp[e], f, z[m]);
                                         });
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    const int t = 16 * row_tile(m) + n;
                    const float f = A.out_scale * W.decay[t];
                    const bool on = t >= a && t < b;
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[m][i] = on ? z[m][i] * f : o[m][i];
                }
            }
            if (!ends || A.sf) {
                if (have) {
                    const float d = W.decay[b - 1];
#pragma unroll
                    for (int m = 0; m < ST; ++m) S[m] *= d;
                } else {
                    clear_state();
                }
                if (ends && A.sf_before) {  // (the sequence needs no state any more)
                } else if (!slow) {
#pragma unroll
                    for (int k = 0; k < NB; ++k) {
                        if (k * KM + KM <= a || k * KM >= b) continue;
                        if (!OUT) read_v(k);
                        F vp[NU];
                        float w[KM / 4];
#pragma unroll
                        for (int i = 0; i < KM / 4; i += 4) *(o_f32x4 *)&w[i] = *(const o_f32x4 *)&W.to[k * KM + KM / 4 * q + i];
                        float x[KM / 4];
#pragma unroll
                        for (int i = 0; i < KM / 4; ++i) {
                            const int s = k * KM + KM / 4 * q + i;
                            x[i] = s >= a && s < b ? (float)vf[k][i] * w[i] : 0.0f;
                        }
                        M::template split<NU, false>(x, vp);
                        in_turn<ST, 3>([&](int m) { return M::down(Ks, LK, k * KM, 16 * m, n, q); },
                                       [&](int m, F kf) {
#pragma unroll
                                           for (int i = NU - 1; i >= 0; --i) S[m] = M::mma(kf, vp[i], S[m]);
                                       });
                    }
                } else {
#pragma unroll 1
                    for (int s = a; s < b; ++s) {
                        const float v = (float)Vs[s * LV + c0 + n] * W.to[s];
#pragma unroll
                        for (int m = 0; m < ST; ++m)
#pragma unroll
                            for (int i = 0; i < 4; ++i) S[m][i] += (float)Ks[s * LK + 16 * m + 4 * q + i] * v;
                    }
                }
                have = true;
                if (ends && A.sf) {
                    float d = 1.0f;
                    if (A.sf_decay) d = expf(log_decay_of(A, lo + at + (dir > 0 ? b - 1 : rows - b), h));
                    save_state(A.sf + ((long long)seq * A.heads + h) * (DK * DV), A.turned, d);
                }
            }
            a = b;
            if (!A.s0 && !A.sf && b < rows) {  // on to the last one
                const int f = seg_first(__builtin_amdgcn_readfirstlane(W.seg[rows - 1]));
                if (f > b) a = f;
            }
        }
        if (OUT) {
            if (dot) {
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    float z = 0.0f;
                    typedef __attribute__((ext_vector_type(4))) ME V4;
                    const o_f32x4 x = __builtin_convertvector(*(const V4 *)(Xs + (16 * row_tile(m) + n) * LV + c0 + 4 * q), o_f32x4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) z += o[m][i] * x[i];
                    z = sum_rows(z);
                    if (q == 0) dots[group][16 * row_tile(m) + n] = z;
                }
            }
            if (!slow) {
                int from[TM];  // the first row that a row tile has weights of
#pragma unroll
                for (int m = 0; m < TM; ++m)
                    from[m] = KM == 16 ? seg_first(__builtin_amdgcn_readfirstlane(W.seg[16 * row_tile(m)])) : 0;
                in_turn<NB * TM * NP, 4>(
                    [&](int i) {
                        F f = {};
                        const int mt = row_tile(i / NP % TM), k = i / NP / TM, part = NP - 1 - i % NP;
                        if (k * KM <= 16 * mt) f = M::along(Ps + part * PSIZE + p_at(mt), p_ld(mt), n, k * KM, q);
                        return f;
                    },
                    [&](int i, F f) {
                        const int k = i / NP / TM, m = i / NP % TM;
                        if (k * KM <= 16 * row_tile(m) && (KM == 32 || k * KM + KM > from[m])) o[m] = M::mma(vf[k], f, o[m]);
                    });
            } else {
                // an infinite or NaN k or v: only the products that the definition has
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    const int t = 16 * row_tile(m) + n, f = seg_first(W.seg[t]);
                    for (int s = f > 0 ? f : 0; s <= t; ++s) {
                        const ME *w = Ps + p_at(row_tile(m)) + n * p_ld(row_tile(m)) + s;
                        float p = (float)w[0];
                        if constexpr (NP == 2) p += (float)w[PSIZE];
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[m][i] += p * (float)Vs[s * LV + c0 + 4 * q + i];
                    }
                }
            }
            // (the chunk's first row is a scalar; 64 rows of a stride fit in 32 bits)
            const int es = A.out_f32 ? 4 : ES;
            char *ob = (char *)A.out + ((long long)(lo + at) * A.os + h * DV + c0) * es;
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                const int t = 16 * row_tile(m) + n;
                if (t < rows) {
                    char *to = ob + (unsigned)((dir > 0 ? t : rows - 1 - t) * (int)A.os + 4 * q) * (unsigned)es;
                    if (A.out_f32) *(o_f32x4 *)to = o[m];
                    else store4<T>((typename T::E *)to, o[m]);
                }
            }
        }
        __syncthreads();
        if (tid == 0) wild[c & 1] = 0;
        if (c + 1 < chunks) put(c + 1);
        if (dot && wave == 0) {
            const int t = lane;
            if (t < rows) {
                double z = 0.0;
                for (int w = 0; w < NW / RG; ++w) z += (double)dots[w][t];
                if (pairs)
                    for (int m = 0; m < 4; ++m) {
                        if (m <= t / 16) z += rowp[tile_at(t / 16, m)][t % 16];
                        if (m >= t / 16) z -= colp[tile_at(m, t / 16)][t % 16];
                    }
                A.db[(long long)(lo + at + (dir > 0 ? t : rows - 1 - t)) * A.heads + h] = z;
            }
        }
        __syncthreads();
    }
    if (!OUT) {
        save_state(A.local + ((long long)p * A.heads + h) * (DK * DV), false, 1.0f);
        if (wave == NW - 1 && lane == 0) A.mult[(long long)p * A.heads + h] = whole ? exp2_of(total) : 0.0f;
    }
}

// Outputs whose rows outside of all sequences become zeros: p null where they are left as they are.
struct DecayClear {
    char *p[4];
    long long stride[4];  // bytes
    int words[4];         // of a row, 4 bytes each
    void add(int i, void *x, int64_t row_stride, int64_t width, size_t size) {
        p[i] = (char *)x, stride[i] = row_stride * (int64_t)size, words[i] = (int)(width * (int64_t)size / 4);
    }
};

// First and past-the-last row of every row's sequence; whether the offsets are in order and inside the array.  A workgroup
// has 1024 rows: it finds the sequence of the first by 256 probes at a time, puts the starts of the sequences that follow
// where they are, and a running maximum tells every row its sequence (a thread a row and a binary search each took 92 us
// for 918 161 rows of 65 536 sequences).  The workgroups behind those pass the states of sequences without rows through,
// `per` sequences each (a launch of their own took 4 us).
__global__ __launch_bounds__(256) void tf_decay_index_kernel(const int32_t *__restrict__ offsets, int n_seqs, int n_rows,
                                                             int2 *__restrict__ info, int *__restrict__ bad,
                                                             int32_t *__restrict__ flags, long long size, int per,
                                                             const float *__restrict__ s0, float *__restrict__ sf, DecayClear C) {
    __shared__ int mark[kIndexRows], top[4];
    const int tid = threadIdx.x;
    if (blockIdx.x < kCheckers) {
        int wrong = 0;
#pragma unroll 8
        for (int i = blockIdx.x * 256 + tid; i <= n_seqs; i += 256 * kCheckers) {
            const int o = offsets[i], e = offsets[i < n_seqs ? i + 1 : i];
            wrong |= o < 0 || o > n_rows || e < o;
        }
        wrong = __syncthreads_or(wrong);
        if (tid == 0) {
            bad[blockIdx.x] = wrong;
            if (wrong && flags) atomicOr(flags, TF_SEQ_BAD_OFFSETS);
        }
        return;
    }
    const int tile = (int)blockIdx.x - kCheckers, tiles = (n_rows + kIndexRows - 1) / kIndexRows;
    if (tile >= tiles) {
        const long long first = (long long)(tile - tiles) * per, end = first + per < n_seqs ? first + per : n_seqs;
        for (long long s = first; s < end; s += 64) {
            const long long mine = s + tid % 64;  // (every wave looks at all of them)
            unsigned long long empty = __ballot(mine < end && offsets[mine < end ? mine : s] == offsets[mine < end ? mine + 1 : s]);
            for (; empty; empty &= empty - 1) {
                const long long i = s + __builtin_ctzll(empty);
                for (long long e = 4 * tid; e < size; e += 1024)
                    *(o_f32x4 *)(sf + i * size + e) = s0 ? *(const o_f32x4 *)(s0 + i * size + e) : o_f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
        return;
    }
    const int r0 = tile * kIndexRows, r1 = n_rows - r0 < kIndexRows ? n_rows : r0 + kIndexRows;
    const int first = offsets[0], last = offsets[n_seqs];
    // how many of the n_seqs + 1 offsets are at most r0
    int lo = 0, hi = n_seqs + 1;
    while (lo < hi) {
        const int step = (hi - lo + 255) / 256, i = lo + tid * step;
        const int below = __syncthreads_count(i < hi && offsets[i] <= r0);  // these are the first ones
        if (below == 0) break;
        const int end = lo + below * step;
        lo = lo + (below - 1) * step + 1;
        hi = end < hi ? end : hi;
    }
#pragma unroll
    for (int j = 0; j < kIndexRows / 256; ++j) mark[tid + 256 * j] = 0;
    __syncthreads();
    for (int i = lo;; i += 256) {  // the offsets behind r0, to the tile's end
        const int o = i + tid <= n_seqs ? offsets[i + tid] : n_rows;
        if (o > r0 && o < r1) atomicMax(&mark[o - r0], i + tid + 1);  // offsets at most this row's
        if (__syncthreads_count(i + tid <= n_seqs && o < r1) < 256) break;
    }
    int m[4], best = tid == 0 ? lo : 0;
    const int4 four = *(const int4 *)&mark[4 * tid];
    m[0] = four.x, m[1] = four.y, m[2] = four.z, m[3] = four.w;
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = best = best > m[j] ? best : m[j];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(best, d);
        if (tid % 64 >= d && o > best) best = o;
    }
    if (tid % 64 == 63) top[tid / 64] = best;
    __syncthreads();
    int before = __shfl_up(best, 1);
    if (tid % 64 == 0) before = 0;
    for (int w = 0; w < tid / 64; ++w) before = before > top[w] ? before : top[w];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r = r0 + 4 * tid + j, k = m[j] > before ? m[j] : before;
        if (r < n_rows) info[r] = k == 0 || k > n_seqs ? int2{-1, -1} : int2{offsets[k - 1], offsets[k]};
    }
    // The tile's rows before the first sequence and behind the last.
    if (first <= r0 && last >= r1) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (C.p[i])
            for (int r = r0 + tid / 64; r < r1; r += 4)
                if (r < first || r >= last)
                    for (int w = tid % 64; w < C.words[i]; w += 64) *(unsigned *)(C.p[i] + r * C.stride[i] + 4 * w) = 0;
}

// The states at the spans' ends from the spans' own contributions, in order along each cut sequence.  A wave has 128
// values of one head's states and every `chains`-th span; where that is a sequence's first cut it follows the sequence, the
// next spans' contributions on their way while it adds (each sum stays for the span that follows).  A chain's latency bounds
// it: 64 spans of 8 heads of 128 x 128, 67 MB read and written in 13 us.
__global__ __launch_bounds__(256) void tf_decay_chain_kernel(DecayRuns R, int size, int chains) {
    const DecayRun &A = R.run[blockIdx.z];
    if (any_bad(A.bad)) return;
    const int heads = A.heads, spans = A.spans.n, dir = A.dir, lane = threadIdx.x % 64;
    const int h = blockIdx.x / (chains / 4), e = (blockIdx.y * 64 + lane) * 2;
    const long long step = (long long)dir * heads * size;
    for (int first = blockIdx.x % (chains / 4) * 4 + threadIdx.x / 64; first < spans; first += chains * 64) {
        const int mine = first + chains * lane;
        unsigned long long starts = __ballot(mine < spans && A.kind[mine < spans ? mine : 0] == 1);
        while (starts) {
            const int p = first + chains * __builtin_ctzll(starts);
            starts &= starts - 1;
            int cuts = 0;
            for (int i = p + dir; i >= 0 && i < spans; i += 64 * dir) {  // how many spans it goes on through whole
                const int j = i + dir * lane;
                const bool in = j >= 0 && j < spans;
                const unsigned long long on = __ballot(in && A.kind[in ? j : 0] == 2);
                const int run = ~on ? __builtin_ctzll(~on) : 64;
                cuts += run;
                if (run < 64) break;
            }
            if (cuts == 0) continue;
            float *l = A.local + ((long long)p * heads + h) * size + e;
            const float *m = A.mult + (long long)p * heads + h;
            o_f32x2 s = *(const o_f32x2 *)l;
            // Batches in turn, so that a batch's loads are waited for behind the next one's and not behind its stores (stores
            // under a branch would be waited for one by one: behind the end the last sum is stored again).
            constexpr int BATCH = 8;
            o_f32x2 x[2][BATCH];
            float w[2][BATCH];
            auto load = [&](int b, int i) {
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    const int k = i + j < cuts ? i + j + 1 : cuts;
                    x[b][j] = *(const o_f32x2 *)(l + k * step), w[b][j] = m[(long long)k * dir * heads];
                }
            };
            auto add = [&](int b, int i) {
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    const bool in = i + j < cuts;
                    if (in) s = x[b][j] + s * w[b][j];
                    *(o_f32x2 *)(l + (in ? i + j + 1 : cuts) * step) = s;
                }
            };
            load(0, 0);
            for (int i = 0; i < cuts; i += 2 * BATCH) {
                load(1, i + BATCH);
                add(0, i);
                load(0, i + 2 * BATCH);
                add(1, i + BATCH);
            }
        }
    }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    return v;
}

struct DecayGrad {
    Spans spans;
    const float *S, *U;          // the states and their gradients at the spans' ends
    const float *Sl, *Ul;        // from before the sequences' last chunks, decayed to their ends, and the last states' gradients; or null
    float *cut, *last;           // their inner products: [spans][heads], [n_seqs][heads]
    const float *g;
    long long gs;
    const double *da, *db;       // q dq - (k dk within chunks), k dk from the states
    float *dg, *part;            // part: [spans][heads], with one decay a head
    const int32_t *offsets;
    int n_seqs, heads, dir, size;
    const int *bad;
};

// Inner products of states and their gradients: a wave each, of the cut borders and of the sequences' ends.
__global__ __launch_bounds__(256) void tf_decay_dots_kernel(DecayGrad A) {
    if (any_bad(A.bad)) return;
    const long long item = (long long)blockIdx.x * 4 + threadIdx.x / 64, borders = (long long)A.spans.n * A.heads;
    const int lane = threadIdx.x % 64;
    const float *a, *b;
    float *to, d = 1.0f;
    if (item < borders) {
        const int p = (int)(item / A.heads), h = (int)(item % A.heads);
        const Spans::Border e = A.spans.border(p);
        if (!e.cuts) return;
        const int before = A.dir > 0 ? p - 1 : p, after = A.dir > 0 ? p : p - 1;
        a = A.S + ((long long)before * A.heads + h) * A.size;
        b = A.U + ((long long)after * A.heads + h) * A.size;
        const int r = A.dir > 0 ? e.row : e.row - 1;  // the first row after the border
        const float g = A.gs ? A.g[(long long)r * A.gs + h] : A.g[h];
        d = expf(g);
        to = A.cut + item;
    } else {
        const long long i = item - borders;
        if (!A.Sl || i >= (long long)A.n_seqs * A.heads) return;
        const int s = (int)(i / A.heads);
        if (A.offsets[s] == A.offsets[s + 1]) return;
        a = A.Sl + i * A.size, b = A.Ul + i * A.size;
        to = A.last + i;
    }
    float z = 0.0f;
    for (int e = 4 * lane; e < A.size; e += 256) {
        const o_f32x4 x = *(const o_f32x4 *)(a + e), y = *(const o_f32x4 *)(b + e);
        z += (x[0] * y[0] + x[1] * y[1]) + (x[2] * y[2] + x[3] * y[3]);
    }
    z = wave_sum(z);
    if (lane == 0) *to = z == 0.0f ? 0.0f : z * d;
}

// The decays' gradient of a span and head: sums from the span's last row (in the recurrence's order) to
// its first, sequence by sequence, by one wave (lane i).  Both terms' pairs within a chunk are the same numbers, added in fp64,
// so that those of rows that a head has forgotten cancel; what crosses the chunks' borders is good to fp32's digits of itself.
__device__ __forceinline__ void decay_grad(const DecayGrad &A, int item, int i) {
    const int p = item / A.heads, h = item % A.heads, dir = -A.dir;
    if (any_bad(A.bad)) {
        const float nan = __builtin_nanf("");
        const long long lo = (long long)p * A.spans.span;
        const long long hi = lo + A.spans.span < A.spans.n_rows ? lo + A.spans.span : A.spans.n_rows;
        if (A.gs)
            for (long long r = lo + i; r < hi; r += 64) A.dg[r * A.heads + h] = nan;
        else if (i == 0) A.part[(long long)p * A.heads + h] = nan;
        return;
    }
    const Spans::Border b0 = A.spans.border(p), b1 = A.spans.border(p + 1);
    const int olo = A.offsets[0], ohi = A.offsets[A.n_seqs];
    const int lo = b0.row > olo ? b0.row : olo, hi = b1.row < ohi ? b1.row : ohi, len = hi - lo;
    const int chunks = len > 0 ? (len + kChunk - 1) / kChunk : 0;  // the span kernel's
    double carry = 0.0, sum = 0.0;
    if (dir > 0 ? b0.cuts : b1.cuts) carry = (double)A.cut[(long long)(dir > 0 ? p : p + 1) * A.heads + h];
    for (int c = 0; c < chunks; ++c) {
        const int at = (dir > 0 ? c : chunks - 1 - c) * kChunk, rows = len - at < kChunk ? len - at : kChunk;
        const int row0 = dir > 0 ? lo + at : lo + at + rows - 1, r = row0 + dir * i;
        const bool live = i < rows;
        int f = i, e = i;  // the lanes of the sequence's last row (in the recurrence's order) and of its first, in the chunk
        double a = 0.0, b = 0.0, last = 0.0;
        if (live) {
            const int2 s = A.spans.info[r];
            f = dir > 0 ? s.x - row0 : row0 - (s.y - 1), e = dir > 0 ? s.y - 1 - row0 : row0 - s.x;
            a = A.da[(long long)r * A.heads + h], b = A.db[(long long)r * A.heads + h];
            if (f >= 0 && A.last) last = (double)A.last[(long long)seq_of_row(A.offsets, A.n_seqs, r) * A.heads + h];
        }
        double v = sum_from(a - b, f > 0 ? f : 0, i);
        if (A.last) {
            // What crosses the end: of a sequence that ends here, what its rows in the chunk have of the last state's gradient (the
            // same numbers that b takes away again, row by row) and what the state before them has.
            b = sum_from(b, f > 0 ? f : 0, i);
            const double all = __shfl(b, e < rows - 1 ? e : rows - 1) + last;
            if (f >= 0) v += all;
        }
        if (f < 0) v += carry;
        carry = lane_of(v, rows - 1);
        if (live) {
            const float g = A.gs ? A.g[(long long)r * A.gs + h] : A.g[h];
            if (g < -104.0f) v = 0.0;  // exp(g) is 0, and so is what it is multiplied with
            if (A.gs) A.dg[(long long)r * A.heads + h] = (float)v;
            else sum += v;
        }
    }
    if (!A.gs) {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        if (i == 0) A.part[(long long)p * A.heads + h] = (float)sum;
    }
}

__global__ __launch_bounds__(64) void tf_decay_sum_kernel(const float *__restrict__ part, int n, int heads, float *__restrict__ dg) {
    double v = 0.0;
    for (int p = threadIdx.x; p < n; p += 64) v += (double)part[(long long)p * heads + blockIdx.x];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    if (threadIdx.x == 0) dg[blockIdx.x] = (float)v;
}

// Gradients of queries and keys that several heads share: the heads' own, added in order.
struct DecayShare {
    const float *part[2];  // dq, dk
    void *out[2];
    long long stride[2], n_rows;
    const int32_t *offsets;
    const int *bad;
    int group, shared, width, n_seqs, blocks;  // heads that share one; how many are shared; workgroups of each
};
template <class T> __device__ __forceinline__ void decay_share(const DecayShare &S, int which, int block, int blocks, int tid) {
    const float *part = S.part[which];
    typename T::E *out = (typename T::E *)S.out[which];
    const long long stride = S.stride[which];
    const int per = S.shared * S.width / 4;
    const bool wrong = any_bad(S.bad);
    const long long lo = wrong ? 0 : S.offsets[0], hi = wrong ? S.n_rows : S.offsets[S.n_seqs];
    for (long long i = lo * per + (long long)block * 256 + tid; i < hi * per; i += (long long)blocks * 256) {
        const long long r = i / per;
        const int c = (int)(i - r * per) * 4, hk = c / S.width, d = c - hk * S.width;
        const float *p = part + (r * S.shared + hk) * (long long)S.group * S.width + d;
        o_f32x4 v = *(const o_f32x4 *)p;
        for (int j = 1; j < S.group; ++j) v += *(const o_f32x4 *)(p + (long long)j * S.width);
        store4<T>(out + r * stride + c, v);
    }
}

// Both, as they wait for different things: the decays' gradient for one row sum after another (a wave a span and head,
// first of the launch), the sums over sharing heads for memory.  Apart they took 7 and 9 us for 9.6 thousand rows.
template <class T> __global__ __launch_bounds__(256) void tf_decay_last_kernel(DecayGrad G, DecayShare S) {
    const int items = G.spans.n * G.heads, waves = (items + 3) / 4, share = (int)blockIdx.x - waves;
    if (share < 0) {
        const int item = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        if (item < items) decay_grad(G, item, threadIdx.x % 64);
    } else {
        decay_share<T>(S, share & 1, share >> 1, S.blocks, threadIdx.x);
    }
}

// One token of every sequence: the state is read, decayed, added to, multiplied with q and written in one
// pass.  A workgroup of 256 threads has one head's state; a thread four neighbouring columns of every
// 256 / (dv / 4)-th row.  Memory bounds it: 509 sequences of 16 heads of 64 x 128, 538 MB in 98 us (5.5 TB/s; a copy reaches
// 5.1).
template <class T>
__global__ __launch_bounds__(256) void tf_decay_step_kernel(const void *__restrict__ q_, long long qs, const void *__restrict__ k_,
                                                            long long ks, const void *__restrict__ v_, long long vs,
                                                            const float *__restrict__ g, long long gs, int heads, int group,
                                                            int dk, int dv, float scale, const float *s0, float *s1, void *out,
                                                            long long os) {
    typedef typename T::E E;
    __shared__ float qk[2][128];
    __shared__ o_f32x4 sums[256];
    const long long item = blockIdx.x;
    const long long i = item / heads;
    const int h = (int)(item % heads), tid = threadIdx.x, hk = h / group;
    if (tid < 2 * dk) {
        const int w = tid >= dk, d = w ? tid - dk : tid;
        qk[w][d] = w ? (float)((const E *)k_)[i * ks + hk * dk + d] : (float)((const E *)q_)[i * qs + hk * dk + d];
    }
    const int cols = dv / 4, rows = 256 / cols, col = tid % cols, row = tid / cols;
    const float decay = expf(gs ? g[i * gs + h] : g[h]);
    const E *vp = (const E *)v_ + i * vs + (long long)h * dv + 4 * col;
    const o_f32x4 v = {(float)vp[0], (float)vp[1], (float)vp[2], (float)vp[3]};
    const float *s = s0 + item * dk * dv;
    float *t = s1 + item * dk * dv;
    __syncthreads();
    o_f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int d = row; d < dk; d += rows) {
        o_f32x4 x = *(const o_f32x4 *)(s + d * dv + 4 * col);
        x = x * decay + v * qk[1][d];
        *(o_f32x4 *)(t + d * dv + 4 * col) = x;
        o += x * qk[0][d];
    }
    sums[tid] = o;
    __syncthreads();
    if (tid < cols) {
        for (int r = 1; r < rows; ++r) o += sums[r * cols + tid];
        store4<T>((E *)out + i * os + (long long)h * dv + 4 * tid, o * scale);
    }
}

// ---------------------------------------------------------------------------------------------------------

tf_status decay_check(const tf_decay_config *c) {
    if (!c || !elem_ok(c->elem) || c->n_heads < 1 || c->n_qk_heads < 1 || c->n_heads % c->n_qk_heads || c->d_k < 1 || c->d_v < 1)
        return TF_EINVAL;
    if (!std::isfinite(c->scale) || (c->reverse != 0 && c->reverse != 1) || c->clear < 0 || c->clear > 15) return TF_EINVAL;
    auto width = [](int d) { return d == 32 || d == 64 || d == 128; };
    if (!width(c->d_k) || !width(c->d_v) || c->n_heads > 1024) return TF_EUNSUPPORTED;
    return TF_OK;
}

// Rows of a span.  Four workgroups for each compute unit (two of the wide heads'), of which an instance's registers and LDS let
// three, two or one run at a time, and no more than that: every border that cuts a sequence costs a state written and read.  One
// sequence of 32 768 rows, 8 heads of 128 x 128: spans of 128 rows 239 us, 256 194, 512 157, 1024 154.  Not beyond 512 rows: the
// last workgroups' share of 918 161 rows of tracks grows (spans of 512 362 us, 1024 367, 2048 373).
int decay_span(const tf_decay_config *c, int64_t n_rows) {
    int64_t s = n_rows * c->n_heads / (c->d_k * c->d_v > 64 * 64 ? 512 : 1024) / kChunk * kChunk;
    if (s < kMinSpan) s = kMinSpan;
    if (s > 512) s = 512;
    if (n_rows <= 2 * kMinSpan) s = 2 * kMinSpan;  // one span: no state to pass, two launches less
    return (int)s;
}
int64_t decay_spans(const tf_decay_config *c, int64_t n_rows) {
    const int64_t s = decay_span(c, n_rows), n = (n_rows + s - 1) / s;
    return n < 1 ? 1 : n;
}

struct Room {  // parts of the workspace, each at a multiple of 256 bytes
    char *base;
    size_t used = 0;
    explicit Room(void *b) : base((char *)b) {}
    template <class V> V *take(int64_t n) {
        V *p = (V *)(base + used);
        used += ((size_t)n * sizeof(V) + 255) / 256 * 256;
        return p;
    }
};
struct Plan {
    int2 *info;
    int *bad, *kind[2];
    float *local[2], *mult[2];
    double *da, *db;
    float *cut, *last, *sl, *part, *dq, *dk;
    size_t bytes;
};
Plan decay_plan(const tf_decay_config *c, int64_t n_rows, int64_t n_seqs, bool back, bool states, void *base) {
    Room r(base);
    Plan p = {};
    const int64_t spans = decay_spans(c, n_rows), h = c->n_heads, size = (int64_t)c->d_k * c->d_v;
    p.bad = r.take<int>(kCheckers);
    p.info = r.take<int2>(n_rows);
    for (int i = 0; i < (back ? 2 : 1); ++i) {
        p.kind[i] = r.take<int>(spans);
        p.mult[i] = r.take<float>(spans * h);
        p.local[i] = r.take<float>(spans > 1 ? spans * h * size : 0);
    }
    if (back) {
        p.da = r.take<double>(n_rows * h);
        p.db = r.take<double>(n_rows * h);
        p.cut = r.take<float>(spans * h);
        p.part = r.take<float>(spans * h);
        if (states) {
            p.last = r.take<float>(n_seqs * h);
            p.sl = r.take<float>(n_seqs * h * size);
        }
        if (c->n_heads != c->n_qk_heads) {
            p.dq = r.take<float>(n_rows * h * c->d_k);
            p.dk = r.take<float>(n_rows * h * c->d_k);
        }
    }
    p.bytes = r.used;
    return p;
}

template <class T, int DK, int DV> void span_mode(const DecayRuns &R, int runs, int mode, hipStream_t s) {
    const dim3 grid((unsigned)(R.run[0].spans.n * R.run[0].heads), runs), block(span_threads(DV));
    switch (mode) {
        case DECAY_STATE: hipLaunchKernelGGL((tf_decay_span_kernel<T, DK, DV, DECAY_STATE>), grid, block, 0, s, R); break;
        case DECAY_OUT: hipLaunchKernelGGL((tf_decay_span_kernel<T, DK, DV, DECAY_OUT>), grid, block, 0, s, R); break;
        default: hipLaunchKernelGGL((tf_decay_span_kernel<T, DK, DV, DECAY_DOT>), grid, block, 0, s, R); break;
    }
}
template <class T, int DK> void span_dv(const DecayRuns &R, int runs, int dv, int mode, hipStream_t s) {
    if (dv == 32) span_mode<T, DK, 32>(R, runs, mode, s);
    else if (dv == 64) span_mode<T, DK, 64>(R, runs, mode, s);
    else span_mode<T, DK, 128>(R, runs, mode, s);
}
template <class T> void span_dk(const DecayRuns &R, int runs, int dk, int dv, int mode, hipStream_t s) {
    if (dk == 32) span_dv<T, 32>(R, runs, dv, mode, s);
    else if (dk == 64) span_dv<T, 64>(R, runs, dv, mode, s);
    else span_dv<T, 128>(R, runs, dv, mode, s);
}
void span_run(int elem, const DecayRuns &R, int runs, int dk, int dv, int mode, hipStream_t s) {
    if (elem == TF_ELEM_BF16) span_dk<ElemBF16>(R, runs, dk, dv, mode, s);
    else if (elem == TF_ELEM_FP32) span_dk<ElemF32>(R, runs, dk, dv, mode, s);
    else span_dk<ElemF16>(R, runs, dk, dv, mode, s);
}
// The states at the spans' ends of runs whose arguments k, v, g, s0 are set.
void chain_run(int elem, DecayRuns R, int runs, int dk, int dv, hipStream_t s) {
    const DecayRun &A = R.run[0];
    if (A.spans.n < 2) return;
    for (int i = 0; i < runs; ++i) R.run[i].sf = nullptr, R.run[i].turned = 0;
    span_run(elem, R, runs, dk, dv, DECAY_STATE, s);
    // (as many waves for the chains as are on the chip at once: one without a chain still takes 4 us)
    const int64_t pieces = (int64_t)A.heads * (dk * dv / 128) * runs;
    int chains = (int)(1024 / pieces) * 4;
    chains = chains < 4 ? 4 : chains > 64 ? 64 : chains;
    hipLaunchKernelGGL(tf_decay_chain_kernel, dim3((unsigned)(chains / 4 * A.heads), (unsigned)(dk * dv / 128), runs), dim3(256), 0, s, R,
                       dk * dv, chains);
}
// (s0, sf: the states of `size` values that sequences without rows pass through; sf null: none)
void index_run(const int32_t *offsets, int n_seqs, int64_t n_rows, const Plan &p, int32_t *flags, long long size, const float *s0,
               float *sf, const DecayClear &clear, hipStream_t s) {
    const int64_t per = ((int64_t)n_seqs + 1023) / 1024, states = sf && per ? (n_seqs + per - 1) / per : 0;
    hipLaunchKernelGGL(tf_decay_index_kernel, dim3((unsigned)(kCheckers + (n_rows + kIndexRows - 1) / kIndexRows + states)), dim3(256), 0, s,
                       offsets, n_seqs, (int)n_rows, p.info, p.bad, flags, size, (int)per, s0, sf, clear);
}
void last_run(int elem, const DecayGrad &G, const DecayShare &S, hipStream_t s) {
    const dim3 grid((unsigned)((G.spans.n * G.heads + 3) / 4 + 2 * S.blocks)), block(256);
    if (elem == TF_ELEM_BF16) hipLaunchKernelGGL((tf_decay_last_kernel<ElemBF16>), grid, block, 0, s, G, S);
    else if (elem == TF_ELEM_FP32) hipLaunchKernelGGL((tf_decay_last_kernel<ElemF32>), grid, block, 0, s, G, S);
    else hipLaunchKernelGGL((tf_decay_last_kernel<ElemF16>), grid, block, 0, s, G, S);
}

bool decay_sizes_ok(const tf_decay_config *c, int64_t n_rows, int32_t n_seqs) {
    // rows and sequences are 32-bit numbers (with room for the last step of the index's loops), and so are a launch's threads
    return n_rows <= INT32_MAX - 2048 && n_seqs <= INT32_MAX - 512 * kCheckers && decay_spans(c, n_rows) * c->n_heads < 1 << 24;
}

// A chunk's rows are addressed by 32-bit offsets.
constexpr int64_t kFarthest = 1 << 24;

}  // namespace

extern "C" size_t tf_decay_workspace_size(const tf_decay_config *c, int64_t n_rows) {
    if (decay_check(c) != TF_OK || n_rows < 0 || !decay_sizes_ok(c, n_rows, 0)) return 0;
    return decay_plan(c, n_rows, 0, false, false, nullptr).bytes;
}

extern "C" size_t tf_decay_backward_workspace_size(const tf_decay_config *c, int64_t n_rows, int32_t n_seqs, int32_t with_d_state) {
    if (decay_check(c) != TF_OK || n_rows < 0 || n_seqs < 0 || !decay_sizes_ok(c, n_rows, n_seqs)) return 0;
    return decay_plan(c, n_rows, n_seqs, true, with_d_state != 0, nullptr).bytes;
}

extern "C" tf_status tf_decay_attention(const tf_decay_config *c, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                                        const void *v, int64_t v_stride, const float *log_decay, int64_t decay_stride,
                                        int64_t n_rows, const int32_t *offsets, int32_t n_seqs, const float *initial_state,
                                        void *workspace, size_t workspace_bytes, void *out, int64_t out_stride,
                                        float *final_state, int32_t *flags, hipStream_t stream) {
    const tf_status st = decay_check(c);
    if (st != TF_OK) return st;
    const int64_t qw = (int64_t)c->n_qk_heads * c->d_k, vw = (int64_t)c->n_heads * c->d_v;
    if (n_rows < 0 || n_seqs < 0 || (decay_stride != 0 && decay_stride < c->n_heads)) return TF_EINVAL;
    if (!stride_ok(q_stride, qw, c->elem) || !stride_ok(k_stride, qw, c->elem) || !stride_ok(v_stride, vw, c->elem) ||
        !stride_ok(out_stride, vw, c->elem))
        return TF_EINVAL;
    if (!decay_sizes_ok(c, n_rows, n_seqs) || !strides_fit({q_stride, k_stride, v_stride, out_stride}, kFarthest)) return TF_EUNSUPPORTED;
    if (n_seqs == 0 && !(c->clear && n_rows > 0)) return TF_OK;
    if (!offsets || !workspace) return TF_EINVAL;
    if (n_rows > 0 && (!q || !k || !v || !out || !log_decay)) return TF_EINVAL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(initial_state) || !aligned16(final_state) ||
        ((uintptr_t)workspace & 255))
        return TF_EINVAL;
    if (n_rows > 0 && over_inputs({out}, {q, k, v, log_decay})) return TF_EINVAL;
    if (over_inputs({out, final_state, workspace}, {initial_state}) || twice({out, final_state, workspace})) return TF_EINVAL;
    if (over_inputs({workspace, final_state}, {q, k, v, log_decay, offsets})) return TF_EINVAL;
    const Plan p = decay_plan(c, n_rows, n_seqs, false, false, workspace);
    if (workspace_bytes < p.bytes) return TF_EINVAL;
    DecayClear clear = {};
    if (c->clear & 1) clear.add(0, out, out_stride, vw, elem_bytes(c->elem));
    index_run(offsets, n_seqs, n_rows, p, flags, (long long)c->n_heads * c->d_k * c->d_v, initial_state, final_state, clear, stream);
    if (n_seqs > 0 && (n_rows > 0 || final_state)) {
        DecayRun A = {};
        const int group = c->n_heads / c->n_qk_heads;
        A.q = q, A.k = k, A.v = v, A.qs = q_stride, A.ks = k_stride, A.vs = v_stride;
        A.group = group, A.qg = A.kg = 1;
        A.out = out, A.os = out_stride;
        A.g = log_decay, A.gs = decay_stride;
        A.s0 = initial_state, A.sf = final_state;
        A.local = p.local[0], A.mult = p.mult[0], A.kind = p.kind[0];
        A.out_scale = c->scale, A.kv_scale = 1.0f;
        A.offsets = offsets, A.n_seqs = n_seqs, A.heads = c->n_heads, A.dir = c->reverse ? -1 : 1, A.bad = p.bad;
        A.spans = {p.info, (int)n_rows, decay_span(c, n_rows), (int)decay_spans(c, n_rows)};
        const DecayRuns R = {{A}};
        chain_run(c->elem, R, 1, c->d_k, c->d_v, stream);
        span_run(c->elem, R, 1, c->d_k, c->d_v, DECAY_OUT, stream);
    }
    return hipGetLastError() == hipSuccess ? TF_OK : TF_EHIP;
}

extern "C" tf_status tf_decay_attention_backward(const tf_decay_config *c, const void *d_out, int64_t d_out_stride, const void *q,
                                                 int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                                                 int64_t v_stride, const float *log_decay, int64_t decay_stride, int64_t n_rows,
                                                 const int32_t *offsets, int32_t n_seqs, const float *initial_state,
                                                 const float *d_state, void *workspace, size_t workspace_bytes, void *dq,
                                                 int64_t dq_stride, void *dk, int64_t dk_stride, void *dv, int64_t dv_stride,
                                                 float *d_log_decay, float *d_initial, int32_t *flags, hipStream_t stream) {
    const tf_status st = decay_check(c);
    if (st != TF_OK) return st;
    const int64_t qw = (int64_t)c->n_qk_heads * c->d_k, vw = (int64_t)c->n_heads * c->d_v;
    if (n_rows < 0 || n_seqs < 0 || (decay_stride != 0 && decay_stride < c->n_heads)) return TF_EINVAL;
    if (!stride_ok(q_stride, qw, c->elem) || !stride_ok(k_stride, qw, c->elem) || !stride_ok(v_stride, vw, c->elem) ||
        !stride_ok(d_out_stride, vw, c->elem) || !stride_ok(dq_stride, qw, c->elem) || !stride_ok(dk_stride, qw, c->elem) ||
        !stride_ok(dv_stride, vw, c->elem))
        return TF_EINVAL;
    if (!decay_sizes_ok(c, n_rows, n_seqs) ||
        !strides_fit({q_stride, k_stride, v_stride, d_out_stride, dq_stride, dk_stride, dv_stride}, kFarthest))
        return TF_EUNSUPPORTED;
    if (!offsets || !workspace || (!decay_stride && !d_log_decay)) return TF_EINVAL;
    if (n_rows > 0 && (!q || !k || !v || !d_out || !dq || !dk || !dv || !log_decay || !d_log_decay)) return TF_EINVAL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(d_out) || !aligned16(dq) || !aligned16(dk) ||
        !aligned16(dv) || !aligned16(initial_state) || !aligned16(d_state) || !aligned16(d_initial) || ((uintptr_t)workspace & 255))
        return TF_EINVAL;
    if (n_rows > 0 && over_inputs({dq, dk, dv, d_log_decay}, {d_out, q, k, v, log_decay})) return TF_EINVAL;
    if (n_seqs > 0 && over_inputs({d_initial}, {initial_state, d_state})) return TF_EINVAL;
    if (over_inputs({workspace}, {d_out, q, k, v, log_decay, offsets, initial_state, d_state}) ||
        twice({dq, dk, dv, d_log_decay, d_initial, workspace}))
        return TF_EINVAL;
    const Plan p = decay_plan(c, n_rows, n_seqs, true, d_state != nullptr, workspace);
    if (workspace_bytes < p.bytes) return TF_EINVAL;
    const int H = c->n_heads, group = H / c->n_qk_heads, dir = c->reverse ? -1 : 1, size = c->d_k * c->d_v;
    DecayClear clear = {};
    if (c->clear & 1) clear.add(0, dq, dq_stride, qw, elem_bytes(c->elem));
    if (c->clear & 2) clear.add(1, dk, dk_stride, qw, elem_bytes(c->elem));
    if (c->clear & 4) clear.add(2, dv, dv_stride, vw, elem_bytes(c->elem));
    if ((c->clear & 8) && decay_stride) clear.add(3, d_log_decay, H, H, 4);
    index_run(offsets, n_seqs, n_rows, p, flags, (long long)H * size, d_state, d_initial, clear, stream);
    DecayShare S = {};
    DecayRun A = {};
    A.group = group, A.g = log_decay, A.gs = decay_stride;
    A.offsets = offsets, A.n_seqs = n_seqs, A.heads = H, A.bad = p.bad;
    A.spans = {p.info, (int)n_rows, decay_span(c, n_rows), (int)decay_spans(c, n_rows)};
    if (n_seqs > 0 && (n_rows > 0 || d_initial)) {
        // the states at the spans' ends, and their gradients
        DecayRun F = A;
        F.k = k, F.ks = k_stride, F.kg = 1, F.v = v, F.vs = v_stride;
        F.s0 = initial_state, F.dir = dir, F.out_scale = F.kv_scale = 1.0f;
        F.local = p.local[0], F.mult = p.mult[0], F.kind = p.kind[0];
        DecayRun B = A;
        B.k = q, B.ks = q_stride, B.kg = 1, B.v = d_out, B.vs = d_out_stride;
        B.s0 = d_state, B.dir = -dir, B.shift = 1, B.out_scale = 1.0f, B.kv_scale = c->scale;
        B.local = p.local[1], B.mult = p.mult[1], B.kind = p.kind[1];
        chain_run(c->elem, {{F, B}}, 2, c->d_k, c->d_v, stream);
        const bool shared = group > 1;
        // dq
        DecayRun Q = F;
        Q.q = d_out, Q.qs = d_out_stride, Q.qg = 0;
        Q.k = v, Q.ks = v_stride, Q.kg = 0;
        Q.v = k, Q.vs = k_stride, Q.vg = 1;
        Q.x = q, Q.xs = q_stride, Q.xg = 1;
        Q.out = shared ? (void *)p.dq : dq, Q.os = shared ? (int64_t)H * c->d_k : dq_stride, Q.out_f32 = shared;
        Q.turned = 1, Q.sf = p.sl, Q.sf_before = 1, Q.db = p.da, Q.pairs = 1, Q.out_scale = c->scale, Q.kv_scale = 1.0f;
        // dk
        DecayRun K = B;
        K.q = v, K.qs = v_stride, K.qg = 0;
        K.k = d_out, K.ks = d_out_stride, K.kg = 0;
        K.v = q, K.vs = q_stride, K.vg = 1;
        K.x = k, K.xs = k_stride, K.xg = 1;
        K.out = shared ? (void *)p.dk : dk, K.os = shared ? (int64_t)H * c->d_k : dk_stride, K.out_f32 = shared;
        K.turned = 1, K.db = p.db;
        // dv, and the initial states' gradients
        DecayRun V = B;
        V.q = k, V.qs = k_stride, V.qg = 1;
        V.out = dv, V.os = dv_stride;
        V.sf = d_initial, V.sf_decay = 1;
        if (c->d_k == c->d_v) {  // (9.6 thousand rows, which leave compute units idle: together 75 us, apart 59 and 27)
            V.x = nullptr;
            span_run(c->elem, {{Q, K, V}}, 3, c->d_k, c->d_v, DECAY_DOT, stream);
        } else {
            span_run(c->elem, {{Q, K}}, 2, c->d_v, c->d_k, DECAY_DOT, stream);
            span_run(c->elem, {{V}}, 1, c->d_k, c->d_v, DECAY_OUT, stream);
        }
        if (shared) {
            const int64_t items = n_rows * c->n_qk_heads * c->d_k / 4, blocks = (items + 255) / 256;
            S = {{p.dq, p.dk}, {dq, dk}, {dq_stride, dk_stride}, n_rows, offsets, p.bad, group, c->n_qk_heads, c->d_k, n_seqs,
                 (int)(blocks < 8192 ? blocks : 8192)};
        }
    }
    DecayGrad G = {};
    G.spans = A.spans, G.S = p.local[0], G.U = p.local[1], G.Sl = p.sl, G.Ul = d_state, G.cut = p.cut, G.last = p.last;
    G.g = log_decay, G.gs = decay_stride, G.da = p.da, G.db = p.db, G.dg = d_log_decay, G.part = p.part;
    G.offsets = offsets, G.n_seqs = n_seqs, G.heads = H, G.dir = dir, G.size = size, G.bad = p.bad;
    if (n_rows > 0 && n_seqs > 0) {
        const long long items = (long long)G.spans.n * H + (d_state ? (long long)n_seqs * H : 0);
        if (G.spans.n > 1 || d_state)
            hipLaunchKernelGGL(tf_decay_dots_kernel, dim3((unsigned)((items + 3) / 4)), dim3(256), 0, stream, G);
    }
    if (n_rows > 0 || !decay_stride)
        last_run(c->elem, G, S, stream);
    if (!decay_stride)
        hipLaunchKernelGGL(tf_decay_sum_kernel, dim3(H), dim3(64), 0, stream, p.part, G.spans.n, H, d_log_decay);
    return hipGetLastError() == hipSuccess ? TF_OK : TF_EHIP;
}

extern "C" tf_status tf_decay_attention_step(const tf_decay_config *c, const void *q, int64_t q_stride, const void *k,
                                             int64_t k_stride, const void *v, int64_t v_stride, const float *log_decay,
                                             int64_t decay_stride, int32_t n_seqs, const float *state, float *state_out, void *out,
                                             int64_t out_stride, hipStream_t stream) {
    const tf_status st = decay_check(c);
    if (st != TF_OK) return st;
    const int64_t qw = (int64_t)c->n_qk_heads * c->d_k, vw = (int64_t)c->n_heads * c->d_v;
    if (n_seqs < 0 || (decay_stride != 0 && decay_stride < c->n_heads)) return TF_EINVAL;
    if (!stride_ok(q_stride, qw, c->elem) || !stride_ok(k_stride, qw, c->elem) || !stride_ok(v_stride, vw, c->elem) ||
        !stride_ok(out_stride, vw, c->elem))
        return TF_EINVAL;
    if ((int64_t)n_seqs * c->n_heads >= 1 << 24) return TF_EUNSUPPORTED;  // a launch has fewer than 2^32 threads
    if (n_seqs == 0) return TF_OK;
    if (!q || !k || !v || !log_decay || !state || !state_out || !out) return TF_EINVAL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(state) || !aligned16(state_out))
        return TF_EINVAL;
    if (over_inputs({out}, {q, k, v, log_decay, state}) || over_inputs({state_out}, {q, k, v, log_decay}) || out == state_out)
        return TF_EINVAL;
    const dim3 grid((unsigned)((int64_t)n_seqs * c->n_heads));
    const int group = c->n_heads / c->n_qk_heads;
#define TF_STEP(T)                                                                                                               \
    hipLaunchKernelGGL((tf_decay_step_kernel<T>), grid, dim3(256), 0, stream, q, (long long)q_stride, k, (long long)k_stride, v, \
                       (long long)v_stride, log_decay, (long long)decay_stride, (int)c->n_heads, group, (int)c->d_k,             \
                       (int)c->d_v, c->scale, state, state_out, out, (long long)out_stride)
    if (c->elem == TF_ELEM_BF16) TF_STEP(ElemBF16);
    else if (c->elem == TF_ELEM_FP32) TF_STEP(ElemF32);
    else TF_STEP(ElemF16);
#undef TF_STEP
    return hipGetLastError() == hipSuccess ? TF_OK : TF_EHIP;
}
