// Queries and keys normalised per head and rotated by their positions, in one
// pass, with its backward pass (gfx950).
//
//   n = x / sqrt(mean(x^2) + eps) * gain         (each head of a row)
//   (lo, hi) -> (lo cos a - hi sin a, lo sin a + hi cos a),  a = position * base^(-2 j / R)
//
// for pair j of the first R values.  Backward: the rotation is orthogonal, so
// its gradient is the rotation by -a; with w = gain * dz and h = x / rms
//   dx = (w - h mean(w h)) / rms,   dgain = sum over rows and heads of dz h.
//
// A lane holds 16 values of one head, both halves of 8 pairs, so a head is
// D / 16 neighbouring lanes and its sums are log2(D / 16) lane exchanges.
// The angles are the same for all heads of a row: a workgroup takes a tile of
// rows, its threads fill cos and sin of the tile's (row, pair) angles in LDS
// once, and every head of the row reads them from there (lanes of different
// heads read the same words, which LDS broadcasts).  An angle is position times
// frequency in fp64, in turns, less its whole turns: at positions near 2^31 it is
// good to 2^-23 turns, where an fp32 angle has lost whole turns.
// Everything between the loads and the one rounding at the store is fp32.
//
// Memory bounds it: 918 thousand rows of 3 + 3 heads of 64, bf16, 1.41 GB in 315 us (4.5 TB/s; a copy reaches 5.1), and
// backward 22 thousand rows of 16 + 4 heads of 128, 342 MB in 89 us (3.8 TB/s), 8 of them the gains' sums, whose launch is
// latency.  16 values a lane: a lane then has both halves of its pairs in two or four 16-byte loads, and a head's sums are two
// to four exchanges; with 32 registers of gains' sums the backward pass has three workgroups a compute unit.
#include "ops.h"

#include <cmath>

namespace {

constexpr int kNormBlock = 256;
constexpr int kNormAngles = 2048;  // (row, pair) angles of a tile: 16 KB of cos and sin
constexpr int kNormRows = kNormAngles / 8;  // rows of a tile, at most: at least 8 pairs are rotated
constexpr int kMaxPairs = 128;
constexpr int kNormParts = 1024;  // workgroups of a backward launch: each writes a partial gain gradient

struct Turns {  // turns per position of each pair
    double f[kMaxPairs];
};

struct NormArgs {
    const void *x[2];    // q, k
    const void *dy[2];   // backward only
    void *y[2];          // outputs (dx for the backward pass)
    const float *gain[2];
    long long xs[2], ds[2], ys[2];  // row strides, elements
    int heads[2];
    long long n_rows;
    const int32_t *positions, *offsets;
    int n_seqs, rot, tile;  // rotated values; rows of a tile
    int clear;              // outputs (a bit each) whose rows outside of all sequences become zeros
    int blocks;             // workgroups of the tiles
    unsigned per_head[2], per_pair;  // 2^32 over the heads, the pairs (rounded down)
    float eps;
    float *parts;  // backward: [workgroups][2][D]
};

// The 16 values of a lane: pairs (v[i], v[8 + i]).  Rotated and not interleaved, they are 8 values
// of each half of the rotated part; else 16 consecutive ones, neighbours paired when rotated.
template <typename T, bool PAIRED>
__device__ __forceinline__ void norm_load(const typename T::E *p, int l, int rot, float v[16]) {
    const bool turned = 16 * l < rot;
    const int a = (!PAIRED && turned) ? 8 * l : 16 * l;
    const int b = (!PAIRED && turned) ? 8 * l + rot / 2 : 16 * l + 8;
    const o_f32x8 x = load8<T>(p + a), y = load8<T>(p + b);
    if (PAIRED) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = x[2 * i], v[8 + i] = x[2 * i + 1], v[4 + i] = y[2 * i], v[12 + i] = y[2 * i + 1];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = x[i], v[8 + i] = y[i];
    }
}
template <typename T, bool PAIRED>
__device__ __forceinline__ void norm_store(typename T::E *p, int l, int rot, const float v[16]) {
    const bool turned = 16 * l < rot;
    const int a = (!PAIRED && turned) ? 8 * l : 16 * l;
    const int b = (!PAIRED && turned) ? 8 * l + rot / 2 : 16 * l + 8;
    o_f32x8 x, y;
    if (PAIRED) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = v[i], x[2 * i + 1] = v[8 + i], y[2 * i] = v[4 + i], y[2 * i + 1] = v[12 + i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = v[i], y[i] = v[8 + i];
    }
    store8<T>(p + a, x);
    store8<T>(p + b, y);
}

// a / b, with r = 2^32 / b rounded down (or 2^32 - 1): at most one too small.
__device__ __forceinline__ int over(int a, int b, unsigned r) {
    const int d = (int)__umulhi((unsigned)a, r);
    return a - d * b >= b ? d + 1 : d;
}

template <int L> __device__ __forceinline__ float head_sum(float s) {
#pragma unroll
    for (int m = 1; m < L; m *= 2) s += __shfl_xor(s, m);
    return s;
}

// Zeros in the rows before the first sequence and behind the last, of the outputs that are to be cleared, a wave a row: the work
// of the workgroups behind A.blocks (`wave` of `waves`).  Within the tiles' loop it cost the others' registers 9 % of their time.
template <typename T, int D> __device__ __forceinline__ void norm_clear(const NormArgs &A, int wave, int waves, int lane) {
    const long long first = A.offsets[0], last = A.offsets[A.n_seqs];
    for (int w = 0; w < 2; ++w) {
        if (!(A.clear >> w & 1)) continue;
        for (long long r = wave; r < A.n_rows; r += waves) {
            if (r >= first && r < last) {  // on to the first of this wave's rows that is behind the sequences
                r += (last - r - 1) / waves * waves;
                continue;
            }
            typename T::E *y = (typename T::E *)A.y[w] + r * A.ys[w];
            for (int c = lane * 8; c < A.heads[w] * D; c += 512) store8<T>(y + c, o_f32x8{});
        }
    }
}

// (the registers' limits are those that no instance spills at)
template <typename T, int D, bool PAIRED, bool BACK>
__global__ __launch_bounds__(kNormBlock, BACK ? 3 : D <= 64 && !PAIRED ? 5 : 4) void tf_qk_norm_kernel(NormArgs A, Turns turns) {
    constexpr int L = D / 16;  // lanes of a head
    typedef typename T::E E;
    __shared__ __attribute__((aligned(16))) float cs[2 * kNormAngles];  // [row][cos, sin][pair]
    __shared__ double at[kNormRows];  // positions
    __shared__ int live[kNormRows];
    const int tid = threadIdx.x, l = tid % L;
    if ((int)blockIdx.x >= A.blocks) {
        norm_clear<T, D>(A, ((int)blockIdx.x - A.blocks) * (kNormBlock / 64) + tid / 64, ((int)gridDim.x - A.blocks) * (kNormBlock / 64),
                         tid % 64);
        return;
    }
    const int pairs = A.rot / 2;
    const bool turned = 16 * l < A.rot;

    float acc[2][16];
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[w][i] = 0.0f;
    long long first = 0, last = A.n_rows;
    if (A.offsets) {
        const long long o = A.offsets[0], e = A.offsets[A.n_seqs];
        first = o > 0 ? o : 0;
        last = e < last ? e : last;
    }
    const long long tiles = (A.n_rows + A.tile - 1) / A.tile;
    for (long long t = blockIdx.x; t < tiles; t += A.blocks) {
        const long long r0 = t * A.tile;
        const int rows = (int)(A.n_rows - r0 < A.tile ? A.n_rows - r0 : A.tile);
        if (r0 >= last || r0 + rows <= first) continue;
        __syncthreads();  // the last tile's angles are read
        for (int i = tid; i < rows; i += kNormBlock) {
            const long long r = r0 + i;
            double pos = (double)r;
            if (A.positions) pos = (double)A.positions[r];
            else if (A.offsets) {
                const int s = seq_of_row(A.offsets, A.n_seqs, r);
                pos = s < 0 ? 0.0 : (double)(r - A.offsets[s]);
            }
            live[i] = r >= first && r < last;
            at[i] = pos;
        }
        __syncthreads();
        for (int i = tid; i < rows * pairs; i += kNormBlock) {
            const int r = over(i, pairs, A.per_pair), j = i - r * pairs;
            double a = at[r] * turns.f[j];
            a -= rint(a);
            float sn, co;
            if constexpr (sizeof(E) == 4) {
                sincospif(2.0f * (float)a, &sn, &co);
            } else {  // the hardware's, of turns: within 2^-20, below the outputs' rounding
                sn = __builtin_amdgcn_sinf((float)a), co = __builtin_amdgcn_cosf((float)a);
            }
            cs[2 * pairs * r + j] = co, cs[2 * pairs * r + pairs + j] = sn;
        }
        __syncthreads();
        // queries, then keys
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            float gain[16];
            norm_load<ElemF32, PAIRED>(A.gain[w], l, A.rot, gain);
            const int heads = A.heads[w], items = rows * heads * L;
            const unsigned per = A.per_head[w];
            // (the tile's first row is a scalar, 256 rows of a stride fit in 32 bits)
            const E *x = (const E *)A.x[w] + r0 * A.xs[w], *dy = BACK ? (const E *)A.dy[w] + r0 * A.ds[w] : nullptr;
            E *y = (E *)A.y[w] + r0 * A.ys[w];
            const int xs = (int)A.xs[w], ds = (int)A.ds[w], ys = (int)A.ys[w];
            for (int it = tid; it < items; it += kNormBlock) {
                const int rh = it / L, r = over(rh, heads, per), h = rh - r * heads;
                if (!live[r]) continue;  // the lanes of a head agree
                float v[16], c[8], s[8];
                norm_load<T, PAIRED>(x + (unsigned)(r * xs + h * D), l, A.rot, v);
                if (turned) {
                    const o_f32x4 *p = (const o_f32x4 *)&cs[2 * pairs * r + 8 * l], *q = (const o_f32x4 *)&cs[2 * pairs * r + pairs + 8 * l];
                    const o_f32x4 c0 = p[0], c1 = p[1], s0 = q[0], s1 = q[1];
#pragma unroll
                    for (int i = 0; i < 4; ++i) c[i] = c0[i], c[4 + i] = c1[i], s[i] = s0[i], s[4 + i] = s1[i];
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) c[i] = 1.0f, s[i] = 0.0f;
                }
                float sq = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) sq += v[i] * v[i];
                const float inv = 1.0f / sqrtf(head_sum<L>(sq) * (1.0f / D) + A.eps);
                if (!BACK) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = v[i] * inv * gain[i];
                    if (turned) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float a = v[i], b = v[8 + i];
                            v[i] = a * c[i] - b * s[i];
                            v[8 + i] = a * s[i] + b * c[i];
                        }
                    }
                } else {
                    float d[16], dot = 0.0f;
                    norm_load<T, PAIRED>(dy + (unsigned)(r * ds + h * D), l, A.rot, d);
                    if (turned) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float a = d[i], b = d[8 + i];
                            d[i] = a * c[i] + b * s[i];
                            d[8 + i] = b * c[i] - a * s[i];
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        v[i] *= inv;
                        acc[w][i] += d[i] * v[i];
                        d[i] *= gain[i];
                        dot += d[i] * v[i];
                    }
                    dot = head_sum<L>(dot) * (1.0f / D);
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = inv * (d[i] - v[i] * dot);
                }
                norm_store<T, PAIRED>(y + (unsigned)(r * ys + h * D), l, A.rot, v);
            }
        }
    }
    if (BACK) {
        // The lanes with the same part of a head, in a fixed order: within the wave, then over the waves.
        constexpr int waves = kNormBlock / 64;
        float *sum = cs;  // [wave][2][D], in the order of the lanes' values
        static_assert(waves * 2 * D <= 2 * kNormAngles, "partial gains fit");
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float a = acc[w][i];
#pragma unroll
                for (int m = L; m < 64; m *= 2) a += __shfl_xor(a, m);
                if (tid % 64 < L) sum[(tid / 64 * 2 + w) * D + 16 * l + i] = a;
            }
        __syncthreads();
        for (int i = tid; i < 2 * D; i += kNormBlock) {
            float a = 0.0f;
            for (int w = 0; w < waves; ++w) a += sum[w * 2 * D + i];
            A.parts[(long long)blockIdx.x * 2 * D + i] = a;
        }
    }
}

// dgain from the workgroups' partial sums, always in the same order: a workgroup has 64 of their 2 D columns, its 16
// waves every 16th row.
template <int D, bool PAIRED>
__global__ __launch_bounds__(1024) void tf_qk_norm_gain_kernel(const float *__restrict__ parts, int n, int rot,
                                                                float *__restrict__ dq_gain, float *__restrict__ dk_gain) {
    __shared__ float sums[16][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, col = blockIdx.x * 64 + lane;
    float a = 0.0f;
#pragma unroll 16
    for (int p = wave; p < n; p += 16) a += parts[(long long)p * 2 * D + col];
    sums[wave][lane] = a;
    __syncthreads();
    if (wave == 0) {
        a = 0.0f;
        for (int w = 0; w < 16; ++w) a += sums[w][lane];
        const int i = col % D, l = i / 16, j = i % 16;  // lane l's j-th value: where norm_load took it from
        int at;
        if (PAIRED) at = 16 * l + 2 * (j % 8) + j / 8;
        else if (16 * l < rot) at = 8 * l + j % 8 + (j / 8) * (rot / 2);
        else at = 16 * l + j;
        (col / D ? dk_gain : dq_gain)[at] = a;
    }
}

// Rows of a tile: as many angles as the LDS array holds, fewer where that leaves compute units without a tile; and so
// that the tiles come out even for 1024 workgroups (the backward pass has no more; 1059 tiles took it twice 1024's time; 768 of
// them run at a time).
int norm_tile(const tf_qk_norm_config *c, int64_t n_rows) {
    const int64_t most = kNormAngles / (c->rotary_dim / 2);
    const int64_t rounds = (n_rows + 1024 * most - 1) / (1024 * most);
    const int64_t t = rounds ? (n_rows + 1024 * rounds - 1) / (1024 * rounds) : 1;
    return (int)(t < 1 ? 1 : t < most ? t : most);
}

tf_status norm_check(const tf_qk_norm_config *c, int64_t n_rows, int32_t n_seqs) {
    if (!c || n_rows < 0 || n_seqs < 0) return TF_EINVAL;
    if (!elem_ok(c->elem) || c->n_q_heads < 1 || c->n_k_heads < 1 || c->head_dim < 1 || c->rotary_dim < 1 ||
        c->rotary_dim > c->head_dim)
        return TF_EINVAL;
    if (c->clear < 0 || c->clear > 3 || !(c->eps >= 0.0f) || !(c->base > 0.0) || !std::isfinite(c->base) || !std::isfinite(c->eps)) return TF_EINVAL;
    const int d = c->head_dim;
    if ((d != 32 && d != 64 && d != 128 && d != 256) || c->rotary_dim % 16) return TF_EUNSUPPORTED;
    if (c->n_q_heads > 1024 || c->n_k_heads > 1024 || n_rows > INT32_MAX) return TF_EUNSUPPORTED;
    return TF_OK;
}

Turns norm_turns(const tf_qk_norm_config *c) {
    Turns t = {};
    for (int j = 0; j < c->rotary_dim / 2; ++j)
        t.f[j] = std::pow(c->base, -2.0 * j / c->rotary_dim) / (2.0 * 3.14159265358979323846);
    return t;
}

template <typename T, int D, bool BACK>
void norm_launch(const tf_qk_norm_config *c, const NormArgs &A, hipStream_t stream) {
    const Turns t = norm_turns(c);
    // (up to one workgroup a compute unit for the rows to clear)
    const int64_t clear = A.clear ? (A.n_rows + 63) / 64 : 0;
    const dim3 grid((unsigned)(A.blocks + (clear < 256 ? clear : 256)));
    if (c->interleaved)
        hipLaunchKernelGGL((tf_qk_norm_kernel<T, D, true, BACK>), grid, dim3(kNormBlock), 0, stream, A, t);
    else
        hipLaunchKernelGGL((tf_qk_norm_kernel<T, D, false, BACK>), grid, dim3(kNormBlock), 0, stream, A, t);
}
template <int D, bool BACK> void norm_elem(const tf_qk_norm_config *c, const NormArgs &A, hipStream_t stream) {
    if (c->elem == TF_ELEM_FP32) norm_launch<ElemF32, D, BACK>(c, A, stream);
    else if (c->elem == TF_ELEM_BF16) norm_launch<ElemBF16, D, BACK>(c, A, stream);
    else norm_launch<ElemF16, D, BACK>(c, A, stream);
}
template <bool BACK> void norm_width(const tf_qk_norm_config *c, const NormArgs &A, hipStream_t stream) {
    switch (c->head_dim) {
        case 32: norm_elem<32, BACK>(c, A, stream); break;
        case 64: norm_elem<64, BACK>(c, A, stream); break;
        case 128: norm_elem<128, BACK>(c, A, stream); break;
        default: norm_elem<256, BACK>(c, A, stream); break;
    }
}
template <int D> void gain_launch(const tf_qk_norm_config *c, const float *parts, int n, float *dq, float *dk, hipStream_t s) {
    if (c->interleaved)
        hipLaunchKernelGGL((tf_qk_norm_gain_kernel<D, true>), dim3(2 * D / 64), dim3(1024), 0, s, parts, n, (int)c->rotary_dim, dq, dk);
    else
        hipLaunchKernelGGL((tf_qk_norm_gain_kernel<D, false>), dim3(2 * D / 64), dim3(1024), 0, s, parts, n, (int)c->rotary_dim, dq, dk);
}

void norm_sizes(const tf_qk_norm_config *c, int64_t n_rows, NormArgs &A) {
    auto per = [](unsigned n) { return n == 1 ? 0xffffffffu : (unsigned)((1ull << 32) / n); };
    A.rot = c->rotary_dim, A.tile = norm_tile(c, n_rows), A.eps = c->eps, A.clear = A.offsets ? c->clear : 0;
    A.per_head[0] = per((unsigned)c->n_q_heads), A.per_head[1] = per((unsigned)c->n_k_heads), A.per_pair = per((unsigned)c->rotary_dim / 2);
}
constexpr int64_t kFarthest = 1 << 22;  // a tile's rows are addressed by 32-bit offsets

// An output that starts at its input but whose rows lie elsewhere.
bool in_place_elsewhere(const void *x, int64_t x_stride, const void *y, int64_t y_stride, int64_t n_rows) {
    return x == y && x_stride != y_stride && n_rows > 1;
}

int64_t norm_blocks(const tf_qk_norm_config *c, int64_t n_rows, int64_t most) {
    const int tile = norm_tile(c, n_rows);
    const int64_t tiles = (n_rows + tile - 1) / tile;
    return tiles < most ? tiles : most;
}

}  // namespace

extern "C" size_t tf_qk_norm_workspace_size(const tf_qk_norm_config *c, int64_t n_rows) {
    if (norm_check(c, n_rows, 0) != TF_OK) return 0;
    const int64_t b = norm_blocks(c, n_rows, kNormParts);
    return (size_t)(b < 1 ? 1 : b) * 2 * c->head_dim * sizeof(float);
}

extern "C" tf_status tf_qk_norm_rotate(const tf_qk_norm_config *c, const void *q, int64_t q_stride, const void *k,
                                       int64_t k_stride, int64_t n_rows, const float *q_gain, const float *k_gain,
                                       const int32_t *positions, const int32_t *offsets, int32_t n_seqs, void *q_out,
                                       int64_t q_out_stride, void *k_out, int64_t k_out_stride, hipStream_t stream) {
    const tf_status s = norm_check(c, n_rows, n_seqs);
    if (s != TF_OK) return s;
    const int64_t qw = (int64_t)c->n_q_heads * c->head_dim, kw = (int64_t)c->n_k_heads * c->head_dim;
    if (!stride_ok(q_stride, qw, c->elem) || !stride_ok(k_stride, kw, c->elem) || !stride_ok(q_out_stride, qw, c->elem) ||
        !stride_ok(k_out_stride, kw, c->elem))
        return TF_EINVAL;
    if (!strides_fit({q_stride, k_stride, q_out_stride, k_out_stride}, kFarthest)) return TF_EUNSUPPORTED;
    if (n_rows == 0) return TF_OK;
    if (!q || !k || !q_gain || !k_gain || !q_out || !k_out) return TF_EINVAL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(q_gain) || !aligned16(k_gain) || !aligned16(q_out) || !aligned16(k_out))
        return TF_EINVAL;
    if (in_place_elsewhere(q, q_stride, q_out, q_out_stride, n_rows) || in_place_elsewhere(k, k_stride, k_out, k_out_stride, n_rows) ||
        over_inputs({q_out}, {k, q_gain, k_gain}) || over_inputs({k_out}, {q, q_gain, k_gain}) || q_out == k_out)
        return TF_EINVAL;
    NormArgs A = {};
    A.x[0] = q, A.x[1] = k, A.y[0] = q_out, A.y[1] = k_out, A.gain[0] = q_gain, A.gain[1] = k_gain;
    A.xs[0] = q_stride, A.xs[1] = k_stride, A.ys[0] = q_out_stride, A.ys[1] = k_out_stride;
    A.heads[0] = c->n_q_heads, A.heads[1] = c->n_k_heads;
    A.n_rows = n_rows, A.positions = positions, A.offsets = offsets, A.n_seqs = n_seqs;
    norm_sizes(c, n_rows, A);
    A.blocks = (int)norm_blocks(c, n_rows, 1 << 20);
    norm_width<false>(c, A, stream);
    return hipGetLastError() == hipSuccess ? TF_OK : TF_EHIP;
}

extern "C" tf_status tf_qk_norm_rotate_backward(const tf_qk_norm_config *c, const void *dq_out, int64_t dq_out_stride,
                                                const void *dk_out, int64_t dk_out_stride, const void *q,
                                                int64_t q_stride, const void *k, int64_t k_stride, int64_t n_rows,
                                                const float *q_gain, const float *k_gain, const int32_t *positions,
                                                const int32_t *offsets, int32_t n_seqs, void *workspace,
                                                size_t workspace_bytes, void *dq, int64_t dq_stride, void *dk,
                                                int64_t dk_stride, float *dq_gain, float *dk_gain, hipStream_t stream) {
    const tf_status s = norm_check(c, n_rows, n_seqs);
    if (s != TF_OK) return s;
    const int64_t qw = (int64_t)c->n_q_heads * c->head_dim, kw = (int64_t)c->n_k_heads * c->head_dim;
    if (!stride_ok(q_stride, qw, c->elem) || !stride_ok(k_stride, kw, c->elem) || !stride_ok(dq_stride, qw, c->elem) ||
        !stride_ok(dk_stride, kw, c->elem) || !stride_ok(dq_out_stride, qw, c->elem) || !stride_ok(dk_out_stride, kw, c->elem))
        return TF_EINVAL;
    if (!strides_fit({q_stride, k_stride, dq_stride, dk_stride, dq_out_stride, dk_out_stride}, kFarthest)) return TF_EUNSUPPORTED;
    if (!q_gain || !k_gain || !dq_gain || !dk_gain || !workspace || !aligned16(q_gain) || !aligned16(k_gain)) return TF_EINVAL;
    if (workspace_bytes < tf_qk_norm_workspace_size(c, n_rows) || ((uintptr_t)workspace & 3)) return TF_EINVAL;
    if (twice({dq, dk, dq_gain, dk_gain, workspace}) || over_inputs({workspace, dq_gain, dk_gain}, {q_gain, k_gain})) return TF_EINVAL;
    if (n_rows > 0) {
        if (!q || !k || !dq_out || !dk_out || !dq || !dk) return TF_EINVAL;
        if (!aligned16(q) || !aligned16(k) || !aligned16(dq_out) || !aligned16(dk_out) || !aligned16(dq) || !aligned16(dk))
            return TF_EINVAL;
        if (in_place_elsewhere(dq_out, dq_out_stride, dq, dq_stride, n_rows) ||
            in_place_elsewhere(dk_out, dk_out_stride, dk, dk_stride, n_rows) || over_inputs({dq}, {dk_out, q, k, q_gain, k_gain}) ||
            over_inputs({dk}, {dq_out, q, k, q_gain, k_gain}) || over_inputs({workspace, dq_gain, dk_gain}, {dq_out, dk_out, q, k}))
            return TF_EINVAL;
    }
    NormArgs A = {};
    A.x[0] = q, A.x[1] = k, A.dy[0] = dq_out, A.dy[1] = dk_out, A.y[0] = dq, A.y[1] = dk;
    A.gain[0] = q_gain, A.gain[1] = k_gain;
    A.xs[0] = q_stride, A.xs[1] = k_stride, A.ds[0] = dq_out_stride, A.ds[1] = dk_out_stride;
    A.ys[0] = dq_stride, A.ys[1] = dk_stride;
    A.heads[0] = c->n_q_heads, A.heads[1] = c->n_k_heads;
    A.n_rows = n_rows, A.positions = positions, A.offsets = offsets, A.n_seqs = n_seqs;
    norm_sizes(c, n_rows, A);
    A.parts = (float *)workspace;
    int blocks = (int)norm_blocks(c, n_rows, kNormParts);
    if (blocks < 1) blocks = 1;  // no rows: the gradients of the gains are zeros
    A.blocks = blocks;
    norm_width<true>(c, A, stream);
    switch (c->head_dim) {
        case 32: gain_launch<32>(c, A.parts, blocks, dq_gain, dk_gain, stream); break;
        case 64: gain_launch<64>(c, A.parts, blocks, dq_gain, dk_gain, stream); break;
        case 128: gain_launch<128>(c, A.parts, blocks, dq_gain, dk_gain, stream); break;
        default: gain_launch<256>(c, A.parts, blocks, dq_gain, dk_gain, stream); break;
    }
    return hipGetLastError() == hipSuccess ? TF_OK : TF_EHIP;
}
