// Building blocks of the sequence-layer operators (qknorm.hip, decay.hip,
// gated.hip): the tensors' element types, their vector loads and stores, and
// the sequence of a packed row.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <initializer_list>

#include "trackfit.h"

namespace {

typedef __attribute__((ext_vector_type(2))) float o_f32x2;
typedef __attribute__((ext_vector_type(4))) unsigned int o_u32x4;
typedef __attribute__((ext_vector_type(4))) float o_f32x4;
typedef __attribute__((ext_vector_type(8))) float o_f32x8;

// 8 consecutive elements as one or two 16-byte accesses; E is the element
// type, V8 a vector of 8 of them.
struct ElemF32 {
    typedef float E;
    typedef o_f32x8 V8;
};
struct ElemBF16 {
    typedef __bf16 E;
    typedef __attribute__((ext_vector_type(8))) __bf16 V8;
};
struct ElemF16 {
    typedef _Float16 E;
    typedef __attribute__((ext_vector_type(8))) _Float16 V8;
};

template <typename T> __device__ __forceinline__ o_f32x8 load8(const typename T::E *p) {
    return __builtin_convertvector(*(const typename T::V8 *)p, o_f32x8);
}
// Round to nearest even to the element type: the one rounding of an output.
template <typename T> __device__ __forceinline__ void store8(typename T::E *p, o_f32x8 v) {
    *(typename T::V8 *)p = __builtin_convertvector(v, typename T::V8);
}

// The sequence that packed row r belongs to: the last i < n with offsets[i] <= r (so that
// empty sequences own no row), or -1 when there is none or r is at or past its end.
// Any offsets: the search stays inside [0, n].
__device__ __forceinline__ int seq_of_row(const int32_t *__restrict__ offsets, int n, long long r) {
    int lo = 0, hi = n;  // offsets[lo - 1] <= r < offsets[hi], where these exist
    while (lo < hi) {
        const int mid = lo + ((hi - lo) >> 1);
        if (offsets[mid] <= r) lo = mid + 1;
        else hi = mid;
    }
    if (lo == 0 || r >= offsets[lo]) return -1;  // lo <= n: offsets has n + 1 entries
    return lo - 1;
}

// Steps in order, step(i, fragment i), with the fragments of the next DEPTH - 1 steps on their way.  The fences keep that
// order: left to itself the compiler reads a fragment, waits for it and only then multiplies, an LDS latency a step.
template <int N, int DEPTH, class Load, class Step> __device__ __forceinline__ void in_turn(Load load, Step step) {
    decltype(load(0)) w[DEPTH];
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i)
        if (i < N) w[i] = load(i);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i + DEPTH - 1 < N) w[(i + DEPTH - 1) % DEPTH] = load(i + DEPTH - 1);
        __builtin_amdgcn_sched_barrier(0);
        step(i, w[i % DEPTH]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
inline size_t elem_bytes(int e) { return e == TF_ELEM_FP32 ? 4 : 2; }
inline bool elem_ok(int e) { return e == TF_ELEM_FP32 || e == TF_ELEM_BF16 || e == TF_ELEM_FP16; }
// A row stride in elements that keeps 16-byte accesses of an aligned array aligned.
inline bool stride_ok(int64_t stride, int64_t width, int e) {
    return stride >= width && (stride * (int64_t)elem_bytes(e)) % 16 == 0;
}

// Whether no row stride is over what 32-bit offsets reach.
inline bool strides_fit(std::initializer_list<int64_t> strides, int64_t most) {
    for (int64_t s : strides)
        if (s > most) return false;
    return true;
}

// Whether an output is one of the inputs: workgroups would read what others have written.
inline bool over_inputs(std::initializer_list<const void *> outputs, std::initializer_list<const void *> inputs) {
    for (const void *o : outputs)
        for (const void *i : inputs)
            if (o && o == i) return true;
    return false;
}

// Whether two outputs (the workspace is one) are the same.
inline bool twice(std::initializer_list<const void *> outputs) {
    for (auto o = outputs.begin(); o != outputs.end(); ++o)
        for (auto p = outputs.begin(); p != o; ++p)
            if (*o && *o == *p) return true;
    return false;
}

}  // namespace
