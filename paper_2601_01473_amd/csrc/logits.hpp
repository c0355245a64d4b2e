// What the kernels that read rows of logits share (distill.hip, policy.hip).
#pragma once

#include "ops.hpp"

namespace agnes {

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float load_any(const void* p, agnes_dtype t, int64_t i) {
    if (t == AGNES_FLOAT32) return ((const float*)p)[i];
    if (t == AGNES_FLOAT16) return (float)((const _Float16*)p)[i];
    return (float)((const __bf16*)p)[i];
}
__device__ __forceinline__ void store_any(void* p, agnes_dtype t, int64_t i, float x) {
    if (t == AGNES_FLOAT32) ((float*)p)[i] = x;
    else if (t == AGNES_FLOAT16) ((_Float16*)p)[i] = (_Float16)x;
    else ((__bf16*)p)[i] = (__bf16)x;
}
__device__ __forceinline__ int64_t load_index(const void* p, bool wide, int64_t i) {
    return wide ? ((const int64_t*)p)[i] : (int64_t)((const int32_t*)p)[i];
}

// Pieces count from the row's first logit wherever that lies, so that equal rows
// have equal sums at any address.  (8192 rows of 50021 bfloat16, which start
// anywhere: 358 us; with pieces at multiples of 16 bytes of memory 309 us, but
// sums that depend on the address.)
template <int E, typename T>
__device__ __forceinline__ void store_typed(T* p, int c, int hi, const float (&x)[E], bool nt) {
    if (c + E <= hi) {
        Vec<T, E>::store(p + c, x, nt);
    } else {
#pragma unroll
        for (int q = 0; q < E; q++)
            if (c + q < hi) p[c + q] = (T)x[q];
    }
}

// A row's piece from column c on, -inf from column hi on.
template <typename T, int E>
__device__ __forceinline__ typename Vec<T, E>::type logits_piece(const T* row, int c, int hi) {
    if (c + E <= hi) return Vec<T, E>::raw(row + c);
    typename Vec<T, E>::type v;
#pragma unroll
    for (int q = 0; q < E; q++) v[q] = c + q < hi ? row[c + q] : (T)-INFINITY;
    return v;
}

// 2^x with results below 2^-126 as 0.
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }

// Makes the compiler take the piece from its packed registers again: it would
// otherwise keep the logits' float32 values from the maximum to the gradient,
// twice the registers, and spill.
template <typename Raw> __device__ __forceinline__ void keep_packed(Raw& v) {
    uint4 w;
    static_assert(sizeof(Raw) == sizeof(w), "a 16-byte piece");
    __builtin_memcpy(&w, &v, 16);
    asm volatile("" : "+v"(w.x), "+v"(w.y), "+v"(w.z), "+v"(w.w));
    __builtin_memcpy(&v, &w, 16);
}

}  // namespace agnes
