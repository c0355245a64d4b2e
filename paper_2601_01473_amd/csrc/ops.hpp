// What the operator kernels (embed.hip, distill.hip, mx4.hip, policy.hip,
// int8.hip, mx8.hip) share: element types, vector accesses at element alignment, argument checks and the host
// entry points that api.hip wraps.
#pragma once

#include <algorithm>

#include "device.hpp"
#include "runtime.hpp"

namespace agnes {

// ----------------------------------------------------------------- elements

// float, _Float16 and __bf16 convert to and from float with single
// instructions; conversions to 16 bits round to nearest, ties to even, and keep
// NaN and infinities.
template <typename T> __device__ __forceinline__ float to_float(T x) { return (float)x; }
template <typename T> __device__ __forceinline__ T from_float(float x) { return (T)x; }

// E consecutive elements, loaded or stored at element alignment: rows of any
// length and stride start anywhere, and the memory system takes wide accesses
// at any address.
template <typename T, int E> struct Vec {
    typedef T type __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    static __device__ __forceinline__ type raw(const T* p) { return *(const type*)p; }
    static __device__ __forceinline__ void load(const T* p, float (&x)[E]) {
        const type v = *(const type*)p;
#pragma unroll
        for (int q = 0; q < E; q++) x[q] = (float)v[q];
    }
    // nt: past the caches, for a result larger than they are
    static __device__ __forceinline__ void store(T* p, const float (&x)[E], bool nt = false) {
        type v;
#pragma unroll
        for (int q = 0; q < E; q++) v[q] = (T)x[q];
        if (nt) __builtin_nontemporal_store(v, (type*)p);
        else *(type*)p = v;
    }
};

// ----------------------------------------------------------------- reductions over lanes

// x of the lane that this one pairs with in step D = 1, 2, .. 32 of a butterfly,
// without a trip through LDS.  Steps 4 and 8 mirror 8 and 16 lanes: once the
// steps before have been taken, all lanes of a half hold the same value.
template <int D> __device__ __forceinline__ float lane_pair(float x) {
    const int v = __float_as_int(x);
    if (D == 1) return __int_as_float(__builtin_amdgcn_update_dpp(v, v, 0xB1, 0xF, 0xF, false));    // quad_perm 1 0 3 2
    if (D == 2) return __int_as_float(__builtin_amdgcn_update_dpp(v, v, 0x4E, 0xF, 0xF, false));    // quad_perm 2 3 0 1
    if (D == 4) return __int_as_float(__builtin_amdgcn_update_dpp(v, v, 0x141, 0xF, 0xF, false));   // row_half_mirror
    return __int_as_float(__builtin_amdgcn_update_dpp(v, v, 0x140, 0xF, 0xF, false));               // row_mirror
}

// Lanes [g L, (g + 1) L) of a wave (L a power of two) reduce among themselves.
template <typename Op> __device__ __forceinline__ float lanes_reduce(float x, int L, Op op) {
    if (L > 1) x = op(x, lane_pair<1>(x));
    if (L > 2) x = op(x, lane_pair<2>(x));
    if (L > 4) x = op(x, lane_pair<4>(x));
    if (L > 8) x = op(x, lane_pair<8>(x));
    if (L > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if (L > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return x;
}
__device__ __forceinline__ float lanes_max(float x, int L) {
    return lanes_reduce(x, L, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float lanes_sum(float x, int L) {
    return lanes_reduce(x, L, [](float a, float b) { return a + b; });
}

// Orders the lanes' LDS accesses within their wave.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ----------------------------------------------------------------- pieces of rows

// Eight elements from column c of a row on, zeros behind its end.
template <typename T> __device__ __forceinline__ void load8(const T* row, int64_t c, int64_t cols, float (&x)[8]) {
    if (c + 8 <= cols) {
        Vec<T, 8>::load(row + c, x);
    } else {
#pragma unroll
        for (int q = 0; q < 8; q++) x[q] = c + q < cols ? to_float(row[c + q]) : 0.f;
    }
}

// The largest magnitude as bits: NaN above infinity above all finite values.
__device__ __forceinline__ uint32_t top_bits(const float (&x)[8]) {
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < 8; q++) top = max(top, __float_as_uint(x[q]) & 0x7FFFFFFFu);
    return top;
}

// Pieces of 8 elements are numbered row after row; a workgroup takes kPieces
// rounds of kBlock of them.
constexpr int kPieces = 4;

struct PieceAt {
    int64_t row;
    int32_t piece;
};
// Piece i of rows of `per_row` pieces; base: the workgroup's first piece.
__device__ __forceinline__ PieceAt piece_at(int64_t base_row, uint32_t base_piece, uint32_t off, uint32_t per_row) {
    const uint32_t x = base_piece + off;           // both below 2^30
    return {base_row + x / per_row, (int32_t)(x % per_row)};
}

// ----------------------------------------------------------------- tiles

// f(Const<0>{}), f(Const<1>{}), ..: indices that are constants.
template <auto N> struct Const { static constexpr auto value = N; };
template <int N, int I = 0, typename F> __device__ __forceinline__ void static_for(F&& f) {
    if constexpr (I < N) {
        f(Const<I>{});
        static_for<N, I + 1>(f);
    }
}

constexpr int kVmcnt0 = 0x0F70;                    // s_waitcnt vmcnt(0) and nothing else

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;

// ----------------------------------------------------------------- host side

inline size_t elem_size(agnes_dtype t) { return t == AGNES_FLOAT32 ? 4 : 2; }
inline bool is_float(agnes_dtype t) { return t == AGNES_FLOAT32 || t == AGNES_FLOAT16 || t == AGNES_BFLOAT16; }
inline bool is_index(agnes_dtype t) { return t == AGNES_INT32 || t == AGNES_INT64; }

// Results above this size leave the caches before anyone reads them: they are
// written with non-temporal stores, which leave the caches to what is read
// (lookup of 500000 rows of 512 bytes: 4.3 -> 5.3 TB/s).
constexpr int64_t kStreamBytes = (int64_t)64 << 20;

// Calls f with a value of the element type.
template <typename F> void with_float(agnes_dtype t, F&& f) {
    if (t == AGNES_FLOAT32) f(float{});
    else if (t == AGNES_FLOAT16) f(_Float16{});
    else f(__bf16{});
}
template <typename F> void with_index(agnes_dtype t, F&& f) {
    if (t == AGNES_INT64) f(int64_t{});
    else f(int32_t{});
}

// Calls launch(first row, pieces, workgroups) for parts of `rows` rows of
// per_row <= 2^28 pieces, each of at most kLaunchGroups workgroups, which take U
// rounds of kBlock pieces: a launch holds fewer than 2^32 threads.
constexpr int64_t kLaunchGroups = 1 << 22;
template <int U = kPieces, typename F> void launch_pieces(int64_t rows, int64_t per_row, F&& launch) {
    constexpr int64_t kGroup = kBlock * U;
    const int64_t most = kLaunchGroups * kGroup / per_row;
    for (int64_t r = 0; r < rows; r += most) {
        const int64_t n = std::min(most, rows - r), pieces = n * per_row;
        launch(r, pieces, (unsigned)((pieces + kGroup - 1) / kGroup));
    }
}

void check_matrix(const agnes_matrix* m, bool output, const char* name);
void check_workspace(const void* ws, uint64_t have, uint64_t need);

// Parts of a caller's workspace, each aligned to 256 bytes.
struct Carve {
    char* base;
    size_t used = 0;
    explicit Carve(void* p) : base((char*)p) {}
    template <typename T> T* take(int64_t n) {
        T* p = (T*)((uintptr_t)base + used);     // base NULL: sizes alone
        used += ((size_t)n * sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

// ----------------------------------------------------------------- entry points

void embedding_lookup(const agnes_matrix* table, const void* ids, agnes_dtype ids_dtype, float scale,
                      const agnes_matrix* out, hipStream_t st);
uint64_t embedding_grad_bytes(int64_t n, int64_t num_rows, int64_t dim);
void embedding_grad(const agnes_matrix* grad_out, const void* ids, agnes_dtype ids_dtype, float scale,
                    bool accumulate, const agnes_matrix* grad_table, void* ws, uint64_t ws_bytes, hipStream_t st);
void embedding_grad_rows(const agnes_matrix* grad_out, const void* ids, agnes_dtype ids_dtype, float scale,
                         int64_t num_rows, int32_t* row_ids, const agnes_matrix* rows, int64_t* count, void* ws,
                         uint64_t ws_bytes, hipStream_t st);
void batch_embedding_lookup(Batch& b, const agnes_matrix* table, float scale, const agnes_matrix* out,
                            hipStream_t st);
void batch_embedding_grad_rows(Batch& b, const agnes_matrix* grad_out, float scale, int32_t* row_ids,
                               const agnes_matrix* rows, int64_t* count, void* ws, uint64_t ws_bytes, hipStream_t st);

uint64_t distill_bytes(int64_t rows, int64_t classes);
void distill_loss(const agnes_distill* d, float* loss, float* stats, const agnes_matrix* grad, void* ws,
                  uint64_t ws_bytes, hipStream_t st);
void distill_grad(const agnes_distill* d, const float* stats, const agnes_matrix* grad, hipStream_t st);

void mx4_quantize(const agnes_matrix* x, const agnes_mx4* q, hipStream_t st);
void mx4_dequantize(const agnes_mx4* q, const agnes_matrix* x, hipStream_t st);
uint64_t mx4_product_bytes(int64_t M, int64_t N, int64_t K);
void mx4_product(const agnes_mx4* x, const agnes_mx4* w, const float* bias, bool relu, const agnes_matrix* out,
                 void* ws, uint64_t ws_bytes, hipStream_t st);
uint64_t mx4_linear_bytes(int64_t M, int64_t N, int64_t K);
void mx4_linear(const agnes_matrix* x, const agnes_mx4* w, const float* bias, bool relu, const agnes_matrix* out,
                void* ws, uint64_t ws_bytes, hipStream_t st);

uint64_t policy_bytes(int64_t rows, int64_t classes);
void policy_logprob(const agnes_policy* p, float* logp, void* ws, uint64_t ws_bytes, hipStream_t st);
void policy_loss(const agnes_policy* p, float* loss, float* logp, float* stats, const agnes_matrix* grad, void* ws,
                 uint64_t ws_bytes, hipStream_t st);
void policy_grad(const agnes_policy* p, const float* stats, const agnes_matrix* grad, hipStream_t st);

void int8_quantize(const agnes_matrix* x, const agnes_int8* q, hipStream_t st);
void int8_dequantize(const agnes_int8* q, const agnes_matrix* x, hipStream_t st);
uint64_t int8_product_bytes(int64_t M, int64_t N, int64_t K);
void int8_product(const agnes_int8* x, const agnes_int8* w, const float* bias, bool relu, const agnes_matrix* out,
                  void* ws, uint64_t ws_bytes, hipStream_t st);
uint64_t int8_linear_bytes(int64_t M, int64_t N, int64_t K);
void int8_linear(const agnes_matrix* x, const agnes_int8* w, const float* bias, bool relu, const agnes_matrix* out,
                 void* ws, uint64_t ws_bytes, hipStream_t st);

void mx8_quantize(const agnes_matrix* x, const agnes_mx8* q, hipStream_t st);
void mx8_dequantize(const agnes_mx8* q, const agnes_matrix* x, hipStream_t st);
void mx8_activation(const agnes_matrix* x, agnes_act act, bool gated, const agnes_matrix* y, const agnes_mx8* kept,
                    hipStream_t st);
void mx8_activation_grad(const agnes_mx8* kept, agnes_act act, bool gated, const agnes_matrix* grad_y,
                         const agnes_matrix* grad_x, hipStream_t st);
uint64_t mx8_weight_grad_bytes(const agnes_matrix* grad_out, int64_t K);
void mx8_weight_grad(const agnes_matrix* grad_out, const agnes_mx8* kept, bool accumulate,
                     const agnes_matrix* grad_weight, float* grad_bias, void* ws, uint64_t ws_bytes, hipStream_t st);

}  // namespace agnes
