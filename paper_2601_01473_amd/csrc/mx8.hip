// Microscaled 8-bit integers (MXINT8), in which a layer keeps its input until
// the backward pass: rows to codes with one power-of-two scale per block of 32
// elements, back to values, activations that keep their input, their backward
// pass, and a linear layer's weight gradient.
//
// A block's scale is 2^floor(log2 max|x|), a code counts 1/64 of it: a code and
// a power of two are exact in bfloat16, so the weight gradient's products are too.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ops.hpp"

namespace agnes {

constexpr int kMx8Block = 32;                      // elements per scale
static int64_t blocks_of(int64_t cols) { return (cols + kMx8Block - 1) / kMx8Block; }

// ----------------------------------------------------------------- elements

// The scale code of a block whose largest magnitude has the float32 bits `top`:
// their exponent (0 for subnormal numbers; 255 for infinities and NaN).
__device__ __forceinline__ int scale_code(uint32_t top) { return (int)(top >> 23); }

// x in units of 1/64 of the scale; the scaling is exact (or far below 1).
__device__ __forceinline__ int to_code(float x, int scale) {
    const float q = rintf(ldexpf(x, 133 - scale));
    return (int)fminf(fmaxf(q, -127.f), 127.f);
}
// The eight codes as bytes, the first in the low bits.
__device__ __forceinline__ uint2 to_codes(const float (&x)[8], int scale) {
    uint2 w = {0u, 0u};
    if (scale == 255) return w;
#pragma unroll
    for (int q = 0; q < 4; q++) {
        w.x |= (uint32_t)(to_code(x[q], scale) & 255) << (8 * q);
        w.y |= (uint32_t)(to_code(x[q + 4], scale) & 255) << (8 * q);
    }
    return w;
}

__device__ __forceinline__ float from_code(int8_t c, int scale) {
    return scale == 255 ? __uint_as_float(0x7FC00000u) : ldexpf((float)c, scale - 133);
}
__device__ __forceinline__ void from_codes(uint2 w, int scale, float (&x)[8]) {
#pragma unroll
    for (int q = 0; q < 4; q++) {
        x[q] = from_code((int8_t)(w.x >> (8 * q)), scale);
        x[q + 4] = from_code((int8_t)(w.y >> (8 * q)), scale);
    }
}

// The largest magnitude of the four lanes that hold a block.
__device__ __forceinline__ uint32_t block_top(const float (&x)[8]) {
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < 8; q++) top = max(top, __float_as_uint(x[q]) & 0x7FFFFFFFu);
    top = max(top, __float_as_uint(lane_pair<1>(__uint_as_float(top))));
    return max(top, __float_as_uint(lane_pair<2>(__uint_as_float(top))));
}

template <typename T> __device__ __forceinline__ void store8(T* row, int64_t c, int64_t cols, const float (&x)[8], bool nt) {
    if (c + 8 <= cols) {
        Vec<T, 8>::store(row + c, x, nt);
    } else {
#pragma unroll
        for (int q = 0; q < 8; q++)
            if (c + q < cols) row[c + q] = from_float<T>(x[q]);
    }
}

// ----------------------------------------------------------------- rows

// A piece is 8 elements, a block four pieces in adjacent lanes.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_mx8_quantize(const T* __restrict__ x, int64_t stride, int64_t pieces,
                                                         int64_t cols, uint32_t per_row, int8_t* __restrict__ codes,
                                                         uint8_t* __restrict__ scales) {
    const int64_t base = (int64_t)blockIdx.x * (kBlock * kPieces);
    const int64_t base_row = base / per_row;
    const uint32_t base_piece = (uint32_t)(base % per_row);
    float v[kPieces][8];
#pragma unroll
    for (int u = 0; u < kPieces; u++) {
        const uint32_t off = u * kBlock + threadIdx.x;
        if (base + off < pieces) {
            const PieceAt p = piece_at(base_row, base_piece, off, per_row);
            load8<T>(x + p.row * stride, (int64_t)p.piece * 8, cols, v[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < kPieces; u++) {
        const int64_t i = base + u * kBlock + threadIdx.x;
        if (i >= pieces) continue;                 // whole blocks: pieces is a multiple of 4
        const int scale = scale_code(block_top(v[u]));
        *(uint2*)(codes + 8 * i) = to_codes(v[u], scale);
        if (threadIdx.x % 4 == 0) scales[i / 4] = (uint8_t)scale;
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_mx8_dequantize(const int8_t* __restrict__ codes,
                                                           const uint8_t* __restrict__ scales, int64_t pieces,
                                                           int64_t cols, uint32_t per_row, T* __restrict__ x,
                                                           int64_t stride, bool nt) {
    const int64_t base = (int64_t)blockIdx.x * (kBlock * kPieces);
    const int64_t base_row = base / per_row;
    const uint32_t base_piece = (uint32_t)(base % per_row);
    uint2 w[kPieces];
    int s[kPieces];
#pragma unroll
    for (int u = 0; u < kPieces; u++) {
        const int64_t i = base + u * kBlock + threadIdx.x;
        if (i < pieces) {
            w[u] = *(const uint2*)(codes + 8 * i);
            s[u] = scales[i / 4];
        }
    }
#pragma unroll
    for (int u = 0; u < kPieces; u++) {
        const uint32_t off = u * kBlock + threadIdx.x;
        if (base + off >= pieces) continue;
        const PieceAt p = piece_at(base_row, base_piece, off, per_row);
        float v[8];
        from_codes(w[u], s[u], v);
        store8<T>(x + p.row * stride, (int64_t)p.piece * 8, cols, v, nt);
    }
}

// ----------------------------------------------------------------- activations

// act(x) and act'(x).
template <agnes_act ACT> __device__ __forceinline__ void activation(float x, float& value, float& slope) {
    if (ACT == AGNES_SILU) {
        const float e = expf(-x), p = 1.f / (1.f + e);
        value = x * p;
        const float rest = x < -40.f ? 1.f : e * p;             // 1 - p, without a difference
        slope = p * (1.f + x * rest);
    } else {
        const float phi = 0.5f * erfcf(x * -0.70710678118654752440f);
        value = x * phi;
        slope = phi + x * (0.39894228040143267794f * expf(-0.5f * x * x));
    }
}

template <typename T, typename TY, agnes_act ACT>
__global__ __launch_bounds__(kBlock) void k_mx8_act(const T* __restrict__ x, int64_t stride, int64_t rows, int64_t F,
                                                    bool gated, TY* __restrict__ y, int64_t ystride) {
    const int64_t step = (int64_t)gridDim.x * kBlock, n = rows * F;
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += step) {
        const int64_t r = i / F, c = i % F;
        float v, s;
        activation<ACT>(to_float(x[r * stride + c]), v, s);
        if (gated) v *= to_float(x[r * stride + F + c]);
        y[r * ystride + c] = from_float<TY>(v);
    }
}

template <typename TG, typename TX, agnes_act ACT>
__global__ __launch_bounds__(kBlock) void k_mx8_act_grad(const int8_t* __restrict__ codes,
                                                         const uint8_t* __restrict__ scales, int64_t blocks,
                                                         int64_t rows, int64_t F, bool gated, const TG* __restrict__ gy,
                                                         int64_t gystride, TX* __restrict__ gx, int64_t gxstride) {
    const int64_t step = (int64_t)gridDim.x * kBlock, n = rows * F;
    auto kept = [&](int64_t r, int64_t c) {
        return from_code(codes[r * blocks * kMx8Block + c], scales[r * blocks + c / kMx8Block]);
    };
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += step) {
        const int64_t r = i / F, c = i % F;
        const float g = to_float(gy[r * gystride + c]);
        float v, s;
        activation<ACT>(kept(r, c), v, s);
        if (gated) {
            gx[r * gxstride + c] = from_float<TX>(g * kept(r, F + c) * s);
            gx[r * gxstride + F + c] = from_float<TX>(g * v);
        } else {
            gx[r * gxstride + c] = from_float<TX>(g * s);
        }
    }
}

// ----------------------------------------------------------------- weight gradient

// A thread per element of grad_weight; the first column's threads also sum the bias gradient.
template <typename TG, typename TW>
__global__ __launch_bounds__(kBlock) void k_mx8_wgrad(const TG* __restrict__ g, int64_t gstride,
                                                      const int8_t* __restrict__ codes,
                                                      const uint8_t* __restrict__ scales, int64_t blocks, int64_t M,
                                                      int64_t N, int64_t K, bool accumulate, TW* __restrict__ dw,
                                                      int64_t wstride, float* __restrict__ db) {
    const int64_t step = (int64_t)gridDim.x * kBlock, total = N * K;
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < total; i += step) {
        const int64_t n = i / K, k = i % K;
        float sum = 0.f;
        for (int64_t m = 0; m < M; m++)
            sum = fmaf(to_float(g[m * gstride + n]),
                       from_code(codes[m * blocks * kMx8Block + k], scales[m * blocks + k / kMx8Block]), sum);
        TW* const at = dw + n * wstride + k;
        *at = from_float<TW>(accumulate ? to_float(*at) + sum : sum);
    }
    if (!db) return;
    for (int64_t n = (int64_t)blockIdx.x * kBlock + threadIdx.x; n < N; n += step) {
        float sum = 0.f;
        for (int64_t m = 0; m < M; m++) sum += to_float(g[m * gstride + n]);
        db[n] = accumulate ? db[n] + sum : sum;
    }
}

// ----------------------------------------------------------------- host

static void check_mx8(const agnes_mx8* q, const char* name) {
    const std::string n(name);
    AGNES_REQUIRE(q, AGNES_ERR_INVALID, n + " must not be NULL");
    AGNES_REQUIRE(q->rows >= 0 && q->cols >= 0 && q->rows < ((int64_t)1 << 31) && q->cols < ((int64_t)1 << 31),
                  AGNES_ERR_INVALID, n + ": rows and cols must be in [0, 2^31)");
    if (q->rows == 0 || q->cols == 0) return;
    AGNES_REQUIRE(q->codes && q->scales, AGNES_ERR_INVALID, n + ": codes and scales must not be NULL");
    AGNES_REQUIRE(((uintptr_t)q->codes & 15) == 0, AGNES_ERR_INVALID, n + ": codes must be 16-byte aligned");
}

void mx8_quantize(const agnes_matrix* x, const agnes_mx8* q, hipStream_t st) {
    check_matrix(x, false, "x");
    check_mx8(q, "q");
    AGNES_REQUIRE(q->rows == x->rows && q->cols == x->cols, AGNES_ERR_INVALID, "x and q must have equal shapes");
    const int64_t blocks = blocks_of(x->cols), per_row = blocks * 4;
    if (x->rows == 0 || per_row == 0) return;
    with_float(x->dtype, [&](auto t) {
        typedef decltype(t) T;
        launch_pieces(x->rows, per_row, [&](int64_t r, int64_t pieces, unsigned groups) {
            AGNES_LAUNCH((k_mx8_quantize<T>), dim3(groups), dim3(kBlock), 0, st, (const T*)x->data + r * x->stride,
                         x->stride, pieces, x->cols, (uint32_t)per_row, q->codes + r * blocks * kMx8Block,
                         q->scales + r * blocks);
        });
    });
}

void mx8_dequantize(const agnes_mx8* q, const agnes_matrix* x, hipStream_t st) {
    check_matrix(x, true, "x");
    check_mx8(q, "q");
    AGNES_REQUIRE(q->rows == x->rows && q->cols == x->cols, AGNES_ERR_INVALID, "x and q must have equal shapes");
    const int64_t blocks = blocks_of(x->cols), per_row = blocks * 4;
    if (x->rows == 0 || per_row == 0) return;
    with_float(x->dtype, [&](auto t) {
        typedef decltype(t) T;
        launch_pieces(x->rows, per_row, [&](int64_t r, int64_t pieces, unsigned groups) {
            AGNES_LAUNCH((k_mx8_dequantize<T>), dim3(groups), dim3(kBlock), 0, st, q->codes + r * blocks * kMx8Block,
                         q->scales + r * blocks, pieces, x->cols, (uint32_t)per_row, (T*)x->data + r * x->stride,
                         x->stride, x->rows * x->cols * (int64_t)sizeof(T) > kStreamBytes);
        });
    });
}

template <typename F> static void with_act(agnes_act act, F&& f) {
    if (act == AGNES_SILU) f(std::integral_constant<agnes_act, AGNES_SILU>{});
    else f(std::integral_constant<agnes_act, AGNES_GELU>{});
}
static void check_act(agnes_act act) {
    AGNES_REQUIRE(act == AGNES_SILU || act == AGNES_GELU, AGNES_ERR_INVALID, "the activation must be AGNES_SILU or AGNES_GELU");
}

void mx8_activation(const agnes_matrix* x, agnes_act act, bool gated, const agnes_matrix* y, const agnes_mx8* kept,
                    hipStream_t st) {
    check_matrix(x, false, "x");
    check_matrix(y, true, "y");
    check_act(act);
    AGNES_REQUIRE(y->rows == x->rows && x->cols == (gated ? 2 : 1) * y->cols, AGNES_ERR_INVALID,
                  gated ? "y must have x's rows and half its columns" : "y must have x's shape");
    if (kept) mx8_quantize(x, kept, st);
    if (y->rows == 0 || y->cols == 0) return;
    with_float(x->dtype, [&](auto t) {
        with_float(y->dtype, [&](auto ty) {
            with_act(act, [&](auto a) {
                AGNES_LAUNCH((k_mx8_act<decltype(t), decltype(ty), decltype(a)::value>),
                             dim3(grid_for(y->rows * y->cols, 4096)), dim3(kBlock), 0, st, (const decltype(t)*)x->data,
                             x->stride, y->rows, y->cols, gated, (decltype(ty)*)y->data, y->stride);
            });
        });
    });
}

void mx8_activation_grad(const agnes_mx8* kept, agnes_act act, bool gated, const agnes_matrix* grad_y,
                         const agnes_matrix* grad_x, hipStream_t st) {
    check_mx8(kept, "kept");
    check_matrix(grad_y, false, "grad_y");
    check_matrix(grad_x, true, "grad_x");
    check_act(act);
    AGNES_REQUIRE(grad_x->rows == kept->rows && grad_x->cols == kept->cols, AGNES_ERR_INVALID,
                  "grad_x must have the kept rows' shape");
    AGNES_REQUIRE(grad_y->rows == kept->rows && kept->cols == (gated ? 2 : 1) * grad_y->cols, AGNES_ERR_INVALID,
                  gated ? "grad_y must have the kept rows and half their columns" : "grad_y must have the kept rows' shape");
    if (grad_y->rows == 0 || grad_y->cols == 0) return;
    with_float(grad_y->dtype, [&](auto tg) {
        with_float(grad_x->dtype, [&](auto tx) {
            with_act(act, [&](auto a) {
                AGNES_LAUNCH((k_mx8_act_grad<decltype(tg), decltype(tx), decltype(a)::value>),
                             dim3(grid_for(grad_y->rows * grad_y->cols, 4096)), dim3(kBlock), 0, st, kept->codes,
                             kept->scales, blocks_of(kept->cols), grad_y->rows, grad_y->cols, gated,
                             (const decltype(tg)*)grad_y->data, grad_y->stride, (decltype(tx)*)grad_x->data,
                             grad_x->stride);
            });
        });
    });
}

uint64_t mx8_weight_grad_bytes(int64_t M, int64_t N, int64_t K) {
    for (int64_t v : {M, N, K})
        AGNES_REQUIRE(v >= 0 && v < ((int64_t)1 << 31), AGNES_ERR_INVALID, "M, N and K must be in [0, 2^31)");
    return 0;
}

void mx8_weight_grad(const agnes_matrix* grad_out, const agnes_mx8* kept, bool accumulate,
                     const agnes_matrix* grad_weight, float* grad_bias, void* ws, uint64_t ws_bytes, hipStream_t st) {
    check_matrix(grad_out, false, "grad_out");
    check_mx8(kept, "kept");
    check_matrix(grad_weight, true, "grad_weight");
    AGNES_REQUIRE(grad_out->rows == kept->rows, AGNES_ERR_INVALID, "grad_out and kept must have equal rows");
    AGNES_REQUIRE(grad_weight->rows == grad_out->cols && grad_weight->cols == kept->cols, AGNES_ERR_INVALID,
                  "grad_weight must have a row per column of grad_out and the kept rows' columns");
    const int64_t M = kept->rows, N = grad_out->cols, K = kept->cols;
    check_workspace(ws, ws_bytes, mx8_weight_grad_bytes(M, N, K));
    if (N == 0) return;
    with_float(grad_out->dtype, [&](auto tg) {
        with_float(grad_weight->dtype, [&](auto tw) {
            AGNES_LAUNCH((k_mx8_wgrad<decltype(tg), decltype(tw)>), dim3(grid_for(std::max<int64_t>(N * K, N), 4096)),
                         dim3(kBlock), 0, st, (const decltype(tg)*)grad_out->data, grad_out->stride, kept->codes,
                         kept->scales, blocks_of(K), M, N, K, accumulate, (decltype(tw)*)grad_weight->data,
                         grad_weight->stride, grad_bias);
        });
    });
}

}  // namespace agnes
