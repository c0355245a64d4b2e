// Microscaled 4-bit floating point (MXFP4): rows to 4-bit codes with one
// power-of-two scale per block of 32 elements, back to values, and the product
// of two matrices in that form.
//
// A block's scale is 2^(floor(log2 max|x|) - 2): the largest element lands in
// [4, 8), and 2^2 is the largest power of two that the 4-bit format holds.
#include <algorithm>

#include "ops.hpp"

namespace agnes {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kMxBlock = 32;                       // elements per scale
static int64_t mx_blocks(int64_t cols) { return (cols + kMxBlock - 1) / kMxBlock; }

// The 4-bit code of y: nearest magnitude of {0, 0.5, 1, 1.5, 2, 3, 4, 6}, ties to the even code.
__device__ __forceinline__ uint32_t e2m1(float y) {
    const float a = fabsf(y);
    const uint32_t c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.f);
    return c | (y < 0.f ? 8u : 0u);
}

// 2^e for e in [-127, 127] (2^-127 is a subnormal).
__device__ __forceinline__ float exp2_int(int e) {
    return __uint_as_float(e >= -126 ? (uint32_t)(e + 127) << 23 : 1u << 22);
}

// One thread per block of 32.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_mx4_quantize(const T* __restrict__ x, int64_t stride, int64_t rows,
                                                         int64_t cols, int64_t blocks, uint8_t* __restrict__ codes,
                                                         uint8_t* __restrict__ scales) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i >= rows * blocks) return;
    const int64_t r = i / blocks, b = i % blocks;
    float v[kMxBlock];
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < kMxBlock; q++) {
        const int64_t c = b * kMxBlock + q;
        v[q] = c < cols ? to_float(x[r * stride + c]) : 0.f;
        top = max(top, __float_as_uint(v[q]) & 0x7FFFFFFFu);
    }
    const int e = (int)(top >> 23);
    const int code = e == 255 ? 255 : max(e - 2, 0);
    const float inv = code == 255 ? 0.f : exp2_int(127 - code);
    uint32_t out[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int q = 0; q < kMxBlock; q++) out[q / 8] |= (code == 255 ? 0u : e2m1(v[q] * inv)) << (4 * (q % 8));
    scales[i] = (uint8_t)code;
    *(uint4*)(codes + 16 * i) = uint4{out[0], out[1], out[2], out[3]};
}

__device__ __forceinline__ float e2m1_value(uint32_t c) {
    const float mag = (c & 6u) ? __uint_as_float((((c >> 1) & 3u) + 126u) << 23 | (c & 1u) << 22) : 0.5f * (float)(c & 1u);
    return (c & 8u) ? -mag : mag;
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_mx4_dequantize(const uint8_t* __restrict__ codes,
                                                           const uint8_t* __restrict__ scales, int64_t rows,
                                                           int64_t cols, int64_t blocks, T* __restrict__ x,
                                                           int64_t stride) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i >= rows * blocks) return;
    const int64_t r = i / blocks, b = i % blocks;
    const int code = scales[i];
    const float s = code == 255 ? __uint_as_float(0x7FC00000u) : exp2_int(code - 127);
    const uint4 w = *(const uint4*)(codes + 16 * i);
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int q = 0; q < kMxBlock; q++) {
        const int64_t c = b * kMxBlock + q;
        if (c < cols) x[r * stride + c] = from_float<T>(s * e2m1_value((ws[q / 8] >> (4 * (q % 8))) & 15u));
    }
}

// ----------------------------------------------------------------- product

// One wave per 16 x 16 tile of out, K in steps of 128.  v_mfma_scale_f32_16x16x128
// with 4-bit operands: lane l holds 32 consecutive k (one block) of row l % 16
// of either operand, k = 32 (l / 16), and that block's scale; D[4 (l / 16) + r][l % 16].
template <typename T>
__global__ __launch_bounds__(kBlock) void k_mx4_product(const uint8_t* __restrict__ xc, const uint8_t* __restrict__ xs,
                                                        const uint8_t* __restrict__ wc, const uint8_t* __restrict__ ws,
                                                        int64_t M, int64_t N, int64_t blocks,
                                                        const float* __restrict__ bias, bool relu,
                                                        T* __restrict__ out, int64_t stride) {
    const int lane = lane_id();
    const int64_t tiles_n = (N + 15) / 16, tile = (int64_t)blockIdx.x * kWavesPerBlock + wave_id();
    const int64_t m0 = tile / tiles_n * 16, n0 = tile % tiles_n * 16;
    if (m0 >= M) return;
    const int64_t m = m0 + (lane & 15), n = n0 + (lane & 15);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int64_t b0 = 0; b0 < blocks; b0 += 4) {
        const int64_t b = b0 + (lane >> 4);
        i32x4 a = {0, 0, 0, 0}, w = {0, 0, 0, 0};
        int sa = 127, sw = 127;
        if (b < blocks && m < M) {
            a = *(const i32x4*)(xc + 16 * (m * blocks + b));
            sa = xs[m * blocks + b];
        }
        if (b < blocks && n < N) {
            w = *(const i32x4*)(wc + 16 * (n * blocks + b));
            sw = ws[n * blocks + b];
        }
        const i32x8 a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, w8 = {w[0], w[1], w[2], w[3], 0, 0, 0, 0};
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, w8, acc, 4, 4, 0, sa, 0, sw);
    }
    if (n >= N) return;
    const float bn = bias ? bias[n] : 0.f;
#pragma unroll
    for (int r = 0; r < 4; r++) {
        const int64_t row = m0 + 4 * (lane >> 4) + r;
        if (row >= M) continue;
        float y = acc[r] + bn;
        if (relu) y = y < 0.f ? 0.f : y;
        out[row * stride + n] = from_float<T>(y);
    }
}

// ----------------------------------------------------------------- host

static void check_mx4(const agnes_mx4* q, const char* name) {
    const std::string n(name);
    AGNES_REQUIRE(q, AGNES_ERR_INVALID, n + " must not be NULL");
    AGNES_REQUIRE(q->rows >= 0 && q->cols >= 0 && q->rows < ((int64_t)1 << 31) && q->cols < ((int64_t)1 << 31),
                  AGNES_ERR_INVALID, n + ": rows and cols must be in [0, 2^31)");
    if (q->rows == 0 || q->cols == 0) return;
    AGNES_REQUIRE(q->codes && q->scales, AGNES_ERR_INVALID, n + ": codes and scales must not be NULL");
    AGNES_REQUIRE(((uintptr_t)q->codes & 15) == 0, AGNES_ERR_INVALID, n + ": codes must be 16-byte aligned");
}

static unsigned grid_of(int64_t n, int64_t per) {
    const int64_t g = (n + per - 1) / per;
    AGNES_REQUIRE(g < ((int64_t)1 << 31), AGNES_ERR_RANGE, "the matrix is too large");
    return (unsigned)g;
}

void mx4_quantize(const agnes_matrix* x, const agnes_mx4* q, hipStream_t st) {
    check_matrix(x, false, "x");
    check_mx4(q, "q");
    AGNES_REQUIRE(q->rows == x->rows && q->cols == x->cols, AGNES_ERR_INVALID, "x and q must have equal shapes");
    const int64_t blocks = mx_blocks(x->cols), n = x->rows * blocks;
    if (n == 0) return;
    with_float(x->dtype, [&](auto t) {
        typedef decltype(t) T;
        AGNES_LAUNCH((k_mx4_quantize<T>), dim3(grid_of(n, kBlock)), dim3(kBlock), 0, st, (const T*)x->data, x->stride,
                     x->rows, x->cols, blocks, q->codes, q->scales);
    });
}

void mx4_dequantize(const agnes_mx4* q, const agnes_matrix* x, hipStream_t st) {
    check_matrix(x, true, "x");
    check_mx4(q, "q");
    AGNES_REQUIRE(q->rows == x->rows && q->cols == x->cols, AGNES_ERR_INVALID, "x and q must have equal shapes");
    const int64_t blocks = mx_blocks(x->cols), n = x->rows * blocks;
    if (n == 0) return;
    with_float(x->dtype, [&](auto t) {
        typedef decltype(t) T;
        AGNES_LAUNCH((k_mx4_dequantize<T>), dim3(grid_of(n, kBlock)), dim3(kBlock), 0, st, q->codes, q->scales,
                     x->rows, x->cols, blocks, (T*)x->data, x->stride);
    });
}

static void check_sizes(int64_t M, int64_t N, int64_t K) {
    for (int64_t v : {M, N, K})
        AGNES_REQUIRE(v >= 0 && v < ((int64_t)1 << 31), AGNES_ERR_INVALID, "M, N and K must be in [0, 2^31)");
}

uint64_t mx4_product_bytes(int64_t M, int64_t N, int64_t K) {
    check_sizes(M, N, K);
    return 0;
}

uint64_t mx4_linear_bytes(int64_t M, int64_t N, int64_t K) {
    check_sizes(M, N, K);
    Carve c(nullptr);
    c.take<uint8_t>(M * mx_blocks(K) * 16);
    c.take<uint8_t>(M * mx_blocks(K));
    return c.used + mx4_product_bytes(M, N, K);
}

void mx4_product(const agnes_mx4* x, const agnes_mx4* w, const float* bias, bool relu, const agnes_matrix* out,
                 void* ws, uint64_t ws_bytes, hipStream_t st) {
    check_mx4(x, "x");
    check_mx4(w, "w");
    check_matrix(out, true, "out");
    AGNES_REQUIRE(x->cols == w->cols, AGNES_ERR_INVALID, "x and w must have equal columns");
    AGNES_REQUIRE(out->rows == x->rows && out->cols == w->rows, AGNES_ERR_INVALID,
                  "out must have x's rows and one column per row of w");
    const int64_t M = x->rows, N = w->rows, blocks = mx_blocks(x->cols);
    check_workspace(ws, ws_bytes, mx4_product_bytes(M, N, x->cols));
    if (M == 0 || N == 0) return;
    const int64_t tiles = ((M + 15) / 16) * ((N + 15) / 16);
    with_float(out->dtype, [&](auto t) {
        typedef decltype(t) T;
        AGNES_LAUNCH((k_mx4_product<T>), dim3(grid_of(tiles, kWavesPerBlock)), dim3(kBlock), 0, st, x->codes,
                     x->scales, w->codes, w->scales, M, N, blocks, bias, relu, (T*)out->data, out->stride);
    });
}

void mx4_linear(const agnes_matrix* x, const agnes_mx4* w, const float* bias, bool relu, const agnes_matrix* out,
                void* ws, uint64_t ws_bytes, hipStream_t st) {
    check_matrix(x, false, "x");
    check_mx4(w, "w");
    check_matrix(out, true, "out");
    AGNES_REQUIRE(x->cols == w->cols, AGNES_ERR_INVALID, "x and w must have equal columns");
    AGNES_REQUIRE(out->rows == x->rows && out->cols == w->rows, AGNES_ERR_INVALID,
                  "out must have x's rows and one column per row of w");
    check_workspace(ws, ws_bytes, mx4_linear_bytes(x->rows, w->rows, x->cols));
    if (x->rows == 0 || w->rows == 0) return;
    Carve c(ws);
    agnes_mx4 q{};
    q.rows = x->rows;
    q.cols = x->cols;
    q.codes = c.take<uint8_t>(x->rows * mx_blocks(x->cols) * 16);
    q.scales = c.take<uint8_t>(x->rows * mx_blocks(x->cols));
    mx4_quantize(x, &q, st);
    mx4_product(&q, w, bias, relu, out, (char*)ws + c.used, ws_bytes - c.used, st);
}

}  // namespace agnes
