// Rows in 8-bit integers with a scale each, back to values, and the product of
// two matrices in that form.
//
// With s_m and t_n the scales of x's and w's rows:
//   y[m][n] = (float)(sum_k a[m][k] b[n][k]) s_m t_n + bias[n]
// The sum is a whole number below 2^31 for K < 2^17, so it is exact in any order.
#include <algorithm>
#include <type_traits>

#include "ops.hpp"

namespace agnes {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 16;                         // codes: rows are padded to whole chunks
static int64_t chunks_of(int64_t cols) { return (cols + kChunk - 1) / kChunk; }

// ----------------------------------------------------------------- elements

// A row's scale and what its codes are computed with: x and the scale times
// `up` (a power of two, so both stay exact), which keeps the reciprocal finite
// where the scale is no normal number.
struct Scale {
    float scale, up, by, inv;                      // by = scale * up
};
// top: the row's largest magnitude as bits (NaN above infinity above all finite values).
__device__ __forceinline__ Scale row_scale(uint32_t top) {
    Scale s;
    const bool bad = top >= 0x7F800000u;
    s.scale = bad ? __uint_as_float(0x7FC00000u) : __uint_as_float(top) * (1.f / 127.f);
    s.up = s.scale < 0x1p-100f ? 0x1p60f : 1.f;
    s.by = s.scale * s.up;
    s.inv = bad || s.by == 0.f ? 0.f : 1.f / s.by;
    return s;
}

// x / scale to the nearest whole number, ties to even.  The product with the
// reciprocal is off by less than 127 * 2^-22, so its nearest whole number q is the
// quotient's or a neighbour of it, and only where the quotient lies near a half.  The
// remainder x - q scale, a multiple of half an ulp of the scale below the
// scale, is exact in float32 and decides.
__device__ __forceinline__ int to_code(float x, const Scale& s) {
    const float v = x * s.up;
    float q = rintf(v * s.inv);
    const float r = fmaf(-q, s.by, v), over = fabsf(r) * 2.f - s.by;
    if (over > 0.f || (over == 0.f && ((int)q & 1))) q += copysignf(1.f, r);
    return (int)fminf(fmaxf(q, -127.f), 127.f);
}

// ----------------------------------------------------------------- quantisation

template <typename T>
__global__ __launch_bounds__(kBlock) void k_int8_quantize(const T* __restrict__ x, int64_t stride, int64_t cols,
                                                          int64_t pitch, int8_t* __restrict__ codes,
                                                          float* __restrict__ scales) {
    __shared__ uint32_t red[kWavesPerBlock];
    const int64_t r = blockIdx.x;
    const T* row = x + r * stride;
    uint32_t top = 0;
    for (int64_t c = threadIdx.x; c < cols; c += kBlock) top = max(top, __float_as_uint(to_float(row[c])) & 0x7FFFFFFFu);
    for (int d = 32; d; d /= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if (lane_id() == 0) red[wave_id()] = top;
    __syncthreads();
    for (int w = 0; w < kWavesPerBlock; w++) top = max(top, red[w]);
    const Scale s = row_scale(top);
    if (threadIdx.x == 0) scales[r] = s.scale;
    for (int64_t c = threadIdx.x; c < pitch; c += kBlock)
        codes[r * pitch + c] = c < cols && s.inv != 0.f ? (int8_t)to_code(to_float(row[c]), s) : (int8_t)0;
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_int8_dequantize(const int8_t* __restrict__ codes,
                                                            const float* __restrict__ scales, int64_t rows,
                                                            int64_t cols, int64_t pitch, T* __restrict__ x,
                                                            int64_t stride) {
    const int64_t step = (int64_t)gridDim.x * kBlock, n = rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += step) {
        const int64_t r = i / cols, c = i % cols;
        x[r * stride + c] = from_float<T>((float)codes[r * pitch + c] * scales[r]);
    }
}

// ----------------------------------------------------------------- product

struct Int8Args {
    const int8_t *xc, *wc;
    const float *xs, *ws;
    int64_t M, N;
    int32_t chunks;                                // per row
    const float* bias;
    bool relu;
    void* out;
    int64_t stride;
};

__device__ __forceinline__ float finish(int sum, float s, float t, float bias, bool relu) {
    const float y = (float)sum * s * t + bias;
    return relu && y < 0.f ? 0.f : y;
}

// v_mfma_i32_16x16x64_i8: lane l holds 16 consecutive k (one chunk) of row l %
// 16 of either operand, k = 16 (l / 16); D[4 (l / 16) + r][l % 16].  The
// weight goes in first, so a lane holds four adjacent columns of a row of out.
// A wave per 16 x 16 elements of out.
template <typename T> __global__ __launch_bounds__(kWave) void k_int8_wave(Int8Args a) {
    const int lane = lane_id();
    const int64_t tn = (a.N + 15) / 16;
    const int64_t m = (int64_t)blockIdx.x / tn * 16 + lane % 16, n0 = (int64_t)blockIdx.x % tn * 16, n = n0 + lane % 16;
    const int8_t* const xr = a.xc + min(m, a.M - 1) * a.chunks * kChunk;
    const int8_t* const wr = a.wc + min(n, a.N - 1) * a.chunks * kChunk;
    i32x4 acc = {0, 0, 0, 0};
    for (int c0 = 0; c0 < a.chunks; c0 += 4) {
        const int c = c0 + lane / 16;
        i32x4 x = {0, 0, 0, 0}, w = {0, 0, 0, 0};
        if (c < a.chunks) {
            x = *(const i32x4*)(xr + c * kChunk);
            w = *(const i32x4*)(wr + c * kChunk);
        }
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc, 0, 0, 0);
    }
    if (m >= a.M) return;
    for (int r = 0; r < 4; r++) {
        const int64_t c = n0 + lane / 16 * 4 + r;
        if (c < a.N)
            ((T*)a.out)[m * a.stride + c] =
                from_float<T>(finish(acc[r], a.xs[m], a.ws[c], a.bias ? a.bias[c] : 0.f, a.relu));
    }
}

// ----------------------------------------------------------------- host

static void check_int8(const agnes_int8* q, const char* name) {
    const std::string n(name);
    AGNES_REQUIRE(q, AGNES_ERR_INVALID, n + " must not be NULL");
    AGNES_REQUIRE(q->rows >= 0 && q->cols >= 0 && q->rows < ((int64_t)1 << 31) && q->cols < ((int64_t)1 << 31),
                  AGNES_ERR_INVALID, n + ": rows and cols must be in [0, 2^31)");
    if (q->rows == 0) return;
    AGNES_REQUIRE(q->scales && ((uintptr_t)q->scales & 3) == 0, AGNES_ERR_INVALID,
                  n + ": scales must not be NULL and must be aligned to their type");
    AGNES_REQUIRE(q->codes || q->cols == 0, AGNES_ERR_INVALID, n + ": codes must not be NULL");
    AGNES_REQUIRE(((uintptr_t)q->codes & 15) == 0, AGNES_ERR_INVALID, n + ": codes must be 16-byte aligned");
}

constexpr int64_t kLaunchRows = 1 << 21;           // rows per launch of a workgroup each: a launch holds fewer than 2^32 threads

void int8_quantize(const agnes_matrix* x, const agnes_int8* q, hipStream_t st) {
    check_matrix(x, false, "x");
    check_int8(q, "q");
    AGNES_REQUIRE(q->rows == x->rows && q->cols == x->cols, AGNES_ERR_INVALID, "x and q must have equal shapes");
    const int64_t pitch = chunks_of(x->cols) * kChunk;
    with_float(x->dtype, [&](auto t) {
        typedef decltype(t) T;
        for (int64_t r = 0; r < x->rows; r += kLaunchRows)
            AGNES_LAUNCH((k_int8_quantize<T>), dim3((unsigned)std::min(kLaunchRows, x->rows - r)), dim3(kBlock), 0, st,
                         (const T*)x->data + r * x->stride, x->stride, x->cols, pitch, q->codes + r * pitch, q->scales + r);
    });
}

void int8_dequantize(const agnes_int8* q, const agnes_matrix* x, hipStream_t st) {
    check_matrix(x, true, "x");
    check_int8(q, "q");
    AGNES_REQUIRE(q->rows == x->rows && q->cols == x->cols, AGNES_ERR_INVALID, "x and q must have equal shapes");
    if (x->rows == 0 || x->cols == 0) return;
    with_float(x->dtype, [&](auto t) {
        typedef decltype(t) T;
        AGNES_LAUNCH((k_int8_dequantize<T>), dim3(grid_for(x->rows * x->cols, 4096)), dim3(kBlock), 0, st, q->codes,
                     q->scales, x->rows, x->cols, chunks_of(x->cols) * kChunk, (T*)x->data, x->stride);
    });
}

static void check_sizes(int64_t M, int64_t N, int64_t K) {
    for (int64_t v : {M, N, K})
        AGNES_REQUIRE(v >= 0 && v < ((int64_t)1 << 31), AGNES_ERR_INVALID, "M, N and K must be in [0, 2^31)");
    // 2^14 K stays below 2^31, also for codes of -128
    AGNES_REQUIRE(K < ((int64_t)1 << 17), AGNES_ERR_INVALID, "K must be below 2^17");
}

uint64_t int8_product_bytes(int64_t M, int64_t N, int64_t K) {
    check_sizes(M, N, K);
    AGNES_REQUIRE(((M + 15) / 16) * ((N + 15) / 16) <= (1 << 23) - kXcds, AGNES_ERR_RANGE, "the product has too many tiles");
    return 0;
}

uint64_t int8_linear_bytes(int64_t M, int64_t N, int64_t K) {
    check_sizes(M, N, K);
    Carve c(nullptr);
    c.take<int8_t>(M * chunks_of(K) * kChunk);
    c.take<float>(M);
    return c.used + int8_product_bytes(M, N, K);
}

void int8_product(const agnes_int8* x, const agnes_int8* w, const float* bias, bool relu, const agnes_matrix* out,
                  void* ws, uint64_t ws_bytes, hipStream_t st) {
    check_int8(x, "x");
    check_int8(w, "w");
    check_matrix(out, true, "out");
    AGNES_REQUIRE(x->cols == w->cols, AGNES_ERR_INVALID, "x and w must have equal columns");
    AGNES_REQUIRE(out->rows == x->rows && out->cols == w->rows, AGNES_ERR_INVALID,
                  "out must have x's rows and one column per row of w");
    const int64_t M = x->rows, N = w->rows;
    check_workspace(ws, ws_bytes, int8_product_bytes(M, N, x->cols));   // checks the sizes too
    if (M == 0 || N == 0) return;
    const int64_t tiles = ((M + 15) / 16) * ((N + 15) / 16);
    const Int8Args a{x->codes, w->codes, x->scales, w->scales, M, N, (int32_t)chunks_of(x->cols), bias, relu, out->data,
                     out->stride};
    with_float(out->dtype, [&](auto t) {
        typedef decltype(t) T;
        AGNES_LAUNCH((k_int8_wave<T>), dim3((unsigned)tiles), dim3(kWave), 0, st, a);
    });
}

void int8_linear(const agnes_matrix* x, const agnes_int8* w, const float* bias, bool relu, const agnes_matrix* out,
                 void* ws, uint64_t ws_bytes, hipStream_t st) {
    check_matrix(x, false, "x");
    check_int8(w, "w");
    check_matrix(out, true, "out");
    AGNES_REQUIRE(x->cols == w->cols, AGNES_ERR_INVALID, "x and w must have equal columns");
    AGNES_REQUIRE(out->rows == x->rows && out->cols == w->rows, AGNES_ERR_INVALID,
                  "out must have x's rows and one column per row of w");
    check_workspace(ws, ws_bytes, int8_linear_bytes(x->rows, w->rows, x->cols));
    if (x->rows == 0 || w->rows == 0) return;
    Carve c(ws);
    agnes_int8 q{};
    q.rows = x->rows;
    q.cols = x->cols;
    q.codes = c.take<int8_t>(x->rows * chunks_of(x->cols) * kChunk);
    q.scales = c.take<float>(x->rows);
    int8_quantize(x, &q, st);
    int8_product(&q, w, bias, relu, out, (char*)ws + c.used, ws_bytes - c.used, st);
}

}  // namespace agnes
