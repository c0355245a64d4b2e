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
__device__ __forceinline__ int mx8_scale(uint32_t top) { return (int)(top >> 23); }

// x in units of 1/64 of the scale; the scaling is exact (or far below 1).
__device__ __forceinline__ int to_code(float x, int scale) {
    const float q = rintf(ldexpf(x, 133 - scale));
    return (int)fminf(fmaxf(q, -127.f), 127.f);
}
// The eight codes as bytes, the first in the low bits.
__device__ __forceinline__ uint2 mx8_codes(const float (&x)[8], int scale) {
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
    uint32_t top = top_bits(x);
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

// A piece is 8 elements, a block four pieces in adjacent lanes.  Bound by memory:
// 16384 x 16384 bfloat16 148 us (5.5 TB/s), and back 140 us (5.8 TB/s).
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
        const int scale = mx8_scale(block_top(v[u]));
        *(uint2*)(codes + 8 * i) = mx8_codes(v[u], scale);
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

// exp(x), exp(x + low) for x in [-180, 0], in all their digits: 2^n 2^f with |f| <=
// 1/2, whose factor log2 e is held in two parts.  (2 to the rounded product x log2 e would be
// off by |x| 2^-24, and 0 below 2^-126.)
constexpr float kLog2e = 1.44269504088896340736f, kLog2eLow = 1.92596299112661746810e-8f;
__device__ __forceinline__ float exp_below(float x) {
    const float n = rintf(x * kLog2e);
    return ldexpf(__builtin_amdgcn_exp2f(fmaf(x, kLog2eLow, fmaf(x, kLog2e, -n))), (int)n);
}
__device__ __forceinline__ float exp_below(float x, float low) {
    const float n = rintf(x * kLog2e);
    return ldexpf(__builtin_amdgcn_exp2f(fmaf(low, kLog2e, fmaf(x, kLog2eLow, fmaf(x, kLog2e, -n)))), (int)n);
}
// x's magnitude, at most `most`; 0 for NaN.
__device__ __forceinline__ float magnitude(float x, float most) { return __builtin_amdgcn_fmed3f(fabsf(x), 0.f, most); }

// act(x) and act'(x) without a difference of near numbers but the slopes' own.
//
// SiLU: with u = exp(-|x|), which does not overflow, the logistic function is p = 1 /
// (1 + u) at |x| and u p at -|x|.
// GELU: with e = exp(-x^2 / 2), Phi(-|x|) = e R(|x|); R falls from 1/2 like 0.4 / |x|, and is
// t P(t) with t = 1 / (1 + c |x|).  P was fitted here to erfc's definition for |x| <= 14.5
// (behind it e is 0), by weighted least squares until the largest error was least.
// The density is 0.3989 e, so the pair costs one exponential and one reciprocal.
//
// FULL, for float32 results: within 2^-20 of the value, or of the slope's two
// terms.  2.5 u (u = 2^-24) come from the exponential, 3 u from the reciprocal of a
// rounded sum, which moves R by 2.3 times as much, 3 u from P (degree 8: 3.2e-8),
// 3 u from products; measured 5.6 u at most.
// Else, for results that are rounded to 16 bits, half of whose step is 2^-12 or
// more: within 2^-16, with P of degree 6 (2.9e-6 of R, 4.1e-8 of 1) and exponents
// rounded once (x^2 / 2 or |x| up to 88: 6e-6); silu below -87 and gelu below -13,
// all under 2^-119, are 0.  (16384 x 8192 bfloat16, forward and backward: gated silu
// 220 and 202 us, with FULL 239 and 219; gelu 150 and 144 us, with FULL 173 and 165.)
template <agnes_act ACT, bool FULL> __device__ __forceinline__ void activation(float x, float& value, float& slope) {
    if constexpr (ACT == AGNES_SILU && FULL) {
        const float u = exp_below(-magnitude(x, 120.f)), p = __builtin_amdgcn_rcpf(1.f + u), up = u * p;
        value = x * (x < 0.f ? up : p);
        slope = (x < 0.f ? up : p) * fmaf(x, x < 0.f ? p : up, 1.f);
    } else if constexpr (ACT == AGNES_SILU) {
        const float e = __builtin_amdgcn_exp2f(x * -kLog2e), p = __builtin_amdgcn_rcpf(1.f + e);
        value = x * p;
        slope = p * fmaf(x, x < -40.f ? 1.f : e * p, 1.f);
    } else {
        float e, r;
        if constexpr (FULL) {
            const float a = magnitude(x, 16.f), h = a * a, t = __builtin_amdgcn_rcpf(fmaf(a, 0.35f, 1.f));
            e = exp_below(-0.5f * h, -0.5f * fmaf(a, a, -h));
            r = fmaf(-0.029157886f, t, 0.14403091f);
            r = fmaf(r, t, -0.25583899f);
            r = fmaf(r, t, 0.1593197f);
            r = fmaf(r, t, -0.02321235f);
            r = fmaf(r, t, 0.1055525f);
            r = fmaf(r, t, 0.11982129f);
            r = fmaf(r, t, 0.13986352f);
            r = fmaf(r, t, 0.1396213f) * t;
        } else {
            const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(x), 0.26f, 1.f));
            e = __builtin_amdgcn_exp2f(x * x * (-0.5f * kLog2e));
            r = fmaf(-0.072636306f, t, 0.22740768f);
            r = fmaf(r, t, -0.10354217f);
            r = fmaf(r, t, 0.16375984f);
            r = fmaf(r, t, 0.07458535f);
            r = fmaf(r, t, 0.106882535f);
            r = fmaf(r, t, 0.10354302f) * t;
        }
        const float tail = e * r, s = e * fmaf(fabsf(x), -0.39894228040143267794f, r);
        value = x * (x < 0.f ? tail : 1.f - tail);
        slope = x < 0.f ? s : 1.f - s;
    }
}

// Forward: a piece is 8 columns of y; x's blocks are four adjacent lanes, in
// either half of a gated row too if the halves are whole blocks.  KEEP: 8-bit
// codes of x as well.  Bound by memory: gated silu of 16384 x 8192 bfloat16 196 to 220
// us (4.9 to 5.5 TB/s); with halves that meet inside a block (8200 columns) 305 us.
template <typename T, typename TY, agnes_act ACT, bool GATED, bool KEEP>
__global__ __launch_bounds__(kBlock) void k_mx8_act(const T* __restrict__ x, int64_t stride, int64_t pieces, int64_t F,
                                                    uint32_t per_row, int8_t* __restrict__ codes,
                                                    uint8_t* __restrict__ scales, int64_t blocks, TY* __restrict__ y,
                                                    int64_t ystride, bool nt) {
    constexpr int HALVES = GATED ? 2 : 1, U = kPieces / HALVES;
    const int64_t base = (int64_t)blockIdx.x * (kBlock * U);
    const int64_t base_row = base / per_row;
    const uint32_t base_piece = (uint32_t)(base % per_row);
    float v[U][HALVES][8];
#pragma unroll
    for (int u = 0; u < U; u++) {
        const uint32_t off = u * kBlock + threadIdx.x;
        if (base + off < pieces) {
            const PieceAt p = piece_at(base_row, base_piece, off, per_row);
#pragma unroll
            for (int h = 0; h < HALVES; h++) load8<T>(x + p.row * stride + h * F, (int64_t)p.piece * 8, F, v[u][h]);
        }
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
        const uint32_t off = u * kBlock + threadIdx.x;
        if (base + off >= pieces) continue;        // whole blocks: with KEEP pieces is a multiple of 4
        const PieceAt p = piece_at(base_row, base_piece, off, per_row);
        const int64_t c = (int64_t)p.piece * 8;
        if constexpr (KEEP) {
#pragma unroll
            for (int h = 0; h < HALVES; h++) {
                const int scale = mx8_scale(block_top(v[u][h]));
                const int64_t at = p.row * blocks * kMx8Block + h * F + c;
                *(uint2*)(codes + at) = mx8_codes(v[u][h], scale);
                if (threadIdx.x % 4 == 0) scales[at / kMx8Block] = (uint8_t)scale;
            }
        }
        float o[8];
#pragma unroll
        for (int q = 0; q < 8; q++) {
            float slope;
            activation<ACT, sizeof(TY) == 4>(v[u][0][q], o[q], slope);
            if constexpr (GATED) o[q] *= v[u][1][q];
        }
        store8<TY>(y + p.row * ystride, c, F, o, nt);
    }
}

// Eight kept values from column c of a row on, in whatever blocks they lie; zeros from column `cols` on.
__device__ __forceinline__ void load_kept(const int8_t* codes, const uint8_t* scales, int64_t c, int64_t cols, float (&x)[8]) {
    typedef uint2 __attribute__((aligned(1))) u64_bytes;
    uint2 w = {0u, 0u};
    if (c + 8 <= cols) {
        w = *(const u64_bytes*)(codes + c);
    } else {
        for (int q = 0; q < 8 && c + q < cols; q++) {
            const uint32_t b = (uint32_t)(uint8_t)codes[c + q] << (q % 4 * 8);
            if (q < 4) w.x |= b;
            else w.y |= b;
        }
    }
    const int64_t first = c / kMx8Block, last = min(c + 7, cols - 1) / kMx8Block;
    const int lo = scales[first], hi = scales[last], turn = (int)((first + 1) * kMx8Block - c);
#pragma unroll
    for (int q = 0; q < 8; q++) x[q] = from_code((int8_t)((q < 4 ? w.x : w.y) >> (q % 4 * 8)), q < turn ? lo : hi);
}

// Backward: a piece is 8 columns of grad_y.  WHOLE: the halves of a gated row are
// whole blocks.  The same case: 188 to 202 us (5.4 to 5.7 TB/s), of 8200 columns 216 us.
template <typename TG, typename TX, agnes_act ACT, bool GATED, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_mx8_act_grad(const int8_t* __restrict__ codes,
                                                         const uint8_t* __restrict__ scales, int64_t blocks,
                                                         int64_t pieces, int64_t F, uint32_t per_row,
                                                         const TG* __restrict__ gy, int64_t gystride, TX* __restrict__ gx,
                                                         int64_t gxstride, bool nt) {
    constexpr int HALVES = GATED ? 2 : 1, U = kPieces / HALVES;
    const int64_t base = (int64_t)blockIdx.x * (kBlock * U);
    const int64_t base_row = base / per_row;
    const uint32_t base_piece = (uint32_t)(base % per_row);
    uint2 w[U][HALVES];
    int s[U][HALVES];
    float g[U][8];
#pragma unroll
    for (int u = 0; u < U; u++) {
        const uint32_t off = u * kBlock + threadIdx.x;
        if (base + off < pieces) {
            const PieceAt p = piece_at(base_row, base_piece, off, per_row);
            const int64_t at = p.row * blocks * kMx8Block + (int64_t)p.piece * 8;
#pragma unroll
            for (int h = 0; h < (WHOLE ? HALVES : 1); h++) {
                w[u][h] = *(const uint2*)(codes + at + h * F);
                s[u][h] = scales[(at + h * F) / kMx8Block];
            }
            load8<TG>(gy + p.row * gystride, (int64_t)p.piece * 8, F, g[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
        const uint32_t off = u * kBlock + threadIdx.x;
        if (base + off >= pieces) continue;
        const PieceAt p = piece_at(base_row, base_piece, off, per_row);
        const int64_t c = (int64_t)p.piece * 8;
        float a[8], b[8], o[8];
        from_codes(w[u][0], s[u][0], a);
        if constexpr (GATED) {
            if constexpr (WHOLE) from_codes(w[u][HALVES - 1], s[u][HALVES - 1], b);
            else load_kept(codes + p.row * blocks * kMx8Block, scales + p.row * blocks, F + c, 2 * F, b);
        }
        TX* const row = gx + p.row * gxstride;
#pragma unroll
        for (int q = 0; q < 8; q++) {
            float value, slope;
            activation<ACT, sizeof(TX) == 4>(a[q], value, slope);
            o[q] = GATED ? g[u][q] * b[q] * slope : g[u][q] * slope;
            b[q] = g[u][q] * value;
        }
        store8<TX>(row, c, F, o, nt);
        if constexpr (GATED) store8<TX>(row + F, c, F, b, nt);
    }
}

// ----------------------------------------------------------------- weight gradient

// out[n][k] = sum over rows m of g[m][n] x[m][k]: both operands have m as their
// slow axis, and the multiplication wants 8 consecutive m per lane.  Both lie in
// LDS as they lie in memory, row m after row, as bfloat16, and are read with
// ds_read_tr16_b64, which transposes: of 16 lanes, lane i names 4 columns (8
// bytes) of row i / 4, and receives column i of the four rows.
//
// v_mfma_f32_16x16x32_bf16: lane l holds 8 m of row l % 16 of either operand;
// D[4 (l / 16) + r][l % 16].  x goes in first, so a lane holds four adjacent
// columns of a row of out.
//
// A float16 or float32 gradient is cut into 2 or 3 bfloat16 that add up to it,
// planes of LDS that all meet the same x.
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct WgradArgs {
    const void* g;
    int64_t gstride, gplane;                       // elements between rows, and between the planes of a cut gradient
    const int8_t* codes;
    const uint8_t* scales;
    int64_t M, N, K, blocks;                       // blocks per kept row
    void* out;
    int64_t stride;
    bool accumulate, nt;
    float* parts;                                  // [gridDim.y][N][K]: sums over parts of the rows instead of out, or NULL
    const float* bias_sums;                        // [bias_parts][N], for the join
    int bias_parts;
    float* db;
};

// Rows of a matrix that are read a step (32 rows) at a time, as buffers: reads
// behind a buffer bring zeros, so that rows behind the last one need no branch.
// All of it is scalar.  Offsets stay below 2^31: kMaxPitch.
typedef __amdgpu_buffer_rsrc_t Buffer;
constexpr uint32_t kNowhere = 0x80000000u;         // an offset behind every such buffer
constexpr int64_t kMaxPitch = (int64_t)1 << 25;    // bytes
// Values that are the same in all lanes, in scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
    return (uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x);
}
struct Rows {
    uint64_t at;                                   // the next step's first row, at the tile's first column
    int left, pitch, skip;                         // rows from there on; bytes of a row, and before the tile's first column
    __device__ __forceinline__ Rows(const void* p, int64_t rows, int64_t row_bytes, int64_t before)
        : at(uniform((uint64_t)p)), left(uniform((int)rows)), pitch(uniform((int)row_bytes)), skip(uniform((int)before)) {}
    __device__ __forceinline__ Buffer buffer(int row, uint64_t offset = 0) const {     // from that row of the step on
        int n = max(left - row, 0);
        asm("" : "+s"(n));                         // the two bounds would become one vector instruction
        const int bytes = max(min(n, 32) * pitch - skip, 0);
        return __builtin_amdgcn_make_buffer_rsrc((void*)(at + offset + (uint64_t)row * (uint32_t)pitch), 0, bytes, 0x00020000);
    }
    __device__ __forceinline__ void advance() {
        at += 32 * (uint64_t)(uint32_t)pitch;
        left -= 32;
    }
};

constexpr int kStepRows = 32, kImages = 3;         // rows m of a step; steps in LDS

// An image: kStepRows rows of WIDTH bfloat16, in blocks of 1024 bytes (what a wave
// fetches at once) with PAD bytes between them; chunk c (32 bytes) of row m of
// its block at place c ^ key(m).  A wave reads one chunk of eight consecutive rows at
// once: they lie in different banks (no conflict is counted).  Fewer key bits than an
// unpadded image would need leave fewer addresses for a lane to hold.  The stores
// of converted codes, 16 bytes a lane at places 32 bytes apart, meet in pairs: 8 of
// their 16 cycles each, 66 of the 72 thousand cycles of conflicts that 16384 x 4096 x
// 4096 bfloat16 counts among 339 thousand of LDS.
template <int WIDTH> struct Image {
    static constexpr int ROW = WIDTH * 2, BLOCK_ROWS = 1024 / ROW, PAD = WIDTH == 256 ? 64 : WIDTH == 128 ? 128 : 0;
    static constexpr int BLOCK = 1024 + PAD, BYTES = kStepRows / BLOCK_ROWS * BLOCK, KEYS = WIDTH == 256 ? 2 : 4;
    static __device__ __forceinline__ int key(int m) { return WIDTH == 64 ? m / 2 % 4 : m % KEYS; }
    static __device__ __forceinline__ int row(int m) { return m / BLOCK_ROWS * BLOCK + m % BLOCK_ROWS * ROW; }
};

// Two floats to bfloat16, which both are exactly.
__device__ __forceinline__ uint32_t pack_exact(float a, float b) {
    return __float_as_uint(a) >> 16 | (__float_as_uint(b) & 0xFFFF0000u);
}

// x as P bfloat16 that add up to it: its bits cut into eights.  Infinities and NaN are
// whole in the first.  What a float32 has below 2^-133, the smallest bfloat16, is left
// out: nothing from 2^-110 on up.  (The parts are summed in one accumulator and
// meet the same x, so none of them can be scaled up by itself.)
template <int P> __device__ __forceinline__ void cut(float x, float (&part)[P]) {
    const uint32_t b = __float_as_uint(x);
    const bool finite = (b & 0x7F800000u) != 0x7F800000u;
    part[0] = __uint_as_float(finite || (b & 0x007FFFFFu) == 0 ? b & 0xFFFF0000u : 0x7FC00000u);
    float rest = finite ? x - part[0] : 0.f;
#pragma unroll
    for (int p = 1; p < P; p++) {
        part[p] = __uint_as_float(__float_as_uint(rest) & 0xFFFF0000u);
        rest -= part[p];
    }
}

template <typename TG> constexpr int kParts = sizeof(TG) == 4 ? 3 : std::is_same<TG, _Float16>::value ? 2 : 1;

// Eight gradients, as loaded.
template <typename TG> struct Eight {
    typename Vec<TG, 8>::type v;
};

// A workgroup of WM x WN waves computes a tile of out, a wave 16 F rows (n) and
// 16 G columns (k) of it, in steps of 32 m.  DIRECT: P planes of bfloat16 whose rows are
// whole 16-byte pieces go from memory straight to LDS, three steps ahead; else
// gradients of type TG pass through registers and are cut there.  The kept codes
// pass through registers too, a step ahead of being converted and three of
// their use.  A wave reads a step's operands into registers while it multiplies
// the step before.
//
// 16384 x 4096 x 4096 bfloat16 in tiles of 256: 490 to 502 us (1.1 PFLOP/s), the matrix
// cores busy half of the cycles; LDS, which delivers the operands in pieces of 8 bytes and takes
// the converted codes, is busy a third, so waits for each step's barrier and first
// operands are what is left.  On the way: scalar buffer descriptors in place of
// addresses per lane 1047 -> 896 us, one set of x operands in place of two 663, sums in
// accumulation registers 580, no spilled registers 500.
template <typename TG, int P, typename TW, bool DIRECT, int WM, int WN, int F, int G>
__global__ __launch_bounds__(kWave* WM* WN) void k_mx8_wgrad(WgradArgs a) {
    constexpr int THREADS = kWave * WM * WN, ROWS = WM * 16 * F, COLS = WN * 16 * G;
    typedef Image<ROWS> GI;
    typedef Image<COLS> XI;
    static_assert(DIRECT ? std::is_same<TG, __bf16>::value : P == kParts<TG>, "");
    // An object per image and operand, addressed with constants: that way the
    // compiler sees that a fetch under way does not write what is being read.
    __shared__ __attribute__((aligned(1024))) char g0[P * GI::BYTES], g1[P * GI::BYTES], g2[P * GI::BYTES];
    __shared__ __attribute__((aligned(1024))) char x0[XI::BYTES], x1[XI::BYTES], x2[XI::BYTES];
    const int t = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), wm = wave / WN, wn = wave % WN;
    // XCD x takes a contiguous run of tiles, in strips of 8 tile rows.
    const int64_t tm = (a.N + ROWS - 1) / ROWS, tn = (a.K + COLS - 1) / COLS, tiles = tm * tn;
    const int64_t per = (tiles + kXcds - 1) / kXcds, id = blockIdx.x % kXcds * per + blockIdx.x / kXcds;
    if ((int64_t)blockIdx.x / kXcds >= per || id >= tiles) return;
    const int64_t strip = id / (8 * tn), high = min((int64_t)8, tm - strip * 8), in = id - strip * 8 * tn;
    const int64_t n0 = (strip * 8 + in % high) * ROWS, k0 = in / high * COLS;

    f32x4 acc[F][G];
#pragma unroll
    for (int i = 0; i < F; i++)
#pragma unroll
        for (int j = 0; j < G; j++) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    // This part's steps; fetches behind its end bring zeros, so that every step has equally many.
    const int all = (int)((a.M + kStepRows - 1) / kStepRows), share = (all + gridDim.y - 1) / gridDim.y;
    const int first = min(all, share * (int)blockIdx.y), steps = min(all, first + share) - first;
    const int64_t row0 = (int64_t)first * kStepRows;
    const int rows = (int)(min(a.M, row0 + (int64_t)steps * kStepRows) - row0);                   // of this part
    auto gat = [&](auto s) -> char* { constexpr int S = decltype(s)::value % kImages; return S == 0 ? g0 : S == 1 ? g1 : g2; };
    auto xat = [&](auto s) -> char* { constexpr int S = decltype(s)::value % kImages; return S == 0 ? x0 : S == 1 ? x1 : x2; };

    // The gradient: pieces of 8 elements, THREADS per round.
    constexpr int GPIECES = ROWS / 8, GROUNDS = kStepRows * GPIECES / THREADS, GSTEP = THREADS / GPIECES;   // rows per round
    static_assert(GROUNDS >= 1 && GSTEP % GI::BLOCK_ROWS == 0, "rounds have the same places");
    const int grow = t / GPIECES;
    const int gpiece = DIRECT ? t % GPIECES ^ GI::key(grow) << 1 : t % GPIECES;       // by place in LDS, or by place in memory
    const int64_t gn = n0 + gpiece * 8;
    const TG* const gfrom = (const TG*)a.g + row0 * a.gstride + n0;
    const uint32_t gplace = DIRECT && gn < a.N ? (grow * (uint32_t)a.gstride + gpiece * 8) * 2 : kNowhere;
    Rows grows(gfrom, rows, DIRECT ? a.gstride * 2 : 0, 0);
    auto fetch_g = [&](auto image, auto round) {                                      // DIRECT; the last round advances
        constexpr int Q = decltype(round)::value / GROUNDS, I = decltype(round)::value % GROUNDS;
        const Buffer b = grows.buffer(I * GSTEP, Q * (uint64_t)a.gplane * 2);
        if constexpr (decltype(round)::value == P * GROUNDS - 1) grows.advance();
        char* const to = gat(image) + wave * GI::BLOCK;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (lds_void*)(to + Q * GI::BYTES + I * (THREADS / kWave) * GI::BLOCK), 16, gplace, 0, 0, 0);
    };
    // Through registers: whole pieces; the one that a row's end cuts is the row's
    // last 8 elements, shifted on the way to LDS.  Rows behind the last repeat it and are
    // zeroed on that way.  (A row of fewer than 8 elements is loaded by elements.)
    struct Loaded {
        Eight<TG> e[DIRECT ? 1 : GROUNDS];
        int left;                                  // of the step's rows, those from this thread's first on
    };
    Loaded gring[DIRECT ? 1 : kImages];
    const int64_t gcol = max(min(gn, a.N - 8), (int64_t)0);
    const bool gcut = gn < a.N && gn + 8 > a.N;
    const int gshift = a.N >= 8 && gcut ? (int)(gn - gcol) : 0;
    auto load_g = [&](Loaded& to, int s) {
        to.left = rows - s * kStepRows - grow;
        if (rows <= 0) return;
#pragma unroll
        for (int i = 0; i < (DIRECT ? 0 : GROUNDS); i++) {
            const int m = min(s * kStepRows + grow + i * GSTEP, rows - 1);
            const TG* const p = (const TG*)a.g + (row0 + m) * a.gstride;
            if (a.N >= 8) {
                to.e[i].v = Vec<TG, 8>::raw(p + gcol);
            } else if (gcut) {
#pragma unroll
                for (int q = 0; q < 8; q++) to.e[i].v[q] = gn + q < a.N ? p[gn + q] : (TG)0.f;
            }
        }
    };
    auto put_g = [&](auto image, const Loaded& from) {
#pragma unroll
        for (int i = 0; i < (DIRECT ? 0 : GROUNDS); i++) {
            char* const to = gat(image) + GI::row(grow) + i * (GSTEP / GI::BLOCK_ROWS) * GI::BLOCK +
                             (t % GPIECES ^ GI::key(grow) << 1) * 16;
            u32x4 w[P];
            const bool there = i * GSTEP < from.left;
            Eight<TG> e = from.e[i];
            if (gshift) {
#pragma unroll
                for (int d = 4; d; d /= 2)
                    if (gshift & d) {
#pragma unroll
                        for (int q = 0; q < 8; q++) e.v[q] = q + d < 8 ? e.v[q + d < 8 ? q + d : q] : (TG)0.f;
                    }
            }
            if constexpr (P == 1) {
                __builtin_memcpy(&w[0], &e.v, 16);
                w[0] = there ? w[0] : u32x4{0u, 0u, 0u, 0u};
            } else {
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    float lo[P], hi[P];
                    cut<P>(there ? (float)e.v[2 * q] : 0.f, lo);
                    cut<P>(there ? (float)e.v[2 * q + 1] : 0.f, hi);
#pragma unroll
                    for (int p = 0; p < P; p++) w[p][q] = pack_exact(lo[p], hi[p]);
                }
            }
#pragma unroll
            for (int p = 0; p < P; p++) *(u32x4*)(to + p * GI::BYTES) = w[p];
        }
    };

    // The kept rows: pieces of 16 codes, one per thread (in tiles of 64 the second half of the threads has none).
    constexpr int XPIECES = COLS / 16, XTHREADS = kStepRows * XPIECES;
    static_assert(XTHREADS <= THREADS, "one piece per thread");
    const int xt = t % XTHREADS, xrow = xt / XPIECES, xpiece = xt % XPIECES;
    const int64_t xb = (k0 + xpiece * 16) / kMx8Block;
    const bool xin = xb < a.blocks;
    const int64_t pitch = a.blocks * kMx8Block;
    Rows crows(a.codes + row0 * pitch + k0, rows, pitch, k0);
    Rows srows(a.scales + row0 * a.blocks + k0 / kMx8Block, rows, a.blocks, k0 / kMx8Block);
    const uint32_t cplace = xin ? xrow * (uint32_t)pitch + xpiece * 16 : kNowhere;
    const uint32_t splace = xin ? xrow * (uint32_t)a.blocks + xpiece * 16 / kMx8Block : kNowhere;
    int xput = XI::row(xrow) + (xpiece ^ XI::key(xrow)) * 32;
    struct Kept {
        u32x4 c;
        int scale;
    };
    Kept xring[kImages];
    auto load_x = [&] {                            // a load for every thread: waits count them
        const Buffer c = crows.buffer(0), e = srows.buffer(0);
        crows.advance();
        srows.advance();
        return Kept{__builtin_amdgcn_raw_buffer_load_b128(c, cplace, 0, 0), __builtin_amdgcn_raw_buffer_load_b8(e, splace, 0, 0)};
    };
    // Pair N of the 8 pairs of codes; four of them are a store.
    u32x4 xword;
    auto put_x = [&](auto image, auto pair, const Kept& r) {
        constexpr int N = decltype(pair)::value;
        const uint32_t c = r.c[N / 2] >> (N % 2 * 16);
        const float scale = r.scale == 255 ? __uint_as_float(0x7FC00000u) : ldexpf(1.f, r.scale - 133);
        xword[N % 4] = pack_exact((float)(int8_t)c * scale, (float)(int8_t)(c >> 8) * scale);
        if constexpr (N % 4 == 3)
            if (XTHREADS == THREADS || t < XTHREADS) *(u32x4*)(xat(image) + xput + N / 4 * 16) = xword;
    };

    // Operands.  A lane's 8 m are 4 (lane / 16) + {0 .. 3} and those plus 16, in both operands.
    const int mrow = lane / 4 % 4 + lane / 16 * 4;
    int gr[GI::KEYS], xr[XI::KEYS];                // for tiles that differ in the key's bits
#pragma unroll
    for (int q = 0; q < GI::KEYS; q++) gr[q] = GI::row(mrow) + ((wm * F + q) ^ GI::key(mrow)) * 32 + lane % 4 * 8;
#pragma unroll
    for (int q = 0; q < XI::KEYS; q++) xr[q] = XI::row(mrow) + ((wn * G + q) ^ XI::key(mrow)) * 32 + lane % 4 * 8;
    static_assert((F % GI::KEYS == 0 || F < GI::KEYS) && (G % XI::KEYS == 0 || G < XI::KEYS), "");
    auto read = [&](const char* at, int half) {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        union {
            s16x4 s[2];
            bf16x8 v;
        } r;
        r.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
        r.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + half));
        return r.v;
    };
    bf16x8 gv[P][F], xv[G];
    auto read_g = [&](auto s, auto i) {
        constexpr int I = decltype(i)::value;
        static_for<P>([&](auto p) {
            constexpr int Q = decltype(p)::value;
            gv[Q][I] = read(gat(s) + Q * GI::BYTES + gr[I % GI::KEYS] + I / GI::KEYS * GI::KEYS * 32, GI::row(16));
        });
    };
    auto read_x = [&](auto s, auto j) {
        constexpr int J = decltype(j)::value;
        xv[J] = read(xat(s) + xr[J % XI::KEYS] + J / XI::KEYS * XI::KEYS * 32, XI::row(16));
    };
    // A wave's fetches, but the last step's ones, and its own stores are in LDS; then all waves'.
    constexpr int COUNTED = P * GROUNDS + 2;
    auto arrived = [](auto later) {
        if constexpr (DIRECT) __builtin_amdgcn_s_waitcnt(0x0070 | decltype(later)::value);
        else __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0) alone
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    static_assert(!DIRECT || COUNTED < 16, "what a wait can count here");

    // Step s, whose image is the constant, on its way to registers, and from there into LDS.
    auto load = [&](auto image, int s) {
        xring[decltype(image)::value % kImages] = load_x();
        if constexpr (!DIRECT) load_g(gring[decltype(image)::value % kImages], s);
    };
    auto put = [&](auto image, auto pair) {
        if constexpr (!DIRECT && decltype(pair)::value == 0) put_g(image, gring[decltype(image)::value % kImages]);
        put_x(image, pair, xring[decltype(image)::value % kImages]);
    };
    // Steps 0 .. 2 on their way, 0 and 1 in LDS.
    if constexpr (DIRECT)
        static_for<3>([&](auto i) {
            static_for<P * GROUNDS>([&](auto r) { fetch_g(i, r); });
        });
    static_for<3>([&](auto i) { load(i, decltype(i)::value); });
    static_for<2>([&](auto i) {
        static_for<8>([&](auto n) { put(i, n); });
    });
    arrived(Const<0>{});
    static_for<F>([&](auto i) { read_g(Const<0>{}, i); });
    static_for<G>([&](auto j) { read_x(Const<0>{}, j); });
    // Step s: its operands are in registers.  Behind the barrier step s + 1 is in
    // LDS, and nobody reads the images of step s and before any more (a wave waits
    // for its reads before the barrier), so step s + 3 may take that of step s.
    auto step = [&](auto image, int s) {
        constexpr int S = decltype(image)::value;
        arrived(Const<DIRECT ? COUNTED : 0>{});
        // Addresses in an image are sums of these; kept over the loop for all
        // images they would not fit the registers.
#pragma unroll
        for (int q = 0; q < GI::KEYS; q++) asm volatile("" : "+v"(gr[q]));
#pragma unroll
        for (int q = 0; q < XI::KEYS; q++) asm volatile("" : "+v"(xr[q]));
        asm volatile("" : "+v"(xput));
        static_for<F>([&](auto ci) {               // 16 rows of out
            constexpr int I = decltype(ci)::value;
            static_for<G>([&](auto cj) {
                constexpr int J = decltype(cj)::value;
                static_for<P>([&](auto p) {        // the smallest part first
                    acc[I][J] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv[J], gv[P - 1 - decltype(p)::value][I], acc[I][J], 0,
                                                                       0, 0);
                });
                if constexpr (I == F - 1) read_x(Const<S + 1>{}, cj);
            });
            read_g(Const<S + 1>{}, ci);            // in the place of what has been multiplied
            static_for<8>([&](auto n) {
                if constexpr (decltype(n)::value * F / 8 == I) put(Const<S + 2>{}, n);
            });
            if constexpr (I == (F > 2 ? 1 : 0)) load(Const<S + 3>{}, s + 3);
            if constexpr (DIRECT)
                static_for<P * GROUNDS>([&](auto r) {          // behind the kept codes' loads
                    constexpr int R = decltype(r)::value, AT = F > 2 ? 2 + R * (F - 2) / (P * GROUNDS) : 1;
                    if constexpr (AT == I) fetch_g(Const<S + 3>{}, r);
                });
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    for (int s = 0; s < steps; s += kImages) {     // steps behind the last one multiply zeros
        // Sums in accumulation registers: the compiler would let them wander
        // through all 256 and spill operands.
#pragma unroll
        for (int i = 0; i < F; i++)
#pragma unroll
            for (int j = 0; j < G; j++) asm volatile("" : "+a"(acc[i][j]));
        static_for<kImages>([&](auto i) { step(i, s + decltype(i)::value); });
    }
    __builtin_amdgcn_s_waitcnt(kVmcnt0);           // the last fetches, before LDS is used again
    __syncthreads();

    // Rows leave through LDS, each wave its own part in strips of 16 rows, as
    // pieces along a row.
    constexpr int E = 16 / (int)sizeof(TW), PITCH = 16 * G + 4;
    constexpr int SHARE = (WM * WN + 3) / 4;       // waves per LDS object
    static_assert(SHARE * 16 * PITCH * 4 <= P * GI::BYTES && SHARE * 16 * PITCH * 4 <= XI::BYTES, "a strip per wave");
    char* const part = wave / SHARE == 0 ? g0 : wave / SHARE == 1 ? g1 : wave / SHARE == 2 ? g2 : x0;
    float* const strip_at = (float*)part + wave % SHARE * 16 * PITCH;
    TW* const out = a.parts ? (TW*)a.parts + (int64_t)blockIdx.y * a.N * a.K : (TW*)a.out;      // parts: launched with TW = float
    const int64_t ostride = a.parts ? a.K : a.stride;
    const bool accumulate = !a.parts && a.accumulate;
    const int64_t wn0 = n0 + wm * 16 * F, wk0 = k0 + wn * 16 * G;
#pragma unroll
    for (int i = 0; i < F; i++) {
#pragma unroll
        for (int j = 0; j < G; j++) *(f32x4*)(strip_at + lane % 16 * PITCH + j * 16 + lane / 16 * 4) = acc[i][j];
        wave_sync();
        constexpr int PER_ROW = 16 * G / E, ROUNDS = (16 * PER_ROW + kWave - 1) / kWave;
#pragma unroll
        for (int q = 0; q < ROUNDS; q++) {
            const int at = q * kWave + lane, row = at / PER_ROW, c = at % PER_ROW * E;
            const int64_t n = wn0 + i * 16 + row, k = wk0 + c;
            if (row >= 16 || n >= a.N || k >= a.K) continue;
            TW* const to = out + n * ostride + k;
            float y[E];
#pragma unroll
            for (int e = 0; e < E; e++) y[e] = strip_at[row * PITCH + c + e];
            if (k + E <= a.K) {
                if (accumulate) {
                    float old[E];
                    Vec<TW, E>::load(to, old);
#pragma unroll
                    for (int e = 0; e < E; e++) y[e] += old[e];
                }
                Vec<TW, E>::store(to, y, a.nt);
            } else {
#pragma unroll
                for (int e = 0; e < E; e++)
                    if (k + e < a.K) to[e] = from_float<TW>(accumulate ? to_float(to[e]) + y[e] : y[e]);
            }
        }
        wave_sync();
    }
}

constexpr int kJoinCols = 16;                      // of the bias gradient per workgroup, the other threads' share of the parts each
constexpr int kJoinLanes = 16;                     // threads that share the parts of four elements of a small gradient

// Adds what `lanes` threads hold, kBlock / lanes apart; the first of them has the sum.
template <int E> __device__ __forceinline__ void join_lanes(float (*red)[4], float (&y)[E], int lanes) {
    const int side = kBlock / lanes, l = threadIdx.x / side;
#pragma unroll
    for (int e = 0; e < E; e++) red[threadIdx.x][e] = y[e];
    for (int d = lanes / 2; d; d /= 2) {
        __syncthreads();
        if (l < d) {
#pragma unroll
            for (int e = 0; e < E; e++) red[threadIdx.x][e] += red[threadIdx.x + d * side][e];
        }
    }
#pragma unroll
    for (int e = 0; e < E; e++) y[e] = red[threadIdx.x][e];
}

// out from the sum of the parts, always in the same order, by the first `groups`
// workgroups, `lanes` threads for every four elements; the bias gradient from its
// parts by the others, 16 columns at a time.  (9 x 150 in 341 parts, by one thread each: 150 us.)
template <typename TW> __global__ __launch_bounds__(kBlock) void k_mx8_wgrad_join(WgradArgs a, int parts, int groups, int lanes) {
    __shared__ float red[kBlock][4];
    if ((int)blockIdx.x >= groups) {
        constexpr int LANES = kBlock / kJoinCols;
        const int l = threadIdx.x / kJoinCols;
        for (int64_t n0 = (int64_t)(blockIdx.x - groups) * kJoinCols; n0 < a.N; n0 += (int64_t)(gridDim.x - groups) * kJoinCols) {
            const int64_t n = n0 + threadIdx.x % kJoinCols;
            float s[1] = {0.f};
            if (n < a.N) {
#pragma unroll 8
                for (int p = l; p < a.bias_parts; p += LANES) s[0] += a.bias_sums[(int64_t)p * a.N + n];
            }
            join_lanes(red, s, LANES);
            if (l == 0 && n < a.N) a.db[n] = a.accumulate ? a.db[n] + s[0] : s[0];
            __syncthreads();                       // red is used again
        }
        return;
    }
    const int side = kBlock / lanes, l = threadIdx.x / side;
    const int64_t total = a.N * a.K, step = (int64_t)groups * side * 4;
    // with several lanes the workgroups cover everything in one round
    for (int64_t i = ((int64_t)blockIdx.x * side + threadIdx.x % side) * 4; i < total || lanes > 1; i += step) {
        const int count = (int)max((int64_t)0, min((int64_t)4, total - i));
        float y[4] = {0.f, 0.f, 0.f, 0.f};
        if (count == 4) {
#pragma unroll 8
            for (int p = l; p < parts; p += lanes) {
                float v[4];
                Vec<float, 4>::load(a.parts + p * total + i, v);
#pragma unroll
                for (int e = 0; e < 4; e++) y[e] += v[e];
            }
        } else {
            for (int p = l; p < parts; p += lanes)
                for (int e = 0; e < count; e++) y[e] += a.parts[p * total + i + e];
        }
        if (lanes > 1) {
            join_lanes(red, y, lanes);
            if (l > 0 || count == 0) return;
        }
        const int64_t n = i / a.K, k = i % a.K;
        if (k + 4 <= a.K) {                        // all in one row
            TW* const to = (TW*)a.out + n * a.stride + k;
            if (a.accumulate) {
                float old[4];
                Vec<TW, 4>::load(to, old);
#pragma unroll
                for (int e = 0; e < 4; e++) y[e] += old[e];
            }
            Vec<TW, 4>::store(to, y);
        } else {
            for (int e = 0; e < count; e++) {
                TW* const to = (TW*)a.out + (i + e) / a.K * a.stride + (i + e) % a.K;
                *to = from_float<TW>(a.accumulate ? to_float(*to) + y[e] : y[e]);
            }
        }
        if (lanes > 1) return;
    }
}

// ----------------------------------------------------------------- columns of the gradient

// One pass over g: its planes of bfloat16 with rows of whole pieces (P > 0), and
// the sums of its columns over parts of the rows (sums not NULL).  A thread takes 8 columns
// of every (kBlock / L)-th row of its workgroup's part; L threads side by side.
template <typename TG, int P>
__global__ __launch_bounds__(kBlock) void k_mx8_columns(const TG* __restrict__ g, int64_t gstride, int64_t M, int64_t N, int L,
                                                        int64_t share, uint16_t* __restrict__ planes, int64_t pitch,
                                                        float* __restrict__ sums) {
    __shared__ float red[kBlock][8];
    const int l = threadIdx.x / L, lanes = kBlock / L;
    const int64_t n = ((int64_t)blockIdx.x * L + threadIdx.x % L) * 8, m0 = share * blockIdx.y, m1 = min(M, m0 + share);
    constexpr int U = 4;
    float s[8] = {};
    if (n < N)
        for (int64_t m = m0 + l; m < m1; m += U * lanes) {
            float x[U][8];
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (m + u * lanes < m1) {
                    load8<TG>(g + (m + u * lanes) * gstride, n, N, x[u]);
                } else {
#pragma unroll
                    for (int q = 0; q < 8; q++) x[u][q] = 0.f;
                }
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
#pragma unroll
                for (int q = 0; q < 8; q++) s[q] += x[u][q];
                if constexpr (P > 0) {
                    if (m + u * lanes >= m1) continue;
                    u32x4 w[P];
#pragma unroll
                    for (int q = 0; q < 4; q++) {
                        float lo[P], hi[P];
                        cut<P>(x[u][2 * q], lo);
                        cut<P>(x[u][2 * q + 1], hi);
#pragma unroll
                        for (int p = 0; p < P; p++) w[p][q] = pack_exact(lo[p], hi[p]);
                    }
#pragma unroll
                    for (int p = 0; p < P; p++) *(u32x4*)(planes + (p * M + m + u * lanes) * pitch + n) = w[p];
                }
            }
        }
    if (!sums) return;
#pragma unroll
    for (int q = 0; q < 8; q++) red[threadIdx.x][q] = s[q];
    for (int d = lanes / 2; d; d /= 2) {           // a power of two of lanes
        __syncthreads();
        if (l < d) {
#pragma unroll
            for (int q = 0; q < 8; q++) red[threadIdx.x][q] += red[threadIdx.x + d * L][q];
        }
    }
    if (l == 0 && n < N) {
#pragma unroll
        for (int q = 0; q < 8; q++)
            if (n + q < N) sums[(int64_t)blockIdx.y * N + n + q] = red[threadIdx.x][q];
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
template <typename F> static void with_bools(bool a, bool b, F&& f) {
    if (a && b) f(std::true_type{}, std::true_type{});
    else if (a) f(std::true_type{}, std::false_type{});
    else if (b) f(std::false_type{}, std::true_type{});
    else f(std::false_type{}, std::false_type{});
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
    const int64_t R = y->rows, F = y->cols, blocks = blocks_of(x->cols);
    // halves that meet inside a block: their codes by a pass of their own
    const bool apart = kept && gated && F % kMx8Block != 0;
    if (kept) {
        check_mx8(kept, "kept");
        AGNES_REQUIRE(kept->rows == x->rows && kept->cols == x->cols, AGNES_ERR_INVALID, "x and kept must have equal shapes");
    }
    if (R == 0 || F == 0) return;
    if (apart) mx8_quantize(x, kept, st);
    const bool keep = kept && !apart, nt = R * F * (int64_t)elem_size(y->dtype) > kStreamBytes;
    const int64_t per_row = keep ? blocks_of(F) * 4 : (F + 7) / 8;
    with_float(x->dtype, [&](auto t) {
        with_float(y->dtype, [&](auto ty) {
            with_act(act, [&](auto a) {
                with_bools(gated, keep, [&](auto g, auto k) {
                    typedef decltype(t) T;
                    typedef decltype(ty) TY;
                    constexpr int U = kPieces / (decltype(g)::value ? 2 : 1);
                    launch_pieces<U>(R, per_row, [&](int64_t r, int64_t pieces, unsigned groups) {
                        AGNES_LAUNCH((k_mx8_act<T, TY, decltype(a)::value, decltype(g)::value, decltype(k)::value>), dim3(groups),
                                     dim3(kBlock), 0, st, (const T*)x->data + r * x->stride, x->stride, pieces, F,
                                     (uint32_t)per_row, keep ? kept->codes + r * blocks * kMx8Block : nullptr,
                                     keep ? kept->scales + r * blocks : nullptr, blocks, (TY*)y->data + r * y->stride,
                                     y->stride, nt);
                    });
                });
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
    const int64_t R = grad_y->rows, F = grad_y->cols, blocks = blocks_of(kept->cols), per_row = (F + 7) / 8;
    if (R == 0 || F == 0) return;
    const bool whole = !gated || F % kMx8Block == 0, nt = R * kept->cols * (int64_t)elem_size(grad_x->dtype) > kStreamBytes;
    with_float(grad_y->dtype, [&](auto tg) {
        with_float(grad_x->dtype, [&](auto tx) {
            with_act(act, [&](auto a) {
                with_bools(gated, whole, [&](auto g, auto w) {
                    typedef decltype(tg) TG;
                    typedef decltype(tx) TX;
                    constexpr int U = kPieces / (decltype(g)::value ? 2 : 1);
                    launch_pieces<U>(R, per_row, [&](int64_t r, int64_t pieces, unsigned groups) {
                        AGNES_LAUNCH((k_mx8_act_grad<TG, TX, decltype(a)::value, decltype(g)::value, decltype(w)::value>),
                                     dim3(groups), dim3(kBlock), 0, st, kept->codes + r * blocks * kMx8Block,
                                     kept->scales + r * blocks, blocks, pieces, F, (uint32_t)per_row,
                                     (const TG*)grad_y->data + r * grad_y->stride, grad_y->stride,
                                     (TX*)grad_x->data + r * grad_x->stride, grad_x->stride, nt);
                    });
                });
            });
        });
    });
}

constexpr int64_t kPartSteps = 4;                  // fewest steps of a part
constexpr int64_t kColumnGrid = 1024;              // workgroups that a pass over the gradient's columns aims at
constexpr int64_t kColumnRows = 64;                // fewest rows of its parts

// How a gradient is computed, by sizes, by how many planes it has and by whether they go straight to LDS.
struct WgradPlan {
    int rows, cols, parts;                         // of a tile; of M
    int lanes;                                     // of the pass over columns: its threads side by side,
    int64_t share;                                 // rows of its parts
    int column_parts;
};

// The tile and the parts that are fastest by what their steps have measured (us
// per step of one workgroup alone on its compute unit, and per step and
// workgroup of a full one; and what a workgroup needs before its first step and
// behind its last), with the joining of the parts at 4 TB/s.
// 16384 x 4096 x 4096: bfloat16 in tiles of 256, 128 and 64 takes 490, 680 and 1800
// us; float16 in tiles of 128 x 256, 128 and 64 takes 960, 1305 and 2960 us, float32
// 1370, 1815 and 3775 us.  65536 x 256 x 1024 bfloat16: 88, 70 and 96 us in each tile's best
// parts; 8192 x 512 x 512: 42, 23 and 26 us.
static WgradPlan plan_wgrad(int64_t M, int64_t N, int64_t K, int planes, bool straight) {
    WgradPlan p{64, 64, 1, 1, 1, 1};
    const int64_t steps = (M + kStepRows - 1) / kStepRows;
    auto tiles = [&](int64_t r, int64_t c) { return ((N + r - 1) / r) * ((K + c - 1) / c); };
    struct Tile {
        int rows, cols;
        double alone[3], full[3], ends;            // of 1, 2, 3 planes
    };
    static const Tile kTiles[] = {{256, 256, {1.0, 0, 0}, {1.0, 0, 0}, 10},
                                  {128, 256, {0, 0.92, 1.25}, {0, 0.92, 1.25}, 10},
                                  {128, 128, {0.49, 0.63, 0.86}, {0.33, 0.63, 0.86}, 10},
                                  {64, 64, {0.28, 0.42, 0.6}, {0.21, 0.32, 0.46}, 4}};
    double best = 0;
    for (const Tile& t : kTiles) {
        if (t.full[planes - 1] == 0 || (t.rows > 64 && !straight)) continue;
        for (int64_t grid : {1, 256, 512, 1024}) {
            const int64_t parts = std::max<int64_t>(1, std::min(grid / std::max<int64_t>(1, tiles(t.rows, t.cols)), steps / kPartSteps));
            const double each = (double)((steps + parts - 1) / parts), groups = (double)(tiles(t.rows, t.cols) * parts);
            const double us = t.ends + std::max(each * t.alone[planes - 1], std::ceil(groups / 256) * each * t.full[planes - 1]) +
                              (parts > 1 ? 6 + (double)(parts * N * K) * 8 / 4e6 : 0);
            if (best == 0 || us < best) {
                best = us;
                p.rows = t.rows;
                p.cols = t.cols;
                p.parts = (int)parts;
            }
        }
    }
    const int64_t pieces = (N + 7) / 8;
    while (p.lanes < 32 && p.lanes < pieces) p.lanes *= 2;
    const int64_t across = (pieces + p.lanes - 1) / p.lanes;
    if (across > 0) {
        const int64_t least = std::max(kColumnRows, (int64_t)kBlock / p.lanes * 4);      // a round of loads for every thread
        const int64_t want = std::max<int64_t>(1, std::min<int64_t>((kColumnGrid + across - 1) / across, M / least));
        p.share = std::max<int64_t>(1, (M + want - 1) / want);
        p.column_parts = (int)std::max<int64_t>(1, (M + p.share - 1) / p.share);
    }
    return p;
}

// Gradients that cannot go straight to LDS are cut into planes by a pass of
// their own, where there is work enough for it: otherwise every tile cuts them
// again, and rows that start at odd addresses are read slowly by every tile.  (us, with that pass / cut in tiles:
// 16384 x 4095 x 4096 bfloat16 580 / 2600, 60000 x 47 x 256 float32 78 / 91, 8192 x 515 x 512
// 58 / 70, 2048 x 512 x 512 27 / 23, 2048 x 512 x 128 23 / 18.)
static bool make_planes(int64_t M, int64_t N, int64_t K) { return M * N >= (1 << 21) || (K >= 1024 && M >= 256); }

static int64_t plane_pitch(int64_t N) { return (N + 7) / 8 * 8; }

// How a gradient reaches its tiles.
struct WgradWay {
    int planes;                                    // bfloat16 that add up to an element
    bool direct, cut;                              // straight to LDS as it is; cut into planes first
    bool straight() const { return direct || cut; }
};
static WgradWay way_of(const agnes_matrix* g, int64_t K) {
    const int64_t M = g->rows, N = g->cols;
    WgradWay w{g->dtype == AGNES_FLOAT32 ? 3 : g->dtype == AGNES_FLOAT16 ? 2 : 1, false, false};
    // bfloat16 rows of whole 16-byte pieces, within a buffer's reach
    w.direct = w.planes == 1 && ((uintptr_t)g->data & 15) == 0 && g->stride % 8 == 0 && N % 8 == 0 && g->stride >= N &&
               g->stride * 2 <= kMaxPitch;
    w.cut = !w.direct && make_planes(M, N, K) && plane_pitch(N) * 2 <= kMaxPitch;
    return w;
}

static void check_wgrad(const agnes_matrix* grad_out, int64_t K) {
    check_matrix(grad_out, false, "grad_out");
    AGNES_REQUIRE(K >= 0 && K <= kMaxPitch, AGNES_ERR_INVALID, "K must be in [0, 2^25]");
    // by the smallest tile, so that no gradient is refused for its type or layout
    AGNES_REQUIRE((grad_out->cols + 63) / 64 * ((K + 63) / 64) <= (1 << 23) - kXcds, AGNES_ERR_RANGE,
                  "the gradient has too many tiles");
}

uint64_t mx8_weight_grad_bytes(const agnes_matrix* grad_out, int64_t K) {
    check_wgrad(grad_out, K);
    const int64_t M = grad_out->rows, N = grad_out->cols;
    const WgradWay w = way_of(grad_out, K);
    const WgradPlan p = plan_wgrad(M, N, K, w.planes, w.straight());
    Carve c(nullptr);
    if (p.parts > 1) c.take<float>(p.parts * N * K);
    c.take<float>(p.column_parts * N);
    if (w.cut) c.take<uint16_t>(w.planes * M * plane_pitch(N));
    return c.used;
}

template <typename TG, int P, typename TW, bool DIRECT, int WM, int WN, int F, int G>
static void launch_tiles(const WgradArgs& a, int parts, hipStream_t st) {
    constexpr int R = WM * 16 * F, C = WN * 16 * G;
    const int64_t tiles = ((a.N + R - 1) / R) * ((a.K + C - 1) / C);
    const unsigned grid = (unsigned)((tiles + kXcds - 1) / kXcds * kXcds);
    AGNES_LAUNCH((k_mx8_wgrad<TG, P, TW, DIRECT, WM, WN, F, G>), dim3(grid, (unsigned)parts), dim3(kWave * WM * WN), 0, st, a);
}

// TG: float, _Float16 or __bf16 through registers, or P planes straight to LDS.
template <typename TG, int P, typename TW, bool DIRECT>
static void launch_wgrad(const WgradArgs& a, const WgradPlan& p, hipStream_t st) {
    if constexpr (DIRECT && P == 1) {
        if (p.rows == 256) return launch_tiles<TG, P, TW, DIRECT, 2, 4, 8, 4>(a, p.parts, st);
    }
    if constexpr (DIRECT && P > 1) {
        if (p.cols == 256) return launch_tiles<TG, P, TW, DIRECT, 2, 4, 4, 4>(a, p.parts, st);
    }
    if constexpr (DIRECT) {
        if (p.rows == 128) return launch_tiles<TG, P, TW, DIRECT, 2, 2, 4, 4>(a, p.parts, st);
    }
    launch_tiles<TG, P, TW, DIRECT, 2, 2, 2, 2>(a, p.parts, st);
}

template <typename TG, int P>
static void launch_columns(const agnes_matrix* g, const WgradPlan& p, uint16_t* planes, float* sums, hipStream_t st) {
    const int64_t pieces = (g->cols + 7) / 8;
    AGNES_LAUNCH((k_mx8_columns<TG, P>), dim3((unsigned)((pieces + p.lanes - 1) / p.lanes), (unsigned)p.column_parts),
                 dim3(kBlock), 0, st, (const TG*)g->data, g->stride, g->rows, g->cols, p.lanes, p.share, planes,
                 plane_pitch(g->cols), sums);
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
    check_workspace(ws, ws_bytes, mx8_weight_grad_bytes(grad_out, K));      // checks K and the number of tiles too
    if (N == 0) return;
    const WgradWay way = way_of(grad_out, K);
    const bool direct = way.direct, planes = way.cut;
    with_float(grad_out->dtype, [&](auto tg) {
        typedef decltype(tg) TG;
        constexpr int P = kParts<TG>;
        const WgradPlan p = plan_wgrad(M, N, K, P, way.straight());
        Carve c(ws);
        WgradArgs a{};
        a.g = grad_out->data;
        a.gstride = grad_out->stride;
        a.codes = kept->codes;
        a.scales = kept->scales;
        a.M = M;
        a.N = N;
        a.K = K;
        a.blocks = blocks_of(K);
        a.out = grad_weight->data;
        a.stride = grad_weight->stride;
        a.accumulate = accumulate;
        a.nt = !accumulate && N * K * (int64_t)elem_size(grad_weight->dtype) > kStreamBytes;
        if (p.parts > 1) a.parts = c.take<float>(p.parts * N * K);
        float* const sums = grad_bias ? p.column_parts > 1 ? c.take<float>(p.column_parts * N) : grad_bias : nullptr;
        const bool join_bias = grad_bias && (p.column_parts > 1 || accumulate);
        float* const first = join_bias && p.column_parts == 1 ? c.take<float>(N) : sums;
        if (planes) {
            uint16_t* const to = c.take<uint16_t>(P * M * plane_pitch(N));
            launch_columns<TG, P>(grad_out, p, to, first, st);
            a.g = to;
            a.gstride = plane_pitch(N);
            a.gplane = M * plane_pitch(N);
        } else if (grad_bias) {
            launch_columns<TG, 0>(grad_out, p, nullptr, first, st);
        }
        a.bias_sums = first;
        a.bias_parts = p.column_parts;
        a.db = grad_bias;
        auto tiles = [&](auto tw) {
            typedef decltype(tw) TW;
            if (planes || direct) launch_wgrad<__bf16, P, TW, true>(a, p, st);
            else launch_wgrad<TG, P, TW, false>(a, p, st);
        };
        if (K > 0 && p.parts > 1) tiles(float{});
        with_float(grad_weight->dtype, [&](auto tw) {
            if (K > 0 && p.parts == 1) tiles(tw);
            const int lanes = p.parts >= kJoinLanes && N * K <= (1 << 18) ? kJoinLanes : 1;
            const int64_t fours = (N * K + 3) / 4;
            const int groups = K == 0 || p.parts == 1 ? 0
                               : lanes > 1 ? (int)((fours * lanes + kBlock - 1) / kBlock) : (int)grid_for(fours, 4096);
            const int more = join_bias ? (int)std::min<int64_t>((N + kJoinCols - 1) / kJoinCols, kLaunchGroups) : 0;
            if (groups + more > 0)
                AGNES_LAUNCH((k_mx8_wgrad_join<decltype(tw)>), dim3(groups + more), dim3(kBlock), 0, st, a, p.parts, groups,
                             lanes);
        });
    });
}

}  // namespace agnes
