// Microscaled 4-bit floating point (MXFP4): rows to 4-bit codes with one
// power-of-two scale per block of 32 elements, back to values, and the product
// of two matrices in that form.
//
// A block's scale is 2^(floor(log2 max|x|) - 2): the largest element lands in
// [4, 8), and 2^2 is the largest power of two that the 4-bit format holds.
#include <algorithm>
#include <type_traits>

#include "ops.hpp"

namespace agnes {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kMxBlock = 32;                       // elements per scale
static int64_t mx_blocks(int64_t cols) { return (cols + kMxBlock - 1) / kMxBlock; }

// ----------------------------------------------------------------- elements

// 2^e for e in [-127, 127] (2^-127 is a subnormal).
__device__ __forceinline__ float exp2_int(int e) {
    return __uint_as_float(e >= -126 ? (uint32_t)(e + 127) << 23 : 1u << 22);
}

// The scale code of a block whose largest magnitude has the float32 bits `top`.
__device__ __forceinline__ int scale_code(uint32_t top) {
    const int e = (int)(top >> 23);
    return e == 255 ? 255 : max(e - 2, 0);
}

// Eight elements times 2^(127 - code), to eight 4-bit codes, the first in the
// low bits: nearest, ties to the even code, magnitudes above 6 to 6.  The
// product is exact, so the conversion instruction rounds once; its own scale
// is 1.
__device__ __forceinline__ uint32_t to_codes(const float (&x)[8], int code) {
    const float inv = code == 255 ? 0.f : exp2_int(127 - code);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0] * inv, x[1] * inv, 1.f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2] * inv, x[3] * inv, 1.f, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4] * inv, x[5] * inv, 1.f, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6] * inv, x[7] * inv, 1.f, 3);
    if (code == 255) return 0;                     // 0 * inf above
    const uint32_t zero = ((x[0] == 0.f) << 3) | ((x[1] == 0.f) << 7) | ((x[2] == 0.f) << 11) | ((x[3] == 0.f) << 15) |
                          ((x[4] == 0.f) << 19) | ((x[5] == 0.f) << 23) | ((x[6] == 0.f) << 27) |
                          ((uint32_t)(x[7] == 0.f) << 31);
    return r & ~zero;                              // -0 as 0
}

// ----------------------------------------------------------------- quantisation

// A piece is 8 elements, a block four pieces in adjacent lanes.  Pieces are
// numbered row after row; a workgroup takes kPieces rounds of 256, all loads
// first.  Bound by memory: 65536 x 1024 bfloat16 to codes 40 us (4.3 TB/s), and
// back 27 us (6.4 TB/s).
template <typename T>
__global__ __launch_bounds__(kBlock) void k_mx4_quantize(const T* __restrict__ x, int64_t stride, int64_t pieces,
                                                         int64_t cols, uint32_t per_row, uint8_t* __restrict__ codes,
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
        float top = __uint_as_float(top_bits(v[u]));
        // as unsigned numbers, NaN above infinity above all finite values
        uint32_t t = __float_as_uint(top);
        t = max(t, __float_as_uint(lane_pair<1>(__uint_as_float(t))));
        t = max(t, __float_as_uint(lane_pair<2>(__uint_as_float(t))));
        const int code = scale_code(t);
        *(uint32_t*)(codes + 4 * i) = to_codes(v[u], code);
        if (threadIdx.x % 4 == 0) scales[i / 4] = (uint8_t)code;
    }
}

// Two 4-bit codes to float32, exactly; the scale is applied by a product, since
// 2^-127 is no normal number.
template <int BYTE> __device__ __forceinline__ void from_codes(uint32_t c, float s, float (&x)[8]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, BYTE);
    x[2 * BYTE] = v[0] * s;
    x[2 * BYTE + 1] = v[1] * s;
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_mx4_dequantize(const uint8_t* __restrict__ codes,
                                                           const uint8_t* __restrict__ scales, int64_t pieces,
                                                           int64_t cols, uint32_t per_row, T* __restrict__ x,
                                                           int64_t stride, bool nt) {
    const int64_t base = (int64_t)blockIdx.x * (kBlock * kPieces);
    const int64_t base_row = base / per_row;
    const uint32_t base_piece = (uint32_t)(base % per_row);
    uint32_t w[kPieces], s[kPieces];
#pragma unroll
    for (int u = 0; u < kPieces; u++) {
        const int64_t i = base + u * kBlock + threadIdx.x;
        if (i < pieces) {
            w[u] = *(const uint32_t*)(codes + 4 * i);
            s[u] = scales[i / 4];
        }
    }
#pragma unroll
    for (int u = 0; u < kPieces; u++) {
        const uint32_t off = u * kBlock + threadIdx.x;
        if (base + off >= pieces) continue;
        const PieceAt p = piece_at(base_row, base_piece, off, per_row);
        const float f = s[u] == 255 ? __uint_as_float(0x7FC00000u) : exp2_int((int)s[u] - 127);
        float v[8];
        from_codes<0>(w[u], f, v);
        from_codes<1>(w[u], f, v);
        from_codes<2>(w[u], f, v);
        from_codes<3>(w[u], f, v);
        T* row = x + p.row * stride;
        const int64_t c = (int64_t)p.piece * 8;
        if (c + 8 <= cols) {
            Vec<T, 8>::store(row + c, v, nt);
        } else {
#pragma unroll
            for (int q = 0; q < 8; q++)
                if (c + q < cols) row[c + q] = from_float<T>(v[q]);
        }
    }
}

// ----------------------------------------------------------------- product

// v_mfma_scale_f32_16x16x128 with 4-bit operands: lane l holds 32 consecutive k
// (one block, 16 bytes) of row l % 16 of either operand, k = 32 (l / 16), and
// that block's scale code in one byte of a register; D[4 (l / 16) + r][l % 16].  The
// weight goes in first, so a lane holds four adjacent columns of a row of out.
struct MxArgs {
    const uint8_t *xc, *xs, *wc, *ws;
    int64_t M, N;
    int32_t blocks;                                // per row
    const float* bias;
    bool relu, nt;
    void* out;
    int64_t stride;
    float* parts;                                  // [gridDim.y][M][N]: sums over parts of K instead of out, or NULL
};

__device__ __forceinline__ i32x8 operand(i32x4 v) { return i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; }

__device__ __forceinline__ float finish(float y, float bias, bool relu) {
    y += bias;
    return relu && y < 0.f ? 0.f : y;
}

// Sixteen zero bytes: blocks behind the last one of a row.
static __device__ const uint4 k_mx4_zero = {0u, 0u, 0u, 0u};

// A workgroup of WM x WN waves computes a tile of out, a wave 16 F x 16 G of it,
// in steps of 256 k: 128 bytes per row, a whole cache line.  (8192^3: 293 us, 3.75
// PFLOP/s; the matrix cores are busy 44 % of it and LDS 23 %, the rest is the
// wait for a step's first operands behind its barrier.  Wave tiles of 128 x 128,
// one wave per SIMD: 401 us.)  The next step's
// codes go from memory straight to the other half of LDS while this step's are
// multiplied.  A step's LDS image: row after row, 8 pieces of 16 bytes each,
// piece p of row r at place p ^ (r % 8): the 16 rows that a wave reads at once
// then lie in different banks.  Scales pass through registers into the order in
// which lanes read them: per 128 k and four 16-row tiles one register per lane
// holds all four tiles' codes, and the MFMA picks its byte.
constexpr int kStep = 8;                           // blocks per step

// One operand of a workgroup: WAVES waves of F 16-row tiles.
template <int WAVES, int F> struct MxSide {
    static constexpr int ROWS = WAVES * 16 * F;
    static constexpr int GROUPS = (F + 3) / 4;     // registers of scale codes per lane and 128 k
    static constexpr int CODES = ROWS * 16 * kStep;
    static constexpr int SCALES = 2 * WAVES * GROUPS * 256;
};

// One operand's rows of a step, codes straight to LDS.  The rows are `last` + 1
// from `codes` on; rows behind them repeat the last: they are not stored.
// TAIL: the step is a row's last and partial; zeros behind its end.
template <bool TAIL, int THREADS, int ROWS>
__device__ __forceinline__ void fetch_codes(const uint8_t* __restrict__ codes, int last, int blocks, int b0, char* lds) {
    const int t = threadIdx.x, r = t / 8, piece = (t % 8) ^ (r % 8);
    const uint32_t row_bytes = (uint32_t)blocks * 16;
    const uint8_t* const from = codes + (int64_t)b0 * 16;
    char* const to = lds + t / kWave * kWave * 16;
#pragma unroll
    for (int i = 0; i < ROWS * 8 / THREADS; i++) {
        const uint8_t* p = from + ((uint32_t)min(r + i * (THREADS / 8), last) * row_bytes + (uint32_t)piece * 16);
        if (TAIL && b0 + piece >= blocks) p = (const uint8_t*)&k_mx4_zero;
        __builtin_amdgcn_global_load_lds((global_void*)p, (lds_void*)(to + i * THREADS * 16), 16, 0, 0);
    }
}

// A row's scale codes of a step: 8 bytes; 1 behind its end, where codes are 0.
template <bool TAIL> __device__ __forceinline__ uint64_t fetch_scales(const uint8_t* __restrict__ row, int blocks, int b0) {
    typedef uint64_t __attribute__((aligned(1))) u64_bytes;
    if (!TAIL) return *(const u64_bytes*)(row + b0);
    uint64_t v = 0;
    for (int b = 0; b < kStep; b++) v |= (uint64_t)(b0 + b < blocks ? row[b0 + b] : 127) << (8 * b);
    return v;
}

// Where row r's codes go: block b of a step at + b / 4 * half + b % 4 * 64.
template <int WAVES, int F> __device__ __forceinline__ int scale_place(int r) {
    const int part = r / (16 * F), tile = r % (16 * F) / 16;
    return (part * MxSide<WAVES, F>::GROUPS + tile / 4) * 256 + r % 16 * 4 + tile % 4;
}

template <typename T, int WM, int WN, int F, int G>
__global__ __launch_bounds__(kWave* WM* WN) void k_mx4_gemm(MxArgs a) {
    typedef MxSide<WM, F> X;
    typedef MxSide<WN, G> W;
    constexpr int THREADS = kWave * WM * WN;
    // An object per operand and half, addressed with one offset: that way the
    // compiler sees that a fetch under way does not write what is being read, and
    // adds no wait of its own for it.
    __shared__ __attribute__((aligned(1024))) char x0[X::CODES], x1[X::CODES], w0[W::CODES], w1[W::CODES];
    __shared__ __attribute__((aligned(16))) char scales[2][X::SCALES + W::SCALES];
    const int t = threadIdx.x, lane = lane_id(), wave = wave_id(), wm = wave / WN, wn = wave % WN;
    // XCD x takes a contiguous run of tiles, in strips of 8 tile rows: the tiles
    // that run at once on it share rows of both operands in its L2.
    const int64_t tm = (a.M + X::ROWS - 1) / X::ROWS, tn = (a.N + W::ROWS - 1) / W::ROWS, tiles = tm * tn;
    const int64_t per = (tiles + kXcds - 1) / kXcds, id = blockIdx.x % kXcds * per + blockIdx.x / kXcds;
    if ((int64_t)blockIdx.x / kXcds >= per || id >= tiles) return;
    const int64_t strip = id / (8 * tn), high = min((int64_t)8, tm - strip * 8), in = id - strip * 8 * tn;
    const int64_t m0 = (strip * 8 + in % high) * X::ROWS, n0 = in / high * W::ROWS;
    const int xlast = (int)min((int64_t)X::ROWS, a.M - m0) - 1, wlast = (int)min((int64_t)W::ROWS, a.N - n0) - 1;

    f32x4 acc[F][G];
#pragma unroll
    for (int i = 0; i < F; i++)
#pragma unroll
        for (int j = 0; j < G; j++) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    // A thread carries the scale codes of row t of both operands, the first's rows
    // first (threads behind them repeat them: a branch here would keep the
    // compiler from ordering the multiplications among the loads), or of two rows.
    constexpr int SROWS = X::ROWS + W::ROWS, PER = (SROWS + THREADS - 1) / THREADS;
    static_assert(SROWS % THREADS == 0 || SROWS < THREADS, "the same rows per thread");
    struct Codes {
        uint64_t row[PER];
    };
    const uint8_t* srow[PER];
    char* splace[PER];
    int shalf[PER];
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int r = (t + i * THREADS) % SROWS;
        const bool of_x = r < X::ROWS;
        srow[i] = of_x ? a.xs + (m0 + min(r, xlast)) * a.blocks : a.ws + (n0 + min(r - X::ROWS, wlast)) * a.blocks;
        splace[i] = &scales[0][0] + (of_x ? scale_place<WM, F>(r) : X::SCALES + scale_place<WN, G>(r - X::ROWS));
        shalf[i] = of_x ? WM * X::GROUPS * 256 : WN * W::GROUPS * 256;
    }
    auto put_scales = [&](const Codes& v, int half) {
#pragma unroll
        for (int i = 0; i < PER; i++)
#pragma unroll
            for (int b = 0; b < kStep; b++)
                splace[i][half * (X::SCALES + W::SCALES) + b / 4 * shalf[i] + b % 4 * 64] =
                    (char)(uint8_t)(v.row[i] >> (8 * b));
    };
    const uint8_t* const xc = a.xc + m0 * a.blocks * 16;
    const uint8_t* const wc = a.wc + n0 * a.blocks * 16;
    auto fetch = [&](auto tail, int s, auto half) {
        constexpr bool TAIL = decltype(tail)::value, ODD = decltype(half)::value != 0;
        fetch_codes<TAIL, THREADS, X::ROWS>(xc, xlast, a.blocks, s * kStep, ODD ? x1 : x0);
        fetch_codes<TAIL, THREADS, W::ROWS>(wc, wlast, a.blocks, s * kStep, ODD ? w1 : w0);
        Codes v;
#pragma unroll
        for (int i = 0; i < PER; i++) v.row[i] = fetch_scales<TAIL>(srow[i], a.blocks, s * kStep);
        __builtin_amdgcn_sched_barrier(0);         // on their way before the multiplications begin
        return v;
    };
    // A step is 2 G columns of F multiplications: the weight's 16 rows j, 128 k.
    // Operands are read EARLY columns ahead, so that LDS answers while the
    // matrix cores are busy; the barriers keep the compiler from gathering the reads.
    constexpr int EARLY = 3;
    auto multiply = [&](auto half) {
        constexpr bool ODD = decltype(half)::value != 0;
        const char* const sbase = scales[ODD];
        const int xr = (wm * 16 * F + lane % 16) * (16 * kStep), wr = (wn * 16 * G + lane % 16) * (16 * kStep);
        const int piece[2] = {(lane / 16 ^ lane % 8) * 16, ((4 + lane / 16) ^ lane % 8) * 16};
        i32x4 x[2][F], w[2 * G];
        int sx[2][X::GROUPS], sw[2][W::GROUPS];
        auto read_x = [&](auto k, auto i) {
            constexpr int K = decltype(k)::value, I = decltype(i)::value;
            x[K][I] = *(const i32x4*)((ODD ? x1 : x0) + (xr + I * (16 * 16 * kStep) + piece[K]));
        };
        auto read_w = [&](auto c) {
            constexpr int C = decltype(c)::value;
            w[C] = *(const i32x4*)((ODD ? w1 : w0) + (wr + C % G * (16 * 16 * kStep) + piece[C / G]));
        };
#pragma unroll
        for (int k = 0; k < 2; k++) {
#pragma unroll
            for (int i = 0; i < X::GROUPS; i++)
                sx[k][i] = *(const int*)(sbase + ((k * WM + wm) * X::GROUPS + i) * 256 + lane * 4);
#pragma unroll
            for (int j = 0; j < W::GROUPS; j++)
                sw[k][j] = *(const int*)(sbase + X::SCALES + ((k * WN + wn) * W::GROUPS + j) * 256 + lane * 4);
        }
        static_for<F>([&](auto i) { read_x(Const<0>{}, i); });
        static_for<EARLY>([&](auto c) { read_w(c); });
        __builtin_amdgcn_sched_barrier(0);
        static_for<2 * G>([&](auto c) {
            constexpr int C = decltype(c)::value, K = C / G, J = C % G;
            if constexpr (C + EARLY < 2 * G) read_w(Const<C + EARLY>{});
            // the second half's rows of x, spread over the first half's last columns
            if constexpr (C < G)
                static_for<F>([&](auto i) {
                    if constexpr (decltype(i)::value * G / F / 2 + G / 2 == C) read_x(Const<1>{}, i);
                });
            static_for<F>([&](auto ci) {
                constexpr int I = decltype(ci)::value;
                acc[I][J] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(w[C]), operand(x[K][I]), acc[I][J], 4, 4,
                                                                            J % 4, sw[K][J / 4], I % 4, sx[K][I / 4]);
            });
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // What a wave has fetched to LDS is there: a barrier alone does not wait for
    // loads that are under way.  The scales, fetched behind the codes, have been
    // waited for before, so this costs nothing.
    auto arrived = [] {
        __builtin_amdgcn_s_waitcnt(kVmcnt0);
        __syncthreads();
    };
    // Whole steps of this part of K, two at a time, one for each half of LDS;
    // behind the last one it is fetched again, into memory that nobody reads any more.
    const int all = a.blocks / kStep, share = (all + gridDim.y - 1) / gridDim.y;
    const int end = min(all, share * ((int)blockIdx.y + 1));
    int s = min(all, share * (int)blockIdx.y);
    if (s < end) put_scales(fetch(Const<false>{}, s, Const<0>{}), 0);
    for (; s + 1 < end; s += 2) {
        arrived();                                 // step s has arrived; nobody reads the other half
        Codes sc = fetch(Const<false>{}, s + 1, Const<1>{});
        multiply(Const<0>{});
        put_scales(sc, 1);
        arrived();
        sc = fetch(Const<false>{}, min(s + 2, end - 1), Const<0>{});
        multiply(Const<1>{});
        put_scales(sc, 0);
    }
    arrived();
    if (s < end) multiply(Const<0>{});
    if (all * kStep < a.blocks && blockIdx.y + 1 == gridDim.y) {
        put_scales(fetch(Const<true>{}, all, Const<1>{}), 1);
        arrived();
        multiply(Const<1>{});
    }
    // Rows leave through LDS, each wave its own part in strips of 16 rows, as
    // pieces of 16 bytes along a row: whole lines per store.
    constexpr int E = 16 / (int)sizeof(T), PITCH = 16 * G + E;
    constexpr int SHARE = (WM * WN + 3) / 4;       // waves per LDS object
    static_assert(SHARE * 16 * PITCH * sizeof(T) <= X::CODES && X::CODES == W::CODES, "a strip per wave");
    __syncthreads();
    char* const part = wave / SHARE < 2 ? (wave / SHARE == 0 ? x0 : x1) : (wave / SHARE == 2 ? w0 : w1);
    T* const strip_at = (T*)part + wave % SHARE * 16 * PITCH;
    // a part of K: float32 sums, no bias (launched with T = float)
    T* const out = a.parts ? (T*)a.parts + (int64_t)blockIdx.y * a.M * a.N : (T*)a.out;
    const int64_t ostride = a.parts ? a.N : a.stride;
    const int64_t wm0 = m0 + wm * 16 * F, wn0 = n0 + wn * 16 * G;
    float bias[G][4];
#pragma unroll
    for (int j = 0; j < G; j++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const int64_t n = wn0 + j * 16 + lane / 16 * 4 + r;
            bias[j][r] = a.bias && n < a.N ? a.bias[n] : 0.f;
        }
#pragma unroll
    for (int i = 0; i < F; i++) {
#pragma unroll
        for (int j = 0; j < G; j++) {
            float y[4];
#pragma unroll
            for (int r = 0; r < 4; r++) y[r] = finish(acc[i][j][r], bias[j][r], a.relu);
            Vec<T, 4>::store(strip_at + lane % 16 * PITCH + j * 16 + lane / 16 * 4, y);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        constexpr int PER_ROW = 16 * G / E, ROUNDS = (16 * PER_ROW + kWave - 1) / kWave;
#pragma unroll
        for (int q = 0; q < ROUNDS; q++) {
            const int at = q * kWave + lane, row = at / PER_ROW, c = at % PER_ROW * E;
            const int64_t m = wm0 + i * 16 + row, n = wn0 + c;
            if (row >= 16 || m >= a.M || n >= a.N) continue;
            T* to = out + m * ostride + n;
            const T* from = strip_at + row * PITCH + c;
            if (n + E <= a.N) {
                typedef typename Vec<T, E>::type Piece;
                const Piece v = *(const Piece*)from;
                if (a.nt) __builtin_nontemporal_store(v, (Piece*)to);
                else *(Piece*)to = v;
            } else {
                for (int e = 0; n + e < a.N; e++) to[e] = from[e];
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// out = act(sum of the parts, in order, + bias).
template <typename T>
__global__ __launch_bounds__(kBlock) void k_mx4_join(MxArgs a, int parts) {
    const int64_t total = a.M * a.N, step = (int64_t)gridDim.x * kBlock * 4;
    for (int64_t i = ((int64_t)blockIdx.x * kBlock + threadIdx.x) * 4; i < total; i += step) {
        const int64_t m = i / a.N, n = i % a.N;
        const int count = (int)min((int64_t)4, total - i);
        float y[4] = {0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < parts; p++) {
            const float* from = a.parts + p * total + i;
            if (count == 4) {
                float v[4];
                Vec<float, 4>::load(from, v);
#pragma unroll
                for (int e = 0; e < 4; e++) y[e] += v[e];
            } else {
                for (int e = 0; e < count; e++) y[e] += from[e];
            }
        }
        if (n + 4 <= a.N) {                        // all in one row
#pragma unroll
            for (int e = 0; e < 4; e++) y[e] = finish(y[e], a.bias ? a.bias[n + e] : 0.f, a.relu);
            Vec<T, 4>::store((T*)a.out + m * a.stride + n, y);
        } else {
            for (int e = 0; e < count; e++) {
                const int64_t mm = (i + e) / a.N, nn = (i + e) % a.N;
                ((T*)a.out)[mm * a.stride + nn] = from_float<T>(finish(y[e], a.bias ? a.bias[nn] : 0.f, a.relu));
            }
        }
    }
}

// ----------------------------------------------------------------- few rows

// Up to 16 Q rows of x, Q = 1 or 2: the weight is read once and bounds the product.  A
// workgroup computes 16 columns of out; its waves take the steps of 256 k (a
// cache line of every row of the weight) in turn and join their sums in LDS.
// Every lane's operand is one 16-byte load, a step ahead of its use.  S is the
// type of x's elements, which the workgroup quantises into LDS first (for one
// row of 4096 to 4096 columns 10 us in all, 14 with a launch for it), or
// uint8_t: x is quantised already.
template <typename S> struct FewRows {
    const S* x;
    int64_t stride;                                // of float rows
    const uint8_t* xs;                             // scale codes of quantised rows
    int64_t cols;
};

template <typename S, typename T, int Q>
__global__ __launch_bounds__(1024) void k_mx4_few(MxArgs a, FewRows<S> f) {
    constexpr bool QUANTISED = std::is_same<S, uint8_t>::value;
    __shared__ f32x4 sums[16][Q][kWave];
    extern __shared__ uint4 own_rows[];            // codes, then scale codes, of x
    const int lane = lane_id(), wave = wave_id(), waves = blockDim.x / kWave;
    const int64_t n0 = (int64_t)blockIdx.x * 16, n = n0 + lane % 16;
    f32x4 acc[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) acc[q] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int64_t wrow = min(n, a.N - 1) * a.blocks;           // columns behind the last are not stored
    struct Weight {
        i32x4 w[2];
        int s[2];
    };
    auto load_w = [&](int b0) {
        Weight v = {{{0, 0, 0, 0}, {0, 0, 0, 0}}, {127, 127}};
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const int b = b0 + k * 4 + lane / 16;
            if (b < a.blocks) {
                v.w[k] = *(const i32x4*)(a.wc + 16 * (wrow + b));
                v.s[k] = a.ws[wrow + b];
            }
        }
        return v;
    };
    Weight next = load_w(wave * 8);
    const uint8_t *xc, *xs;
    if constexpr (QUANTISED) {
        xc = f.x;
        xs = f.xs;
    } else {
        uint8_t* const codes = (uint8_t*)own_rows;
        uint8_t* const scales = codes + a.M * a.blocks * 16;
        const int per_row = a.blocks * 4, pieces = (int)a.M * per_row;
        for (int i = threadIdx.x; i < pieces; i += blockDim.x) {        // a block's four pieces in adjacent lanes
            float v[8];
            load8<S>(f.x + (int64_t)(i / per_row) * f.stride, (int64_t)(i % per_row) * 8, f.cols, v);
            uint32_t top = top_bits(v);
            top = max(top, __float_as_uint(lane_pair<1>(__uint_as_float(top))));
            top = max(top, __float_as_uint(lane_pair<2>(__uint_as_float(top))));
            const int code = scale_code(top);
            *(uint32_t*)(codes + 4 * i) = to_codes(v, code);
            if (i % 4 == 0) scales[i / 4] = (uint8_t)code;
        }
        __syncthreads();
        xc = codes;
        xs = scales;
    }
    for (int b0 = wave * 8; b0 < a.blocks; b0 += waves * 8) {
        const Weight w = next;
        next = load_w(b0 + waves * 8);
        i32x4 x[2][Q] = {};
        int sx[2][Q];
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const int b = b0 + k * 4 + lane / 16;
#pragma unroll
            for (int q = 0; q < Q; q++) {
                const int64_t m = q * 16 + lane % 16;
                sx[k][q] = 127;
                if (b < a.blocks && m < a.M) {
                    x[k][q] = *(const i32x4*)(xc + 16 * (m * a.blocks + b));
                    sx[k][q] = xs[m * a.blocks + b];
                }
            }
        }
#pragma unroll
        for (int k = 0; k < 2; k++)
#pragma unroll
            for (int q = 0; q < Q; q++)
                acc[q] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(w.w[k]), operand(x[k][q]), acc[q], 4, 4, 0,
                                                                         w.s[k], 0, sx[k][q]);
    }
#pragma unroll
    for (int q = 0; q < Q; q++) sums[wave][q][lane] = acc[q];
    __syncthreads();
    for (int q = wave; q < Q; q += waves) {
        f32x4 y = sums[0][q][lane];
        for (int v = 1; v < waves; v++) {
            const f32x4 z = sums[v][q][lane];
#pragma unroll
            for (int r = 0; r < 4; r++) y[r] += z[r];
        }
        const int64_t m = q * 16 + lane % 16, c = n0 + lane / 16 * 4;
        if (m >= a.M) continue;
        T* const to = (T*)a.out + m * a.stride + c;
        float o[4];
#pragma unroll
        for (int r = 0; r < 4; r++) o[r] = finish(y[r], a.bias && c + r < a.N ? a.bias[c + r] : 0.f, a.relu);
        if (c + 4 <= a.N) {
            Vec<T, 4>::store(to, o);
        } else {
#pragma unroll
            for (int r = 0; r < 4; r++)
                if (c + r < a.N) to[r] = from_float<T>(o[r]);
        }
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

void mx4_quantize(const agnes_matrix* x, const agnes_mx4* q, hipStream_t st) {
    check_matrix(x, false, "x");
    check_mx4(q, "q");
    AGNES_REQUIRE(q->rows == x->rows && q->cols == x->cols, AGNES_ERR_INVALID, "x and q must have equal shapes");
    const int64_t blocks = mx_blocks(x->cols), per_row = blocks * 4;
    if (x->rows == 0 || per_row == 0) return;
    with_float(x->dtype, [&](auto t) {
        typedef decltype(t) T;
        launch_pieces(x->rows, per_row, [&](int64_t r, int64_t pieces, unsigned groups) {
            AGNES_LAUNCH((k_mx4_quantize<T>), dim3(groups), dim3(kBlock), 0, st, (const T*)x->data + r * x->stride,
                         x->stride, pieces, x->cols, (uint32_t)per_row, q->codes + r * blocks * 16,
                         q->scales + r * blocks);
        });
    });
}

void mx4_dequantize(const agnes_mx4* q, const agnes_matrix* x, hipStream_t st) {
    check_matrix(x, true, "x");
    check_mx4(q, "q");
    AGNES_REQUIRE(q->rows == x->rows && q->cols == x->cols, AGNES_ERR_INVALID, "x and q must have equal shapes");
    const int64_t blocks = mx_blocks(x->cols), per_row = blocks * 4;
    if (x->rows == 0 || per_row == 0) return;
    with_float(x->dtype, [&](auto t) {
        typedef decltype(t) T;
        launch_pieces(x->rows, per_row, [&](int64_t r, int64_t pieces, unsigned groups) {
            AGNES_LAUNCH((k_mx4_dequantize<T>), dim3(groups), dim3(kBlock), 0, st, q->codes + r * blocks * 16,
                         q->scales + r * blocks, pieces, x->cols, (uint32_t)per_row, (T*)x->data + r * x->stride,
                         x->stride, x->rows * x->cols * (int64_t)sizeof(T) > kStreamBytes);
        });
    });
}

constexpr int64_t kFullGrid = 256;                 // workgroups that fill the chip
constexpr int64_t kPartGrid = 512;                 // and that parts of K aim at
constexpr int64_t kPartSteps = 4;                  // fewest steps of a part

static void check_sizes(int64_t M, int64_t N, int64_t K) {
    for (int64_t v : {M, N, K})
        AGNES_REQUIRE(v >= 0 && v < ((int64_t)1 << 31), AGNES_ERR_INVALID, "M, N and K must be in [0, 2^31)");
    // a tile's rows are addressed with 32 bits
    AGNES_REQUIRE(K <= ((int64_t)1 << 24), AGNES_ERR_INVALID, "K must be at most 2^24");
}

// Which kernel computes M x N x K, by sizes alone.
// k_mx4_few reads x again for every 16 columns of out, and a workgroup's steps
// follow each other, so more than one 16-row tile pays only while rows x K x
// rounds of workgroups is small.  us, k_mx4_few against tiles with K in parts, of
// N x K: 32 rows of 4096 x 4096 7.8 / 9.5, of 8192 x 1000 4.9 / 4.8, of 256 x 2048 4.9 / 7.3;
// 17 rows of 8192 x 8192 18.8 / 14.0, of 1024 x 8192 9.8 / 9.2; 64 rows of 4096 x
// 4096 11.5 / 10.6, of 8192 x 8192 40 / 16, of 8192 x 1000 7.0 / 4.9.
constexpr int64_t kFewTile = 16;                   // rows of k_mx4_few, whatever the sizes,
constexpr int64_t kFewRows = 32;                   // and at most, as long as
constexpr int64_t kFewWork = 1 << 17;              // rows x K x rounds is no more than this
constexpr int64_t kFewQuantize = 16;               // and rows that it quantises itself,
constexpr int64_t kFewBytes = 40 << 10;            // if they take no more LDS than this
static int64_t few_lds(int64_t M, int64_t blocks) { return M * blocks * 17; }
struct MxPlan {
    int rows, cols;                                // of a tile; 0: k_mx4_few
    int parts;                                     // of K
};

// Refuses what one launch cannot hold (2^32 threads), so that callers do before
// they enqueue anything: a tile has at most 512 threads, and their number is
// rounded up to one for each XCD.
static MxPlan plan_product(int64_t M, int64_t N, int64_t K) {
    auto fits = [](MxPlan p, int64_t tiles) {
        AGNES_REQUIRE(tiles <= (1 << 23) - kXcds, AGNES_ERR_RANGE, "the product has too many tiles");
        return p;
    };
    const int64_t rounds = (N + 16 * kFullGrid - 1) / (16 * kFullGrid);
    if (M <= kFewTile || (M <= kFewRows && K <= kFewWork && M * K * rounds <= kFewWork))
        return fits({0, 0, 1}, (N + 15) / 16);
    // the largest tile that still gives every compute unit one (8192^3: 305 us in
    // tiles of 256, 407 in tiles of 128)
    auto tiles = [&](int64_t r) { return ((M + r - 1) / r) * ((N + r - 1) / r); };
    for (int r : {256, 128})
        if (tiles(r) >= kFullGrid) return fits({r, r, 1}, tiles(r));
    // else small tiles, and K in parts of at least kPartSteps steps
    const int64_t steps = mx_blocks(K) / kStep;
    const int64_t parts = std::min<int64_t>(kPartGrid / tiles(64), steps / kPartSteps);
    return {64, 64, (int)std::max<int64_t>(1, parts)};
}

uint64_t mx4_product_bytes(int64_t M, int64_t N, int64_t K) {
    check_sizes(M, N, K);
    if (M == 0 || N == 0) return 0;
    const MxPlan p = plan_product(M, N, K);
    return p.parts > 1 ? (uint64_t)(p.parts * M * N) * 4 : 0;
}

uint64_t mx4_linear_bytes(int64_t M, int64_t N, int64_t K) {
    check_sizes(M, N, K);
    Carve c(nullptr);
    c.take<uint8_t>(M * mx_blocks(K) * 16);
    c.take<uint8_t>(M * mx_blocks(K));
    return c.used + mx4_product_bytes(M, N, K);
}

template <typename T, int WM, int WN, int F, int G> static void launch_tile(const MxArgs& a, int parts, hipStream_t st) {
    constexpr int R = MxSide<WM, F>::ROWS, C = MxSide<WN, G>::ROWS;
    const int64_t tiles = ((a.M + R - 1) / R) * ((a.N + C - 1) / C);
    const unsigned grid = (unsigned)((tiles + kXcds - 1) / kXcds * kXcds);
    AGNES_LAUNCH((k_mx4_gemm<T, WM, WN, F, G>), dim3(grid, (unsigned)parts), dim3(kWave * WM * WN), 0, st, a);
}

template <typename T> static void launch_gemm(const MxPlan& p, const MxArgs& a, hipStream_t st) {
    if (p.rows == 256) launch_tile<T, 2, 4, 8, 4>(a, p.parts, st);
    else if (p.rows == 128) launch_tile<T, 2, 2, 4, 4>(a, p.parts, st);
    else launch_tile<T, 2, 2, 2, 2>(a, p.parts, st);
}

template <typename S, typename T> static void launch_few(const MxArgs& a, const FewRows<S>& f, hipStream_t st) {
    const int64_t groups = (a.N + 15) / 16;
    // more waves where there are few workgroups, but a step for each; above 512
    // workgroups at most 512 threads
    const int steps = (a.blocks + 7) / 8;
    int waves = groups <= 512 ? 16 : 8;
    while (waves > 1 && waves / 2 >= steps) waves /= 2;
    const dim3 grid((unsigned)groups), block((unsigned)(waves * kWave));
    const size_t lds = std::is_same<S, uint8_t>::value ? 0 : (size_t)few_lds(a.M, a.blocks);
    if (a.M <= 16) AGNES_LAUNCH((k_mx4_few<S, T, 1>), grid, block, lds, st, a, f);
    else if constexpr (std::is_same<S, uint8_t>::value) {
        AGNES_LAUNCH((k_mx4_few<S, T, 2>), grid, block, 0, st, a, f);
    }
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
    check_workspace(ws, ws_bytes, mx4_product_bytes(M, N, x->cols));   // checks the sizes too
    if (M == 0 || N == 0) return;
    const MxPlan p = plan_product(M, N, x->cols);
    MxArgs a{x->codes, x->scales, w->codes, w->scales, M, N, (int32_t)blocks, bias, relu,
             M * N * (int64_t)elem_size(out->dtype) > kStreamBytes, out->data, out->stride, nullptr};
    with_float(out->dtype, [&](auto t) {
        typedef decltype(t) T;
        if (p.rows == 0) {
            launch_few<uint8_t, T>(a, FewRows<uint8_t>{x->codes, 0, x->scales, x->cols}, st);
        } else if (p.parts == 1) {
            launch_gemm<T>(p, a, st);
        } else {
            a.parts = (float*)ws;
            MxArgs sums = a;
            sums.bias = nullptr;
            sums.relu = sums.nt = false;
            launch_gemm<float>(p, sums, st);
            AGNES_LAUNCH((k_mx4_join<T>), dim3(grid_for((M * N + 3) / 4, 4096)), dim3(kBlock), 0, st, a, p.parts);
        }
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
    if (x->rows <= kFewQuantize && few_lds(x->rows, mx_blocks(x->cols)) <= kFewBytes) {
        const MxArgs a{nullptr, nullptr, w->codes, w->scales, x->rows, w->rows, (int32_t)mx_blocks(x->cols), bias, relu,
                       false, out->data, out->stride, nullptr};
        with_float(x->dtype, [&](auto ts) {
            with_float(out->dtype, [&](auto t) {
                typedef decltype(ts) S;
                typedef decltype(t) T;
                launch_few<S, T>(a, FewRows<S>{(const S*)x->data, x->stride, nullptr, x->cols}, st);
            });
        });
        return;
    }
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
