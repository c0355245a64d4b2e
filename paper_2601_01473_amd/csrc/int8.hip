// Rows in 8-bit integers with a scale each, back to values, and the product of
// two matrices in that form.
//
// With s_m and t_n the scales of x's and w's rows:
//   y[m][n] = (float)(sum_k a[m][k] b[n][k]) s_m t_n + bias[n]
// The sum is a whole number below 2^31 for K < 2^17, so it is exact in any order.
#include <algorithm>
#include <cmath>
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

__device__ __forceinline__ uint32_t lanes_top(uint32_t top, int L) {
    // as numbers without a sign they are ordered as float32 are, but NaN
    return __float_as_uint(lanes_reduce(__uint_as_float(top), L, [](float a, float b) {
        return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
    }));
}

// Eight codes as bytes, the first in the low bits.
__device__ __forceinline__ uint2 to_codes(const float (&x)[8], const Scale& s) {
    uint2 w = {0u, 0u};
    if (s.inv == 0.f) return w;
#pragma unroll
    for (int q = 0; q < 4; q++) {
        w.x |= (uint32_t)(to_code(x[q], s) & 255) << (8 * q);
        w.y |= (uint32_t)(to_code(x[q + 4], s) & 255) << (8 * q);
    }
    return w;
}

// A row is read once and stays in registers between its maximum and its codes:
// L lanes per row, P pieces of 8 elements per lane; L is at most a wave
// (THREADS = kWave) or the workgroup.  Bound by memory: 65536 x 1024 bfloat16 48
// us (4.2 TB/s), and back 29.5 us (6.8 TB/s).
template <typename T, int THREADS, int P>
__global__ __launch_bounds__(THREADS == kWave ? kBlock : THREADS)
void k_int8_quantize(const T* __restrict__ x, int64_t stride, int64_t rows, int64_t cols, int64_t pitch, int L,
                     int8_t* __restrict__ codes, float* __restrict__ scales) {
    constexpr bool WHOLE = THREADS != kWave;
    __shared__ uint32_t red[THREADS / kWave];
    const int gl = WHOLE ? threadIdx.x : threadIdx.x % L;
    const int64_t r = WHOLE ? blockIdx.x : (int64_t)blockIdx.x * (kBlock / L) + threadIdx.x / L;
    if (!WHOLE && r >= rows) return;
    const T* const row = x + r * stride;
    const int step = WHOLE ? THREADS : L;
    float v[P][8];
    uint32_t top = 0;
#pragma unroll
    for (int p = 0; p < P; p++) load8<T>(row, (int64_t)(gl + p * step) * 8, cols, v[p]);
#pragma unroll
    for (int p = 0; p < P; p++) top = max(top, top_bits(v[p]));
    top = lanes_top(top, WHOLE ? kWave : L);
    if (WHOLE) {
        if (lane_id() == 0) red[wave_id()] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / kWave; w++) top = max(top, red[w]);
    }
    const Scale s = row_scale(top);
    if (gl == 0) scales[r] = s.scale;
#pragma unroll
    for (int p = 0; p < P; p++) {
        const int64_t c = (int64_t)(gl + p * step) * 8;
        if (c < pitch) *(uint2*)(codes + r * pitch + c) = to_codes(v[p], s);
    }
}

// Longer rows are read twice.
template <typename T>
__global__ __launch_bounds__(1024) void k_int8_quantize_long(const T* __restrict__ x, int64_t stride, int64_t cols,
                                                            int64_t pitch, int8_t* __restrict__ codes,
                                                            float* __restrict__ scales) {
    __shared__ uint32_t red[1024 / kWave];
    const int64_t r = blockIdx.x;
    const T* const row = x + r * stride;
    uint32_t top = 0;
    for (int64_t c = threadIdx.x * 8; c < cols; c += 1024 * 8) {
        float v[8];
        load8<T>(row, c, cols, v);
        top = max(top, top_bits(v));
    }
    top = lanes_top(top, kWave);
    if (lane_id() == 0) red[wave_id()] = top;
    __syncthreads();
    for (int w = 0; w < 1024 / kWave; w++) top = max(top, red[w]);
    const Scale s = row_scale(top);
    if (threadIdx.x == 0) scales[r] = s.scale;
    for (int64_t c = threadIdx.x * 8; c < pitch; c += 1024 * 8) {
        float v[8];
        load8<T>(row, c, cols, v);
        *(uint2*)(codes + r * pitch + c) = to_codes(v, s);
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_int8_dequantize(const int8_t* __restrict__ codes,
                                                            const float* __restrict__ scales, int64_t pieces,
                                                            int64_t cols, uint32_t per_row, T* __restrict__ x,
                                                            int64_t stride, bool nt) {
    const int64_t base = (int64_t)blockIdx.x * (kBlock * kPieces);
    const int64_t base_row = base / per_row;
    const uint32_t base_piece = (uint32_t)(base % per_row);
    uint2 w[kPieces];
    float s[kPieces];
    PieceAt at[kPieces];
#pragma unroll
    for (int u = 0; u < kPieces; u++) {
        const uint32_t off = u * kBlock + threadIdx.x;
        if (base + off < pieces) {
            at[u] = piece_at(base_row, base_piece, off, per_row);
            w[u] = *(const uint2*)(codes + 8 * (base + off));
            s[u] = scales[at[u].row];
        }
    }
#pragma unroll
    for (int u = 0; u < kPieces; u++) {
        if (base + u * kBlock + threadIdx.x >= pieces) continue;
        float v[8];
#pragma unroll
        for (int q = 0; q < 4; q++) {
            v[q] = (float)(int8_t)(w[u].x >> (8 * q)) * s[u];
            v[q + 4] = (float)(int8_t)(w[u].y >> (8 * q)) * s[u];
        }
        T* const row = x + at[u].row * stride;
        const int64_t c = (int64_t)at[u].piece * 8;
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

// v_mfma_i32_16x16x64_i8: lane l holds 16 consecutive k (one chunk) of row l %
// 16 of either operand, k = 16 (l / 16); D[4 (l / 16) + r][l % 16].  The
// weight goes in first, so a lane holds four adjacent columns of a row of out.
struct Int8Args {
    const int8_t *xc, *wc;
    const float *xs, *ws;
    int64_t M, N;
    int32_t chunks;                                // per row
    const float* bias;
    bool relu, nt;
    void* out;
    int64_t stride;
    int32_t* parts;                                // [gridDim.y][M][N]: sums over parts of K instead of out, or NULL
};

__device__ __forceinline__ float finish(int sum, float s, float t, float bias, bool relu) {
    const float y = (float)sum * s * t + bias;
    return relu && y < 0.f ? 0.f : y;
}

// Sixteen zero bytes: chunks behind the last one of a row.
static __device__ const uint4 k_int8_zero = {0u, 0u, 0u, 0u};

// A workgroup of WM x WN waves computes a tile of out, a wave 16 F x 16 G of
// it, in steps of 64 k: one multiplication deep.  Codes go from memory straight
// to one of four images in LDS, three steps ahead of their use; a wave reads a
// step's operands into registers while it multiplies the step before.  An
// image: row after row, 4 chunks each, chunk p of row r at place p ^ (-(r / 4) % 4).
// LDS serves lanes 0-3, 12-15 and 20-27 of a wave together, and so on: these 16
// then lie in different banks.
//
// 8192^3: 431 us, 2550 TOPS (449 us on a slower card), the matrix cores busy two
// thirds of the cycles, at a clock that falls as they get busier (1.85 GHz): with
// 32 x 32 x 32 multiplications as many cycles take 493 us.  (Chunk p at place p ^ (r / 4 % 4), where
// lanes meet in pairs: as many us, so LDS does not bound it.)
constexpr int kStepChunks = 4, kImages = 4;
__device__ __forceinline__ int turn(int r) { return -(r / 4) & 3; }

// The weight's or x's rows of a step, a chunk per thread and round.  from[i]: the
// row of the thread's i-th chunk, at the chunk that it fetches in step 0.
template <int THREADS, int ROWS> struct Int8Side {
    static constexpr int ROUNDS = ROWS * kStepChunks / THREADS;
    const int8_t* from[ROUNDS];
    int chunk;                                     // within a step; the same for all rounds
    __device__ __forceinline__ Int8Side(const int8_t* codes, int64_t row0, int64_t rows, int chunks) {
        const int t = threadIdx.x, r = t / kStepChunks;
        chunk = t % kStepChunks ^ turn(r);         // rounds differ by a multiple of 16 rows
#pragma unroll
        for (int i = 0; i < ROUNDS; i++)           // rows behind the last repeat it: they are not stored
            from[i] = codes + min(row0 + r + i * (THREADS / kStepChunks), rows - 1) * ((int64_t)chunks * kChunk) +
                      chunk * kChunk;
    }
    template <int I> __device__ __forceinline__ void fetch(int step, int end, char* image) const {
        const int8_t* p = step * kStepChunks + chunk < end ? from[I] + (int64_t)step * (kStepChunks * kChunk)
                                                          : (const int8_t*)&k_int8_zero;
        char* const to = image + __builtin_amdgcn_readfirstlane(wave_id()) * (kWave * kChunk);
        __builtin_amdgcn_global_load_lds((global_void*)p, (lds_void*)(to + I * THREADS * kChunk), 16, 0, 0);
    }
};

template <typename T, int WM, int WN, int F, int G>
__global__ __launch_bounds__(kWave* WM* WN) void k_int8_gemm(Int8Args a) {
    constexpr int THREADS = kWave * WM * WN, ROWS = WM * 16 * F, COLS = WN * 16 * G, ROW = kStepChunks * kChunk;
    // An object per image and operand, addressed with constants: that way the
    // compiler sees that a fetch under way does not write what is being read, and
    // adds no wait of its own for it.
    __shared__ __attribute__((aligned(1024))) char x0[ROWS * ROW], x1[ROWS * ROW], x2[ROWS * ROW], x3[ROWS * ROW];
    __shared__ __attribute__((aligned(1024))) char w0[COLS * ROW], w1[COLS * ROW], w2[COLS * ROW], w3[COLS * ROW];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), wm = wave / WN, wn = wave % WN;
    // XCD x takes a contiguous run of tiles, in strips of 8 tile rows: the tiles
    // that run at once on it share rows of both operands in its L2.
    const int64_t tm = (a.M + ROWS - 1) / ROWS, tn = (a.N + COLS - 1) / COLS, tiles = tm * tn;
    const int64_t per = (tiles + kXcds - 1) / kXcds, id = blockIdx.x % kXcds * per + blockIdx.x / kXcds;
    if ((int64_t)blockIdx.x / kXcds >= per || id >= tiles) return;
    const int64_t strip = id / (8 * tn), high = min((int64_t)8, tm - strip * 8), in = id - strip * 8 * tn;
    const int64_t m0 = (strip * 8 + in % high) * ROWS, n0 = in / high * COLS;

    i32x4 acc[F][G];
#pragma unroll
    for (int i = 0; i < F; i++)
#pragma unroll
        for (int j = 0; j < G; j++) acc[i][j] = i32x4{0, 0, 0, 0};

    const Int8Side<THREADS, ROWS> xside(a.xc, m0, a.M, a.chunks);
    const Int8Side<THREADS, COLS> wside(a.wc, n0, a.N, a.chunks);
    constexpr int FETCHES = Int8Side<THREADS, ROWS>::ROUNDS + Int8Side<THREADS, COLS>::ROUNDS;   // per thread and step
    static_assert(FETCHES < 16, "what a wait can count here");
    auto xat = [&](auto s) -> char* { constexpr int S = decltype(s)::value % kImages; return S == 0 ? x0 : S == 1 ? x1 : S == 2 ? x2 : x3; };
    auto wat = [&](auto s) -> char* { constexpr int S = decltype(s)::value % kImages; return S == 0 ? w0 : S == 1 ? w1 : S == 2 ? w2 : w3; };
    // This part's steps; fetches behind its end bring zeros, so that every step has equally many.
    const int all = (a.chunks + kStepChunks - 1) / kStepChunks, share = (all + gridDim.y - 1) / gridDim.y;
    const int first = min(all, share * (int)blockIdx.y), steps = min(all, first + share) - first;
    const int end = min(a.chunks, (first + steps) * kStepChunks);
    constexpr int XROUNDS = Int8Side<THREADS, ROWS>::ROUNDS;
    auto fetch_one = [&](auto image, auto n, int s) {
        constexpr int I = decltype(n)::value;
        if constexpr (I < XROUNDS) xside.template fetch<I>(first + s, end, xat(image));
        else wside.template fetch<I - XROUNDS>(first + s, end, wat(image));
    };
    auto fetch = [&](auto image, int s) {
        static_for<FETCHES>([&](auto n) { fetch_one(image, n, s); });
    };
    i32x4 x[2][F], w[G];
    const int place = (lane / 16 ^ turn(lane % 16)) * kChunk;
    const int xr = (wm * 16 * F + lane % 16) * ROW + place, wr = (wn * 16 * G + lane % 16) * ROW + place;
    auto read_x = [&](auto s, auto i) {
        constexpr int S = decltype(s)::value, I = decltype(i)::value;
        x[S % 2][I] = *(const i32x4*)(xat(s) + (xr + I * 16 * ROW));
    };
    auto read_w = [&](auto s, auto j) {
        constexpr int J = decltype(j)::value;
        w[J] = *(const i32x4*)(wat(s) + (wr + J * 16 * ROW));
    };
    // Waits until this wave's fetches, but the LATER last steps' ones, are in LDS, then for all waves.
    auto arrived = [](auto later) {
        __builtin_amdgcn_s_waitcnt(kVmcnt0 | (decltype(later)::value * FETCHES));
        asm volatile("" ::: "memory");             // the compiler moves no access to LDS across the barrier
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    static_assert(2 * FETCHES < 16, "what a wait can count here");
    fetch(Const<0>{}, 0);
    fetch(Const<1>{}, 1);
    fetch(Const<2>{}, 2);
    arrived(Const<2>{});
    static_for<F>([&](auto i) { read_x(Const<0>{}, i); });
    static_for<G>([&](auto j) { read_w(Const<0>{}, j); });
    // Step s: its operands are in registers.  Behind the barrier step s + 1 is in
    // LDS, and nobody reads the image of step s - 1 any more: what was read
    // from it has been multiplied.
    auto step = [&](auto image, int s) {
        constexpr int S = decltype(image)::value;
        arrived(Const<1>{});
        static_for<G>([&](auto cj) {
            constexpr int J = decltype(cj)::value;
            static_for<F>([&](auto i) {
                if constexpr (decltype(i)::value * G / F == J) read_x(Const<S + 1>{}, i);
            });
            static_for<F>([&](auto ci) {
                constexpr int I = decltype(ci)::value;
                acc[I][J] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[J], x[S % 2][I], acc[I][J], 0, 0, 0);
            });
            read_w(Const<S + 1>{}, cj);
            // fetches spread over the columns: at the step's start all waves would
            // queue for the address units before their first multiplication
            // (8192^3: 460 us, 431 so)
            static_for<FETCHES>([&](auto n) {
                if constexpr (decltype(n)::value * G / FETCHES == J) fetch_one(Const<S + 3>{}, n, s + 3);
            });
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    for (int s = 0; s < steps; s += kImages)       // steps behind the last one multiply zeros
        static_for<kImages>([&](auto i) { step(i, s + decltype(i)::value); });
    __builtin_amdgcn_s_waitcnt(kVmcnt0);           // the last fetches, before LDS is used again
    __syncthreads();
    // Rows leave through LDS, each wave its own part in strips of 16 rows, as
    // pieces of 16 bytes along a row: whole lines per store.
    constexpr int E = 16 / (int)sizeof(T), PITCH = 16 * G + E;
    constexpr int SHARE = (WM * WN + 3) / 4;       // waves per LDS object
    static_assert(SHARE * 16 * PITCH * sizeof(T) <= ROWS * ROW && ROWS == COLS, "a strip per wave");
    char* const part = wave / SHARE < 2 ? (wave / SHARE == 0 ? x0 : x1) : (wave / SHARE == 2 ? w0 : w1);
    T* const strip_at = (T*)part + wave % SHARE * 16 * PITCH;
    // a part of K: the sums (launched with T = int32_t)
    T* const out = a.parts ? (T*)a.parts + (int64_t)blockIdx.y * a.M * a.N : (T*)a.out;
    const int64_t ostride = a.parts ? a.N : a.stride;
    const int64_t wm0 = m0 + wm * 16 * F, wn0 = n0 + wn * 16 * G;
    float bias[G][4], ws[G][4], xs[F];
    if constexpr (!std::is_same<T, int32_t>::value) {
#pragma unroll
        for (int j = 0; j < G; j++)
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const int64_t n = wn0 + j * 16 + lane / 16 * 4 + r;
                bias[j][r] = a.bias && n < a.N ? a.bias[n] : 0.f;
                ws[j][r] = n < a.N ? a.ws[n] : 0.f;
            }
#pragma unroll
        for (int i = 0; i < F; i++) {
            const int64_t m = wm0 + i * 16 + lane % 16;
            xs[i] = m < a.M ? a.xs[m] : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < F; i++) {
#pragma unroll
        for (int j = 0; j < G; j++) {
            T* const to = strip_at + lane % 16 * PITCH + j * 16 + lane / 16 * 4;
            if constexpr (std::is_same<T, int32_t>::value) {
                *(i32x4*)to = acc[i][j];
            } else {
                float y[4];
#pragma unroll
                for (int r = 0; r < 4; r++) y[r] = finish(acc[i][j][r], xs[i], ws[j][r], bias[j][r], a.relu);
                Vec<T, 4>::store(to, y);
            }
        }
        wave_sync();
        constexpr int PER_ROW = 16 * G / E, ROUNDS = (16 * PER_ROW + kWave - 1) / kWave;
#pragma unroll
        for (int q = 0; q < ROUNDS; q++) {
            const int at = q * kWave + lane, row = at / PER_ROW, c = at % PER_ROW * E;
            const int64_t m = wm0 + i * 16 + row, n = wn0 + c;
            if (row >= 16 || m >= a.M || n >= a.N) continue;
            T* to = out + m * ostride + n;
            const T* from = strip_at + row * PITCH + c;
            if (n + E <= a.N) {
                typedef T Piece __attribute__((ext_vector_type(E), aligned(sizeof(T))));
                const Piece v = *(const Piece*)from;
                if (a.nt) __builtin_nontemporal_store(v, (Piece*)to);
                else *(Piece*)to = v;
            } else {
                for (int e = 0; n + e < a.N; e++) to[e] = from[e];
            }
        }
        wave_sync();
    }
}

// out from the sum of the parts.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_int8_join(Int8Args a, int parts) {
    const int64_t total = a.M * a.N, step = (int64_t)gridDim.x * kBlock * 4;
    for (int64_t i = ((int64_t)blockIdx.x * kBlock + threadIdx.x) * 4; i < total; i += step) {
        const int64_t m = i / a.N, n = i % a.N;
        const int count = (int)min((int64_t)4, total - i);
        int y[4] = {0, 0, 0, 0};
        for (int p = 0; p < parts; p++) {
            const int32_t* from = a.parts + p * total + i;
            if (count == 4) {
                typedef int Four __attribute__((ext_vector_type(4), aligned(4)));
                const Four v = *(const Four*)from;
#pragma unroll
                for (int e = 0; e < 4; e++) y[e] += v[e];
            } else {
                for (int e = 0; e < count; e++) y[e] += from[e];
            }
        }
        if (n + 4 <= a.N) {                        // all in one row
            float o[4];
#pragma unroll
            for (int e = 0; e < 4; e++) o[e] = finish(y[e], a.xs[m], a.ws[n + e], a.bias ? a.bias[n + e] : 0.f, a.relu);
            Vec<T, 4>::store((T*)a.out + m * a.stride + n, o);
        } else {
            for (int e = 0; e < count; e++) {
                const int64_t mm = (i + e) / a.N, nn = (i + e) % a.N;
                ((T*)a.out)[mm * a.stride + nn] =
                    from_float<T>(finish(y[e], a.xs[mm], a.ws[nn], a.bias ? a.bias[nn] : 0.f, a.relu));
            }
        }
    }
}

// ----------------------------------------------------------------- few rows

// Up to 16 Q rows of x, Q = 1 or 2: the weight is read once and bounds the
// product.  A workgroup computes 16 columns of out; its waves take the steps of
// 128 k (a cache line of every row of the weight) in turn and join their sums in
// LDS.  S is the type of x's elements, up to 16 rows of which the workgroup
// quantises into LDS first (a launch less), or int8_t: x is quantised already.
// (One row of 4096 x 4096: 5.9 us quantised before, 7.4 us in all.)
template <typename S> struct Int8Rows {
    const S* x;
    int64_t stride;                                // of float rows
    int64_t cols;
};
constexpr int kFewDepth = 2;                       // steps whose weight is on its way

template <typename S, typename T, int Q>
__global__ __launch_bounds__(1024) void k_int8_few(Int8Args a, Int8Rows<S> f) {
    constexpr bool QUANTISED = std::is_same<S, int8_t>::value;
    __shared__ i32x4 sums[16][Q][kWave];
    __shared__ uint32_t tops[16][16];
    __shared__ float own_scales[16];
    extern __shared__ uint4 own_rows[];            // codes of x
    const int lane = lane_id(), wave = wave_id(), waves = blockDim.x / kWave;
    const int64_t n0 = (int64_t)blockIdx.x * 16, n = n0 + lane % 16;
    i32x4 acc[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) acc[q] = i32x4{0, 0, 0, 0};
    const int8_t* const wrow = a.wc + min(n, a.N - 1) * ((int64_t)a.chunks * kChunk);   // columns behind the last are not stored
    struct Weight {
        i32x4 w[2];
    };
    auto load_w = [&](int c0) {
        Weight v = {{{0, 0, 0, 0}, {0, 0, 0, 0}}};
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const int c = c0 + k * 4 + lane / 16;
            if (c < a.chunks) v.w[k] = *(const i32x4*)(wrow + (int64_t)c * kChunk);
        }
        return v;
    };
    Weight ring[kFewDepth];
#pragma unroll
    for (int d = 0; d < kFewDepth; d++) ring[d] = load_w((wave + d * waves) * 8);
    const int8_t* xc;
    const float* xs;
    if constexpr (QUANTISED) {
        xc = f.x;
        xs = a.xs;
    } else {
        // `each` waves to a row (a power of two, as their number is)
        int8_t* const codes = (int8_t*)own_rows;
        int each = waves;
        while (each > 1 && each * a.M > waves) each /= 2;
        const int pieces = a.chunks * 2, at_once = waves / each;
        for (int r0 = 0; r0 < a.M; r0 += at_once) {
            const int r = r0 + wave / each, sub = wave % each;
            const S* const row = f.x + (int64_t)r * f.stride;
            uint32_t top = 0;
            if (r < a.M)
                for (int p = sub * kWave + lane; p < pieces; p += each * kWave) {
                    float v[8];
                    load8<S>(row, (int64_t)p * 8, f.cols, v);
                    top = max(top, top_bits(v));
                }
            top = lanes_top(top, kWave);
            if (lane == 0) tops[wave / each][sub] = top;
            __syncthreads();
            if (r < a.M) {
                for (int e = 0; e < each; e++) top = max(top, tops[wave / each][e]);
                const Scale s = row_scale(top);
                if (sub == 0 && lane == 0) own_scales[r] = s.scale;
                for (int p = sub * kWave + lane; p < pieces; p += each * kWave) {
                    float v[8];
                    load8<S>(row, (int64_t)p * 8, f.cols, v);
                    *(uint2*)(codes + ((int64_t)r * a.chunks * 2 + p) * 8) = to_codes(v, s);
                }
            }
            __syncthreads();
        }
        xc = codes;
        xs = own_scales;
    }
    auto multiply = [&](const Weight& w, int c0) {
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const int c = c0 + k * 4 + lane / 16;
#pragma unroll
            for (int q = 0; q < Q; q++) {
                const int64_t m = q * 16 + lane % 16;
                i32x4 x = {0, 0, 0, 0};
                if (c < a.chunks && m < a.M) x = *(const i32x4*)(xc + (m * a.chunks + c) * kChunk);
                acc[q] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w.w[k], x, acc[q], 0, 0, 0);
            }
        }
    };
    for (int c0 = wave * 8; c0 < a.chunks; c0 += kFewDepth * waves * 8) {
#pragma unroll
        for (int d = 0; d < kFewDepth; d++) {
            const Weight w = ring[d];
            ring[d] = load_w(c0 + (kFewDepth + d) * waves * 8);
            multiply(w, c0 + d * waves * 8);       // zeros behind the row's end
        }
    }
#pragma unroll
    for (int q = 0; q < Q; q++) sums[wave][q][lane] = acc[q];
    __syncthreads();
    for (int q = wave; q < Q; q += waves) {
        i32x4 y = sums[0][q][lane];
        for (int v = 1; v < waves; v++) y += sums[v][q][lane];
        const int64_t m = q * 16 + lane % 16, c = n0 + lane / 16 * 4;
        if (m >= a.M) continue;
        T* const to = (T*)a.out + m * a.stride + c;
        const float s = xs[m];
        float o[4];
#pragma unroll
        for (int r = 0; r < 4; r++)
            o[r] = c + r < a.N ? finish(y[r], s, a.ws[c + r], a.bias ? a.bias[c + r] : 0.f, a.relu) : 0.f;
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

template <typename T, int THREADS, int P>
static void launch_quantize(const agnes_matrix* x, const agnes_int8* q, int64_t pitch, int L, hipStream_t st) {
    const int64_t per = THREADS == kWave ? kBlock / L : 1, most = kLaunchRows * per;
    for (int64_t r = 0; r < x->rows; r += most) {
        const int64_t n = std::min(most, x->rows - r);
        AGNES_LAUNCH((k_int8_quantize<T, THREADS, P>), dim3((unsigned)((n + per - 1) / per)),
                     dim3(THREADS == kWave ? kBlock : THREADS), 0, st, (const T*)x->data + r * x->stride, x->stride, n,
                     x->cols, pitch, L, q->codes + r * pitch, q->scales + r);
    }
}

void int8_quantize(const agnes_matrix* x, const agnes_int8* q, hipStream_t st) {
    check_matrix(x, false, "x");
    check_int8(q, "q");
    AGNES_REQUIRE(q->rows == x->rows && q->cols == x->cols, AGNES_ERR_INVALID, "x and q must have equal shapes");
    const int64_t pitch = chunks_of(x->cols) * kChunk, pieces = pitch / 8;
    with_float(x->dtype, [&](auto t) {
        typedef decltype(t) T;
        if (pieces <= 4 * kWave) {
            int L = 8;
            while (L * 4 < pieces) L *= 2;
            if (pieces <= L) launch_quantize<T, kWave, 1>(x, q, pitch, L, st);
            else if (pieces <= 2 * L) launch_quantize<T, kWave, 2>(x, q, pitch, L, st);
            else launch_quantize<T, kWave, 4>(x, q, pitch, L, st);
        } else if (pieces <= 2 * 256) {
            launch_quantize<T, 256, 2>(x, q, pitch, 0, st);
        } else if (pieces <= 4 * 256) {
            launch_quantize<T, 256, 4>(x, q, pitch, 0, st);
        } else if (pieces <= 4 * 1024) {
            launch_quantize<T, 1024, 4>(x, q, pitch, 0, st);
        } else {
            for (int64_t r = 0; r < x->rows; r += kLaunchRows)
                AGNES_LAUNCH((k_int8_quantize_long<T>), dim3((unsigned)std::min(kLaunchRows, x->rows - r)), dim3(1024), 0, st,
                             (const T*)x->data + r * x->stride, x->stride, x->cols, pitch, q->codes + r * pitch,
                             q->scales + r);
        }
    });
}

void int8_dequantize(const agnes_int8* q, const agnes_matrix* x, hipStream_t st) {
    check_matrix(x, true, "x");
    check_int8(q, "q");
    AGNES_REQUIRE(q->rows == x->rows && q->cols == x->cols, AGNES_ERR_INVALID, "x and q must have equal shapes");
    const int64_t chunks = chunks_of(x->cols), per_row = chunks * 2;
    if (x->rows == 0 || x->cols == 0) return;
    with_float(x->dtype, [&](auto t) {
        typedef decltype(t) T;
        launch_pieces(x->rows, per_row, [&](int64_t r, int64_t pieces, unsigned groups) {
            AGNES_LAUNCH((k_int8_dequantize<T>), dim3(groups), dim3(kBlock), 0, st, q->codes + r * chunks * kChunk,
                         q->scales + r, pieces, x->cols, (uint32_t)per_row, (T*)x->data + r * x->stride, x->stride,
                         x->rows * x->cols * (int64_t)sizeof(T) > kStreamBytes);
        });
    });
}

constexpr int64_t kFullGrid = 256;                 // workgroups that fill the chip
constexpr int64_t kPartSteps = 4;                  // fewest steps of a part
constexpr int64_t kNear = (int64_t)32 << 20;       // operands that the caches near the compute units hold

static void check_sizes(int64_t M, int64_t N, int64_t K) {
    for (int64_t v : {M, N, K})
        AGNES_REQUIRE(v >= 0 && v < ((int64_t)1 << 31), AGNES_ERR_INVALID, "M, N and K must be in [0, 2^31)");
    // 2^14 K stays below 2^31, also for codes of -128
    AGNES_REQUIRE(K < ((int64_t)1 << 17), AGNES_ERR_INVALID, "K must be below 2^17");
}

// Which kernel computes M x N x K, by sizes alone.  k_int8_few reads x again for
// every 16 columns of out, and a workgroup's steps follow each other, so more than one
// 16-row tile pays only while rows x K x rounds of workgroups is small.  Up to 16
// rows take it at any size: it is the faster one but for the largest layers.  us,
// k_int8_few against tiles, of N x K: 16 rows of 4096 x 4096 7.0 / 9.6, of 1024 x 8192 9.7 / 12.0, of
// 8192 x 8192 18.9 / 16.8; 17 rows of 4096 x 4096 7.7 / 9.8, of 8192 x 8192 20.9 / 16.8; 32 rows of 4096 x
// 4096 9.0 / 9.9, of 2048 x 2048 5.9 / 6.7, of 8192 x 8192 25.9 / 17.5, of 1024 x 8192 13.1 / 12.5.
constexpr int64_t kFewTile = 16;                   // rows of k_int8_few at any size (16 of 8192 x 8192: 2 us more than tiles),
constexpr int64_t kFewRows = 32;                   // and at most, as long as
constexpr int64_t kFewWork = 1 << 17;              // rows x K x rounds is no more than this
constexpr int64_t kFewBytes = 40 << 10;            // LDS for rows that it quantises itself
struct Int8Plan {
    int rows;                                      // of a tile; 0: k_int8_few
    int parts;                                     // of K
};

// Refuses what no launch can hold (2^32 threads), so that callers do before they
// enqueue anything: a tile has at most 512 threads, and their number is rounded up
// to one for each XCD.
static Int8Plan plan_product(int64_t M, int64_t N, int64_t K) {
    constexpr int64_t kMostTiles = (1 << 23) - kXcds;
    auto require = [](bool fits) { AGNES_REQUIRE(fits, AGNES_ERR_RANGE, "the product has too many tiles"); };
    const int64_t columns = (N + 15) / 16, rounds = (N + 16 * kFullGrid - 1) / (16 * kFullGrid);
    if (M <= kFewTile) {
        require(columns <= kMostTiles);
        return {0, 1};
    }
    if (M <= kFewRows && K <= kFewWork && M * K * rounds <= kFewWork && columns <= kMostTiles) return {0, 1};
    // The tile, and the parts of K, that are fastest by what steps have measured: us
    // per step of one workgroup alone on its compute unit (its operands near, or far), and per
    // step and workgroup of a full chip; what a workgroup needs before and behind its steps;
    // the parts' sums at 3 TB/s.  us, tiles of 256 / 128 / 64: 256 x 4096 x 4096 42 / 24 / 12,
    // 1024 x 4096 x 4096 45 / 28 / 40, 3000 x 4096 x 4096 52 / 74 / 109; 64 rows of 8192 x 8192 in 1, 2, 4
    // and 8 parts 29, 22, 20 and 22; 64 rows of 1024 x 8192 in 1, 8 and 16 parts 16, 11 and 13.
    struct Tile {
        int rows;
        double near, far, full, ends;
    };
    static const Tile kTiles[] = {{256, 0.68, 0.75, 0.9, 5}, {128, 0.42, 0.45, 0.36, 3}, {64, 0.115, 0.22, 0.15, 1.5}};
    const double steps = (double)((chunks_of(K) + kStepChunks - 1) / kStepChunks);
    const bool near = (M + N) * K <= kNear;
    Int8Plan best{64, 1};
    double least = 0;
    for (const Tile& t : kTiles) {
        const int64_t tiles = ((M + t.rows - 1) / t.rows) * ((N + t.rows - 1) / t.rows);
        if (tiles > kMostTiles) continue;
        for (int64_t grid : {1, 256, 512, 1024}) {
            const int64_t parts = t.rows > 64 ? 1 : std::max<int64_t>(1, std::min(grid / tiles, (int64_t)steps / kPartSteps));
            const double each = std::ceil(steps / parts), groups = (double)(tiles * parts) / kFullGrid;
            const double us = t.ends + std::max(each * (near ? t.near : t.far), (t.rows == 256 ? std::ceil(groups) : groups) *
                                                                                   each * (groups < 0.75 ? 0 : t.full)) +
                              (parts > 1 ? 6 + (double)(parts * M * N) * 8 / 3e6 : 0);
            if (least == 0 || us < least) {
                least = us;
                best = {t.rows, (int)parts};
            }
        }
    }
    require(least > 0);
    return best;
}

uint64_t int8_product_bytes(int64_t M, int64_t N, int64_t K) {
    check_sizes(M, N, K);
    if (M == 0 || N == 0) return 0;
    const Int8Plan p = plan_product(M, N, K);
    return p.parts > 1 ? (uint64_t)(p.parts * M * N) * 4 : 0;
}

uint64_t int8_linear_bytes(int64_t M, int64_t N, int64_t K) {
    check_sizes(M, N, K);
    Carve c(nullptr);
    c.take<int8_t>(M * chunks_of(K) * kChunk);
    c.take<float>(M);
    return c.used + int8_product_bytes(M, N, K);
}

template <typename T, int WM, int WN, int F, int G> static void launch_tile(const Int8Args& a, int parts, hipStream_t st) {
    constexpr int R = WM * 16 * F, C = WN * 16 * G;
    const int64_t tiles = ((a.M + R - 1) / R) * ((a.N + C - 1) / C);
    const unsigned grid = (unsigned)((tiles + kXcds - 1) / kXcds * kXcds);
    AGNES_LAUNCH((k_int8_gemm<T, WM, WN, F, G>), dim3(grid, (unsigned)parts), dim3(kWave * WM * WN), 0, st, a);
}

template <typename S, typename T> static void launch_few(const Int8Args& a, const Int8Rows<S>& f, hipStream_t st) {
    constexpr bool QUANTISED = std::is_same<S, int8_t>::value;
    const int64_t groups = (a.N + 15) / 16;
    // more waves where there are few workgroups, but a step for each
    const int steps = (a.chunks + 7) / 8;
    int waves = groups <= 512 ? 16 : 8;
    while (waves > 1 && waves / 2 >= steps) waves /= 2;
    const dim3 grid((unsigned)groups), block((unsigned)(waves * kWave));
    const size_t lds = QUANTISED ? 0 : (size_t)a.M * a.chunks * kChunk;
    if (a.M <= 16) AGNES_LAUNCH((k_int8_few<S, T, 1>), grid, block, lds, st, a, f);
    else if constexpr (QUANTISED) {
        AGNES_LAUNCH((k_int8_few<S, T, 2>), grid, block, 0, st, a, f);
    }
}

static void check_product(const agnes_int8* w, int64_t M, int64_t K, const agnes_matrix* out) {
    check_int8(w, "w");
    check_matrix(out, true, "out");
    AGNES_REQUIRE(K == w->cols, AGNES_ERR_INVALID, "x and w must have equal columns");
    AGNES_REQUIRE(out->rows == M && out->cols == w->rows, AGNES_ERR_INVALID,
                  "out must have x's rows and one column per row of w");
}

static Int8Args args_of(const agnes_int8* x, const agnes_int8* w, const float* bias, bool relu, const agnes_matrix* out) {
    return {x->codes, w->codes, x->scales, w->scales, x->rows, w->rows, (int32_t)chunks_of(x->cols), bias, relu,
            x->rows * w->rows * (int64_t)elem_size(out->dtype) > kStreamBytes, out->data, out->stride, nullptr};
}

void int8_product(const agnes_int8* x, const agnes_int8* w, const float* bias, bool relu, const agnes_matrix* out,
                  void* ws, uint64_t ws_bytes, hipStream_t st) {
    check_int8(x, "x");
    check_product(w, x->rows, x->cols, out);
    const int64_t M = x->rows, N = w->rows;
    check_workspace(ws, ws_bytes, int8_product_bytes(M, N, x->cols));   // checks the sizes too
    if (M == 0 || N == 0) return;
    const Int8Plan p = plan_product(M, N, x->cols);
    Int8Args a = args_of(x, w, bias, relu, out);
    if (p.parts > 1) {
        a.parts = (int32_t*)ws;
        launch_tile<int32_t, 2, 2, 2, 2>(a, p.parts, st);
    }
    with_float(out->dtype, [&](auto t) {
        typedef decltype(t) T;
        if (p.rows == 0) launch_few<int8_t, T>(a, Int8Rows<int8_t>{x->codes, 0, x->cols}, st);
        else if (p.rows == 256) launch_tile<T, 2, 4, 8, 4>(a, 1, st);
        else if (p.rows == 128) launch_tile<T, 2, 2, 4, 4>(a, 1, st);
        else if (p.parts == 1) launch_tile<T, 2, 2, 2, 2>(a, 1, st);
        else AGNES_LAUNCH((k_int8_join<T>), dim3(grid_for((M * N + 3) / 4, 4096)), dim3(kBlock), 0, st, a, p.parts);
    });
}

void int8_linear(const agnes_matrix* x, const agnes_int8* w, const float* bias, bool relu, const agnes_matrix* out,
                 void* ws, uint64_t ws_bytes, hipStream_t st) {
    check_matrix(x, false, "x");
    check_product(w, x->rows, x->cols, out);
    check_workspace(ws, ws_bytes, int8_linear_bytes(x->rows, w->rows, x->cols));
    if (x->rows == 0 || w->rows == 0) return;
    Carve c(ws);
    agnes_int8 q{};
    q.rows = x->rows;
    q.cols = x->cols;
    q.codes = c.take<int8_t>(x->rows * chunks_of(x->cols) * kChunk);
    q.scales = c.take<float>(x->rows);
    if (x->rows <= kFewTile && x->rows * chunks_of(x->cols) * kChunk <= kFewBytes) {
        const Int8Args a = args_of(&q, w, bias, relu, out);
        with_float(x->dtype, [&](auto ts) {
            with_float(out->dtype, [&](auto t) {
                typedef decltype(ts) S;
                launch_few<S, decltype(t)>(a, Int8Rows<S>{(const S*)x->data, x->stride, x->cols}, st);
            });
        });
        return;
    }
    int8_quantize(x, &q, st);
    int8_product(&q, w, bias, relu, out, (char*)ws + c.used, ws_bytes - c.used, st);
}

}  // namespace agnes
