// Loss of a student's logits against a teacher's top logits, and its gradient.
//
// With m = max_j z_j, S_T = sum_j exp((z_j - m) / T) and S_1 = sum_j exp(z_j - m):
//   ln q_j = (z_j - m) / T - ln S_T
//   loss   = w [ a T^2 sum_e p_e (ln p_e - ln q_{c_e}) + b (ln S_1 - (z_y - m)) ]
//   grad_j = w [ a T (P q_j - sum_{c_e = j} p_e) + b (exp(z_j - m) / S_1 - [j = y]) ]
// p is the softmax of the row's valid teacher logits, P = 1 if there are any.
//
// A row of logits is read once, stays in registers between its sums and its
// gradient, and its gradient is written once; the classes that the teacher or
// the label names get their values in a second store behind the row's.
// Variants, by the number of 16-byte pieces of a row:
//   up to 256      some lanes of a wave per row (a whole wave from 33 pieces on)
//   up to 16384    a workgroup of 256 to 1024 threads per row
//   above, or above 1024 with too few rows to fill the chip: the row is split
//     over workgroups; a first launch leaves each part's maximum and sums, a
//     second one joins them and writes the gradient (a second read of the row).
#include <algorithm>
#include <cmath>

#include "ops.hpp"

namespace agnes {

constexpr float kLog2e = 1.44269504088896340736f;

// The descriptor as the kernels take it.
struct DistillArgs {
    const void* z;
    const void* t;
    const void* classes;
    const void* labels;
    const float* weight;
    const float* stats_in;         // the rows' statistics, or NULL: from the logits
    float* loss;
    float* stats;
    void* grad;
    int64_t zstride, tstride, cstride, gstride;
    int64_t rows;
    int32_t C, k;
    agnes_dtype ttype, gtype;
    bool wide;                     // 64-bit classes and labels
    bool nt;                       // gradient past the caches
    float temp, soft, hard;        // T, a, b
    float ct;                      // log2(e) / T: exp(x / T) = 2^(x ct)
};

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

// E gradients from column c on, those before column hi, of the row whose first element is number `at`.
template <int E>
__device__ __forceinline__ void store_grad(const DistillArgs& a, int64_t at, int c, int hi, const float (&x)[E]) {
    if (a.gtype == AGNES_FLOAT32) store_typed<E>((float*)a.grad + at, c, hi, x, a.nt);
    else if (a.gtype == AGNES_FLOAT16) store_typed<E>((_Float16*)a.grad + at, c, hi, x, a.nt);
    else store_typed<E>((__bf16*)a.grad + at, c, hi, x, a.nt);
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

// How exp(d) follows from exp(d / T): kOne: not needed, or the same (T = 1);
// kTwo: an exponential of its own; kSquare: its square (T = 2), a product in
// place of the exponential.  With a label term, T = 2 and T = 3: 8192 rows of
// 65536 bfloat16 423 and 444 us, 65536 rows of 172 float32 37.0 and 38.4 us.
enum { kOne = 0, kTwo = 1, kSquare = 2 };

template <int MODE> __device__ __forceinline__ float plain_exp(float d, float et) {
    if (MODE == kTwo) return pow2(d * kLog2e);
    if (MODE == kSquare) return et * et;
    return et;
}

// Maximum and sums of part of a row, relative to that maximum.
struct Sums {
    float m, st, s1;
};

// Adds E logits (-inf where there are none), none above s.m.  A NaN or +inf
// logit makes the sums NaN, and with them everything that follows; where all
// logits so far are -inf (or NaN, which a maximum passes over) the base is 0.
template <int MODE, int E, typename Raw> __device__ __forceinline__ void add_piece(Sums& s, const Raw& v, float ct) {
    const float base = s.m == -INFINITY ? 0.f : s.m;
#pragma unroll
    for (int q = 0; q < E; q++) {
        const float d = (float)v[q] - base;
        const float e = pow2(d * ct);
        s.st += e;
        if (MODE != kOne) s.s1 += plain_exp<MODE>(d, e);
    }
}

// Brings sums to the maximum m of a larger part.
template <int MODE> __device__ __forceinline__ void rebase(Sums& s, float m, float ct) {
    if (m == -INFINITY) return;                  // the sums are 0 (or NaN)
    const float d = s.m - m;
    s.st *= pow2(d * ct);
    if (MODE != kOne) s.s1 *= pow2(d * kLog2e);
    s.m = m;
}

template <int MODE> __device__ __forceinline__ Sums lanes_join(Sums s, int L, float ct) {
    rebase<MODE>(s, lanes_max(s.m, L), ct);
    s.st = lanes_sum(s.st, L);
    s.s1 = MODE == kOne ? s.st : lanes_sum(s.s1, L);
    return s;
}

// Every logit is -inf.
__device__ __forceinline__ bool no_logits(const Sums& s) { return s.m == -INFINITY && s.st == 0.f; }

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

// What the teacher and the label ask of a row: the factors of q_j and of
// exp(z_j - m) / S_1 in the gradient before the division by the sums.
struct Terms {
    bool some, named;
    int64_t y;
    float w, ca, cb;
};

// A lane's entry e of the teacher and the row's label, as loaded.
struct Entry {
    int64_t c;
    float t;
};
__device__ __forceinline__ Entry load_entry(const DistillArgs& a, int64_t r, int e) {
    Entry x{-1, 0.f};
    if (e < a.k) {
        x.c = load_index(a.classes, a.wide, r * a.cstride + e);
        x.t = load_any(a.t, a.ttype, r * a.tstride + e);
    }
    return x;
}
__device__ __forceinline__ int64_t load_label(const DistillArgs& a, int64_t r) {
    return a.labels ? load_index(a.labels, a.wide, r) : -1;
}

// The teacher's distribution over lanes gl = 0 .. L - 1, entries e = gl (loaded
// before: first), gl + L, ...: classes (-1: padding) to cls, probabilities to
// prob.  Every lane gets the terms.  The largest logit is subtracted before the
// division by T, as for the student: a quotient would overflow at T < 1 where
// logits are the type's lowest or highest value, and lose digits where all of
// a row's logits are large.
__device__ __forceinline__ Terms teacher(const DistillArgs& a, int64_t r, float w, Entry first, int64_t y, int gl,
                                         int L, int32_t* cls, float* prob) {
    float tm = -INFINITY;
    Entry n = first;
    for (int e = gl; e < a.k; e += L) {
        if (e != gl) n = load_entry(a, r, e);
        const bool ok = n.c >= 0 && n.c < a.C;
        const float x = ok ? n.t : -INFINITY;
        cls[e] = ok ? (int32_t)n.c : -1;
        prob[e] = x;
        tm = x != x ? INFINITY : fmaxf(tm, x);   // NaN: as +inf, which makes the sum NaN
    }
    tm = lanes_max(tm, L);
    Terms q;
    q.w = w;
    q.some = a.soft > 0.f && tm != -INFINITY;
    float ts = 0.f;
    for (int e = gl; e < a.k; e += L) {
        const float p = q.some ? pow2((prob[e] - tm) * a.ct) : 0.f;
        prob[e] = p;
        ts += p;
    }
    ts = lanes_sum(ts, L);
    if (q.some) {
        const float inv = 1.f / ts;
        for (int e = gl; e < a.k; e += L) prob[e] *= inv;
    }
    q.y = y;
    q.named = a.hard > 0.f && q.y >= 0 && q.y < a.C;
    q.ca = q.some ? w * a.soft * a.temp : 0.f;
    q.cb = q.named ? w * a.hard : 0.f;
    return q;
}
__device__ __forceinline__ Terms teacher(const DistillArgs& a, int64_t r, float w, int gl, int L, int32_t* cls,
                                         float* prob) {
    return teacher(a, r, w, load_entry(a, r, gl), load_label(a, r), gl, L, cls, prob);
}

// An entry's part of the divergence: T p (ln p - ln q_c), from z - m of its class
// and the logarithm of S_T.  The difference is not divided by T: at T < 1 that
// overflows for a logit at the type's lowest value.
__device__ __forceinline__ float divergence_term(const DistillArgs& a, float p, float zm, float lt) {
    return p * (a.temp * (logf(p) + lt) - zm);
}

// T sum_e p_e (ln p_e - ln q_{c_e}) over the lanes, from z_{c_e} in zc.
__device__ __forceinline__ float divergence(const DistillArgs& a, const Sums& s, const float* prob, const float* zc,
                                            int gl, int L) {
    const float lt = logf(s.st);
    float part = 0.f;
    for (int e = gl; e < a.k; e += L) {
        const float p = prob[e];
        if (p != 0.f) part += divergence_term(a, p, zc[e] - s.m, lt);
    }
    return lanes_sum(part, L);
}

// div: T times the divergence; dy = z_y - m.
__device__ __forceinline__ float row_loss(const DistillArgs& a, const Terms& q, const Sums& s, float div, float dy) {
    if (no_logits(s)) return q.some || q.named ? q.w * INFINITY : 0.f;
    float L = q.some ? a.soft * a.temp * div : 0.f;
    if (q.named) L += a.hard * (logf(s.s1) - dy);
    return q.w * L;
}

// The gradient of logits [c, c + E), without the teacher's and the label's part.
template <int MODE, int E, typename Raw>
__device__ __forceinline__ void grad_piece(const DistillArgs& a, const Raw& v, const Sums& s, float ka, float kb,
                                           float (&x)[E]) {
#pragma unroll
    for (int q = 0; q < E; q++) {
        const float d = (float)v[q] - s.m;
        const float e = pow2(d * a.ct);
        x[q] = ka * e;
        if (MODE != kOne) x[q] += kb * plain_exp<MODE>(d, e);
    }
}

// The factors of exp((z - m) / T) and exp(z - m) in the gradient; with one
// exponential, of T = 1 or of a single term, their sum in ka.  A term that is
// not asked for has the factor 0, whatever its sum holds.
template <int MODE> __device__ __forceinline__ void factors(const Terms& q, const Sums& s, float& ka, float& kb) {
    ka = q.some ? q.ca / s.st : 0.f;
    kb = q.named ? q.cb / s.s1 : 0.f;
    if (MODE == kOne) {
        ka += kb;
        kb = 0.f;
    }
}

// The gradient of class c, named by the teacher with the total probability p.
template <int MODE>
__device__ __forceinline__ float grad_named(const DistillArgs& a, const Terms& q, const Sums& s, float ka, float kb,
                                            float z, int64_t c, float p) {
    const float d = z - s.m;
    const float e = pow2(d * a.ct);
    float x = ka * e;
    if (MODE != kOne) x += kb * plain_exp<MODE>(d, e);
    if (q.some) x -= q.ca * p;
    if (q.named && c == q.y) x -= q.cb;
    return x;
}

// The total probability of class c: of all entries that list it, in their order.
__device__ __forceinline__ float listed(const int32_t* cls, const float* prob, int k, int32_t c) {
    float p = 0.f;
    for (int e = 0; e < k; e++)
        if (cls[e] == c) p += prob[e];
    return p;
}

// Whether the lane's class c (-1: none) may be listed twice: certain if all
// entries are in the L lanes of its group, else assumed.
__device__ __forceinline__ bool listed_twice(const DistillArgs& a, int32_t c, int L) {
    if (a.k > L) return true;
    uint64_t same = __ballot(c >= 0);
    if (L < kWave) same &= ((1ull << L) - 1) << (lane_id() & ~(L - 1));
    for (int b = 0; b < 31 && (a.C >> b); b++) {
        const uint64_t m = __ballot((c >> b) & 1);
        same &= ((c >> b) & 1) ? m : ~m;
    }
    return (same & (same - 1)) != 0;
}

// Stores the gradient of the classes in [lo, hi) that the teacher lists or the
// label names, by one wave.  A class listed twice is stored twice, with the
// same value.
template <int MODE>
__device__ __forceinline__ void store_named(const DistillArgs& a, const Terms& q, const Sums& s, float ka, float kb,
                                            const int32_t* cls, const float* prob, const float* zc, float zy,
                                            int64_t at, int lane, int lo, int hi) {
    wave_sync();                                 // cls and prob of the other lanes
    if (q.some) {
        for (int e0 = 0; e0 < a.k; e0 += kWave) {
            const int e = e0 + lane;
            const int32_t c = e < a.k ? cls[e] : -1;
            const bool again = listed_twice(a, c, kWave);
            if (c < 0 || c < lo || c >= hi) continue;
            const float p = again ? listed(cls, prob, a.k, c) : prob[e];
            store_any(a.grad, a.gtype, at + c, grad_named<MODE>(a, q, s, ka, kb, zc[e], c, p));
        }
    }
    if (q.named && lane == 0 && q.y >= lo && q.y < hi) {
        const float p = q.some ? listed(cls, prob, a.k, (int32_t)q.y) : 0.f;
        store_any(a.grad, a.gtype, at + q.y, grad_named<MODE>(a, q, s, ka, kb, zy, q.y, p));
    }
}

// ----------------------------------------------------------------- lanes of a wave per row

// L lanes per row, P pieces per lane, up to kLaneEntries teacher entries.  What a
// row costs besides its logits is the same for every row of a wave, so a lane
// takes up to four pieces before a row takes more lanes (65536 rows of 172
// float32: 74 us with 64 lanes per row, 36 us with 16).  A row is short work behind a long wait, so a group takes several
// rows, and the next row's logits, entries, label and weight are loaded before
// the present row's arithmetic.  The row also goes to LDS, where the named
// logits are found; then what the named classes lose goes there, so that every
// gradient is stored once.
constexpr int kLaneEntries = 64;
constexpr int kLanesMin = 8;
constexpr int kLaneGroups = 2048;                // workgroups, about what the chip holds at once

template <typename T, int P> struct LaneRow {
    static constexpr int E = 16 / (int)sizeof(T);
    typename Vec<T, E>::type v[P];
    float w;
    Entry first;
    int64_t y;
};

template <typename T, int P, int MODE>
__global__ __launch_bounds__(kBlock) void k_distill_lanes(DistillArgs a, int L) {
    constexpr int E = 16 / (int)sizeof(T);
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int groups = kBlock / L, g = threadIdx.x / L, gl = threadIdx.x % L;
    float* corr = lds + g * (L * P * E);                    // what a column's gradient loses
    T* zrow = (T*)corr;                                     // before that, the row's logits
    int32_t* cls = (int32_t*)(lds + kBlock * P * E) + g * 2 * a.k;
    float* prob = (float*)(cls + a.k);
    const int64_t step = (int64_t)gridDim.x * groups;
    int64_t r = (int64_t)blockIdx.x * groups + g;
    auto load = [&](int64_t i) {
        LaneRow<T, P> x;
        const T* zr = (const T*)a.z + i * a.zstride;
#pragma unroll
        for (int p = 0; p < P; p++) x.v[p] = logits_piece<T, E>(zr, (gl + p * L) * E, a.C);
        x.w = a.weight ? a.weight[i] : 1.f;
        x.first = load_entry(a, i, gl);
        x.y = load_label(a, i);
        return x;
    };
    LaneRow<T, P> next;
    if (r < a.rows) next = load(r);
    for (; r < a.rows; r += step) {                         // per group; nothing below crosses a group
        LaneRow<T, P> x = next;
        if (r + step < a.rows) next = load(r + step);
        const int64_t at = r * a.gstride;
        if (x.w == 0.f) {
            if (gl == 0 && a.loss) a.loss[r] = 0.f;
            if (gl == 0 && a.stats) a.stats[3 * r] = a.stats[3 * r + 1] = a.stats[3 * r + 2] = 0.f;
            if (a.grad) {
                const float zero[E] = {};
#pragma unroll
                for (int p = 0; p < P; p++) store_grad<E>(a, at, (gl + p * L) * E, a.C, zero);
            }
            continue;
        }
        wave_sync();                                        // the row before is done with the LDS
#pragma unroll
        for (int p = 0; p < P; p++) __builtin_memcpy(__builtin_assume_aligned(zrow + (gl + p * L) * E, 16), &x.v[p], 16);
        const Terms q = teacher(a, r, x.w, x.first, x.y, gl, L, cls, prob);
        Sums s{-INFINITY, 0.f, 0.f};
        if (a.stats_in) {
            s = Sums{a.stats_in[3 * r], a.stats_in[3 * r + 1], a.stats_in[3 * r + 2]};
        } else {
#pragma unroll
            for (int p = 0; p < P; p++)
#pragma unroll
                for (int e = 0; e < E; e++) s.m = fmaxf(s.m, (float)x.v[p][e]);
            s.m = lanes_max(s.m, L);
#pragma unroll
            for (int p = 0; p < P; p++) {
                keep_packed(x.v[p]);
                add_piece<MODE, E>(s, x.v[p], a.ct);
                __builtin_amdgcn_sched_barrier(0);
            }
            s.st = lanes_sum(s.st, L);
            s.s1 = MODE == kOne ? s.st : lanes_sum(s.s1, L);
        }
        if (a.loss) {
            wave_sync();                                    // the row is in LDS
            float div = 0.f;
            if (q.some) {
                const float lt = logf(s.st);
                for (int e = gl; e < a.k; e += L) {
                    const float p = prob[e];
                    if (p != 0.f) div += divergence_term(a, p, (float)zrow[cls[e]] - s.m, lt);
                }
                div = lanes_sum(div, L);
            }
            const float zy = q.named ? (float)zrow[q.y] : 0.f;
            if (gl == 0) a.loss[r] = row_loss(a, q, s, div, zy - s.m);
        }
        if (gl == 0 && a.stats) {
            a.stats[3 * r] = s.m;
            a.stats[3 * r + 1] = s.st;
            a.stats[3 * r + 2] = s.s1;
        }
        if (!a.grad) continue;
        wave_sync();                                        // the row's logits have been read
        const bool empty = no_logits(s), live = !empty && (q.some || q.named);
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        f32x4* const mine = (f32x4*)(corr + gl * E);        // piece p: mine[p L E / 4 ..]
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int e = 0; e < E / 4; e++) mine[p * (L * E / 4) + e] = f32x4{0.f, 0.f, 0.f, 0.f};
        wave_sync();
        if (q.some)
            for (int e = gl; e < a.k; e += L) {
                const int32_t c = cls[e];
                const bool again = listed_twice(a, c, L);
                if (c >= 0) corr[c] = q.ca * (again ? listed(cls, prob, a.k, c) : prob[e]);
            }
        wave_sync();
        if (q.named && gl == 0) corr[q.y] += q.cb;
        wave_sync();
        float ka, kb;
        factors<MODE>(q, s, ka, kb);
#pragma unroll
        for (int p = 0; p < P; p++) {
            float y[E] = {};
            keep_packed(x.v[p]);
            if (live) {
                grad_piece<MODE, E>(a, x.v[p], s, ka, kb, y);
#pragma unroll
                for (int e = 0; e < E; e++) y[e] -= mine[p * (L * E / 4) + e / 4][e % 4];
            }
            store_grad<E>(a, at, (gl + p * L) * E, a.C, y);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// ----------------------------------------------------------------- a workgroup per row

template <typename T, int THREADS, int P, int MODE>
__global__ __launch_bounds__(THREADS, THREADS == 1024 && P == 8 ? 8 : 4) void k_distill_block(DistillArgs a) {
    constexpr int E = 16 / (int)sizeof(T), WAVES = THREADS / kWave;
    typedef typename Vec<T, E>::type Raw;
    __shared__ int32_t cls[AGNES_DISTILL_MAX_K];
    __shared__ float prob[AGNES_DISTILL_MAX_K];
    __shared__ float zc[AGNES_DISTILL_MAX_K];
    __shared__ Sums red[WAVES];
    __shared__ Terms terms;
    const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;
    const int64_t r = blockIdx.x;
    const T* zr = (const T*)a.z + r * a.zstride;
    const int64_t at = r * a.gstride;
    const float w = a.weight ? a.weight[r] : 1.f;
    if (w == 0.f) {
        if (tid == 0 && a.loss) a.loss[r] = 0.f;
        if (tid == 0 && a.stats) a.stats[3 * r] = a.stats[3 * r + 1] = a.stats[3 * r + 2] = 0.f;
        if (a.grad) {
            const float zero[E] = {};
            for (int c = tid * E; c < a.C; c += THREADS * E) store_grad<E>(a, at, c, a.C, zero);
        }
        return;
    }
    Raw v[P];
#pragma unroll
    for (int i = 0; i < P; i++)
        if (i * THREADS * E < a.C) v[i] = logits_piece<T, E>(zr, (tid + i * THREADS) * E, a.C);
    Terms q{};
    float zy = 0.f;
    if (wave == 0) {
        q = teacher(a, r, w, lane, kWave, cls, prob);
        for (int e = lane; e < a.k; e += kWave) zc[e] = cls[e] >= 0 ? (float)zr[cls[e]] : 0.f;
        zy = q.named ? (float)zr[q.y] : 0.f;
        if (lane == 0) terms = q;
    }
    Sums s{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < P; i++)
        if (i * THREADS * E < a.C) {
#pragma unroll
            for (int x = 0; x < E; x++) s.m = fmaxf(s.m, (float)v[i][x]);
        }
    s.m = lanes_max(s.m, kWave);
#pragma unroll
    for (int i = 0; i < P; i++)
        if (i * THREADS * E < a.C) {             // no work for rounds that lie behind the row
            keep_packed(v[i]);
            add_piece<MODE, E>(s, v[i], a.ct);
            __builtin_amdgcn_sched_barrier(0);   // one piece's values at a time: registers decide the occupancy
        }
    s.st = lanes_sum(s.st, kWave);
    s.s1 = MODE == kOne ? s.st : lanes_sum(s.s1, kWave);
    if (lane == 0) red[wave] = s;
    __syncthreads();                             // also: the named logits have been read
    s = lane < WAVES ? red[lane] : Sums{-INFINITY, 0.f, 0.f};
    s = lanes_join<MODE>(s, kWave, a.ct);
    q = terms;
    if (wave == 0) {
        if (a.loss) {
            const float div = q.some ? divergence(a, s, prob, zc, lane, kWave) : 0.f;
            if (lane == 0) a.loss[r] = row_loss(a, q, s, div, zy - s.m);
        }
        if (lane == 0 && a.stats) {
            a.stats[3 * r] = s.m;
            a.stats[3 * r + 1] = s.st;
            a.stats[3 * r + 2] = s.s1;
        }
    }
    if (!a.grad) return;
    const bool empty = no_logits(s);
    float ka, kb;
    factors<MODE>(q, s, ka, kb);
#pragma unroll
    for (int i = 0; i < P; i++) {
        if (i * THREADS * E < a.C) {
            const int c = (tid + i * THREADS) * E;
            float x[E] = {};
            keep_packed(v[i]);
            if (!empty && (q.some || q.named)) grad_piece<MODE, E>(a, v[i], s, ka, kb, x);
            store_grad<E>(a, at, c, a.C, x);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    __syncthreads();                             // the row's values are stored before the named classes'
    if (wave == 0 && !empty) store_named<MODE>(a, q, s, ka, kb, cls, prob, zc, zy, at, lane, 0, a.C);
}

// ----------------------------------------------------------------- a row over several workgroups

// Part of a row: its maximum and sums, and of the classes that lie in it the
// teacher's probability and sum_e p_e (z_{c_e} - m), and z_y - m.
struct Part {
    Sums s;
    float mass, cross, label;
    float pad[2];
};

constexpr int kPartThreads = 256;

// blockIdx: (part, row).  A part is `span` logits, a multiple of a piece.
template <typename T, int MODE>
__global__ __launch_bounds__(kPartThreads) void k_distill_part(DistillArgs a, int64_t span, Part* __restrict__ parts) {
    constexpr int E = 16 / (int)sizeof(T), U = 4;
    typedef typename Vec<T, E>::type Raw;
    __shared__ int32_t cls[AGNES_DISTILL_MAX_K];
    __shared__ float prob[AGNES_DISTILL_MAX_K];
    __shared__ Sums red[kPartThreads / kWave];
    const int tid = threadIdx.x, lane = lane_id(), wave = wave_id();
    const int64_t r = blockIdx.y;
    const T* zr = (const T*)a.z + r * a.zstride;
    const float w = a.weight ? a.weight[r] : 1.f;
    if (w == 0.f) return;                        // the second launch skips the row too
    const int lo = (int)(blockIdx.x * span), hi = (int)min((int64_t)a.C, lo + span);
    Sums s{-INFINITY, 0.f, 0.f};
    for (int c0 = lo; c0 < hi; c0 += kPartThreads * E * U) {
        Raw v[U];
#pragma unroll
        for (int i = 0; i < U; i++)
            v[i] = logits_piece<T, E>(zr, c0 + (tid + i * kPartThreads) * E, hi);
        float m = s.m;
#pragma unroll
        for (int i = 0; i < U; i++)
#pragma unroll
            for (int x = 0; x < E; x++) m = fmaxf(m, (float)v[i][x]);
        rebase<MODE>(s, m, a.ct);
#pragma unroll
        for (int i = 0; i < U; i++) add_piece<MODE, E>(s, v[i], a.ct);
    }
    s = lanes_join<MODE>(s, kWave, a.ct);
    if (lane == 0) red[wave] = s;
    __syncthreads();
    if (wave != 0) return;
    s = lane < kPartThreads / kWave ? red[lane] : Sums{-INFINITY, 0.f, 0.f};
    s = lanes_join<MODE>(s, kWave, a.ct);
    const Terms q = teacher(a, r, w, lane, kWave, cls, prob);
    const float m = s.m == -INFINITY ? 0.f : s.m;
    float mass = 0.f, cross = 0.f;
    for (int e = lane; e < a.k; e += kWave)
        if (prob[e] != 0.f && cls[e] >= lo && cls[e] < hi) {
            mass += prob[e];
            cross += prob[e] * ((float)zr[cls[e]] - m);
        }
    mass = lanes_sum(mass, kWave);
    cross = lanes_sum(cross, kWave);
    if (lane == 0) {
        Part p{};
        p.s = s;
        p.mass = mass;
        p.cross = cross;
        p.label = q.named && q.y >= lo && q.y < hi ? (float)zr[q.y] - m : 0.f;
        parts[r * gridDim.x + blockIdx.x] = p;
    }
}

// The row's sums from its parts (or from stats_in), then the loss, by the first
// workgroup, and the gradient of [lo, hi).
template <typename T, int MODE>
__global__ __launch_bounds__(kPartThreads) void k_distill_apply(DistillArgs a, int64_t span, int nparts,
                                                                const Part* __restrict__ parts) {
    constexpr int E = 16 / (int)sizeof(T), U = 4;
    typedef typename Vec<T, E>::type Raw;
    __shared__ int32_t cls[AGNES_DISTILL_MAX_K];
    __shared__ float prob[AGNES_DISTILL_MAX_K];
    __shared__ float zc[AGNES_DISTILL_MAX_K];
    __shared__ Terms terms;
    const int tid = threadIdx.x, lane = lane_id(), wave = wave_id();
    const int64_t r = blockIdx.y;
    const T* zr = (const T*)a.z + r * a.zstride;
    const int64_t at = r * a.gstride;
    const float w = a.weight ? a.weight[r] : 1.f;
    const int lo = (int)(blockIdx.x * span), hi = (int)min((int64_t)a.C, lo + span);
    const bool first = blockIdx.x == 0;
    if (w == 0.f) {
        if (first && tid == 0 && a.loss) a.loss[r] = 0.f;
        if (first && tid == 0 && a.stats) a.stats[3 * r] = a.stats[3 * r + 1] = a.stats[3 * r + 2] = 0.f;
        if (a.grad) {
            const float zero[E] = {};
            for (int c = lo + tid * E; c < hi; c += kPartThreads * E) store_grad<E>(a, at, c, hi, zero);
        }
        return;
    }
    Sums s{-INFINITY, 0.f, 0.f};
    float mass = 0.f, cross = 0.f, label = 0.f;
    if (a.stats_in) {
        s = Sums{a.stats_in[3 * r], a.stats_in[3 * r + 1], a.stats_in[3 * r + 2]};
    } else {
        const Part* p = parts + r * nparts;
        for (int i = lane; i < nparts; i += kWave) s.m = fmaxf(s.m, p[i].s.m);
        s.m = lanes_max(s.m, kWave);
        for (int i = lane; i < nparts; i += kWave) {
            const Part x = p[i];
            Sums y = x.s;
            rebase<MODE>(y, s.m, a.ct);
            s.st += y.st;
            s.s1 += y.s1;
            const float up = x.s.m == -INFINITY ? 0.f : x.s.m;      // what the part's values are relative to
            mass += x.mass;
            if (x.mass != 0.f) cross += x.cross + x.mass * (up - s.m);
            // a label of another part leaves 0, of this part z_y - up
            if (first) {
                const int64_t y0 = (int64_t)i * span;
                const int64_t lab = a.labels ? load_index(a.labels, a.wide, r) : -1;
                if (lab >= y0 && lab < y0 + span && lab < a.C) label = x.label + (up - s.m);
            }
        }
        s.st = lanes_sum(s.st, kWave);
        s.s1 = MODE == kOne ? s.st : lanes_sum(s.s1, kWave);
        mass = lanes_sum(mass, kWave);
        cross = lanes_sum(cross, kWave);
        label = lanes_sum(label, kWave);
    }
    if (wave == 0) {
        const Terms q = teacher(a, r, w, lane, kWave, cls, prob);
        if (lane == 0) terms = q;
        if (a.grad)
            for (int e = lane; e < a.k; e += kWave)
                zc[e] = cls[e] >= lo && cls[e] < hi ? (float)zr[cls[e]] : 0.f;
        if (first && a.loss) {
            float part = 0.f;                    // sum_e p_e ln p_e
            for (int e = lane; e < a.k; e += kWave)
                if (prob[e] != 0.f) part += prob[e] * logf(prob[e]);
            part = lanes_sum(part, kWave);
            const float div = a.temp * (part + mass * logf(s.st)) - cross;
            if (lane == 0) a.loss[r] = row_loss(a, q, s, q.some ? div : 0.f, label);
        }
        if (first && lane == 0 && a.stats) {
            a.stats[3 * r] = s.m;
            a.stats[3 * r + 1] = s.st;
            a.stats[3 * r + 2] = s.s1;
        }
    }
    if (!a.grad) return;
    __syncthreads();
    const Terms q = terms;
    const bool empty = no_logits(s);
    const float zy = q.named && q.y >= lo && q.y < hi ? (float)zr[q.y] : 0.f;
    float ka, kb;
    factors<MODE>(q, s, ka, kb);
    __syncthreads();                             // the named logits are read before anything is stored
    for (int c0 = lo; c0 < hi; c0 += kPartThreads * E * U) {
        Raw v[U];
#pragma unroll
        for (int i = 0; i < U; i++)
            v[i] = logits_piece<T, E>(zr, c0 + (tid + i * kPartThreads) * E, hi);
#pragma unroll
        for (int i = 0; i < U; i++) {
            const int c = c0 + (tid + i * kPartThreads) * E;
            float x[E] = {};
            if (!empty && (q.some || q.named)) grad_piece<MODE, E>(a, v[i], s, ka, kb, x);
            store_grad<E>(a, at, c, hi, x);
        }
    }
    __syncthreads();
    if (wave == 0 && !empty) store_named<MODE>(a, q, s, ka, kb, cls, prob, zc, zy, at, lane, lo, hi);
}

// ----------------------------------------------------------------- host

constexpr int64_t kLanePieces = 4 * kWave;       // a wave's rows
constexpr int64_t kSplitPieces = 1024;           // rows that may be split
constexpr int64_t kBlockPieces = 16 * 1024;      // a workgroup's rows
constexpr int64_t kSplitRows = 512;              // fewer rows leave too many compute units idle
constexpr int64_t kSplitGroups = 1024;           // workgroups that a split aims at
constexpr int64_t kLaunchRows = 1 << 21;         // rows per launch of a workgroup each: a launch holds fewer than 2^32 threads

// Parts of a row of C logits of `size` bytes, or 1 and span 0: not split.  A
// part has at least one round of its workgroup.
static int parts_of(int64_t rows, int64_t C, int64_t size, int64_t& span) {
    const int64_t E = 16 / size, pieces = (C + E - 1) / E, round = (int64_t)kPartThreads * E;
    span = 0;
    const bool many = pieces > kBlockPieces;
    if (!many && (pieces <= kSplitPieces || rows >= kSplitRows)) return 1;
    const int64_t want = std::max<int64_t>((kSplitGroups + rows - 1) / rows, many ? 2 : 1);
    const int64_t rounds = std::max<int64_t>(1, (C + round * want - 1) / (round * want));
    span = rounds * round;
    return (int)((C + span - 1) / span);
}

uint64_t distill_bytes(int64_t rows, int64_t classes) {
    AGNES_REQUIRE(rows >= 0 && classes >= 0 && rows < ((int64_t)1 << 31) && classes < ((int64_t)1 << 31),
                  AGNES_ERR_INVALID, "rows and classes must be in [0, 2^31)");
    if (rows == 0 || classes == 0) return 0;
    int64_t span = 0, most = 0;
    for (int64_t size : {2, 4}) {                // either size of logits
        const int n = parts_of(rows, classes, size, span);
        if (span) most = std::max<int64_t>(most, rows * n * (int64_t)sizeof(Part));
    }
    return (uint64_t)most;
}

static DistillArgs check_distill(const agnes_distill* d, const agnes_matrix* grad) {
    AGNES_REQUIRE(d, AGNES_ERR_INVALID, "the descriptor must not be NULL");
    check_matrix(&d->logits, false, "logits");
    check_matrix(&d->teacher, false, "teacher");
    const int64_t rows = d->logits.rows, C = d->logits.cols, k = d->teacher.cols;
    AGNES_REQUIRE(C >= 1, AGNES_ERR_INVALID, "there must be at least one class");
    AGNES_REQUIRE(C < ((int64_t)1 << 31) - (1 << 16), AGNES_ERR_INVALID, "there must be fewer than 2^31 - 2^16 classes");
    AGNES_REQUIRE(d->teacher.rows == rows, AGNES_ERR_INVALID, "teacher and logits must have equal rows");
    AGNES_REQUIRE(k <= AGNES_DISTILL_MAX_K, AGNES_ERR_INVALID, "the teacher may have at most 1024 entries per row");
    AGNES_REQUIRE(is_index(d->index_dtype), AGNES_ERR_INVALID, "classes and labels must be int32 or int64");
    AGNES_REQUIRE(d->classes || k == 0 || rows == 0, AGNES_ERR_INVALID, "classes must not be NULL");
    AGNES_REQUIRE(d->classes_stride >= 0, AGNES_ERR_INVALID, "classes_stride must not be negative");
    AGNES_REQUIRE(std::isfinite(d->temperature) && d->temperature > 0.f && std::isfinite(kLog2e / d->temperature),
                  AGNES_ERR_INVALID, "the temperature must be positive and finite, and so must log2(e) / temperature");
    AGNES_REQUIRE(std::isfinite(d->soft) && d->soft >= 0.f && std::isfinite(d->hard) && d->hard >= 0.f,
                  AGNES_ERR_INVALID, "soft and hard must be finite and not negative");
    DistillArgs a{};
    if (grad) {
        check_matrix(grad, true, "grad");
        AGNES_REQUIRE(grad->rows == rows && grad->cols == C, AGNES_ERR_INVALID, "grad must have the logits' shape");
        AGNES_REQUIRE(grad->data != d->logits.data || rows == 0 ||
                          (grad->dtype == d->logits.dtype && (rows == 1 || grad->stride == d->logits.stride)),
                      AGNES_ERR_INVALID, "grad may share the logits' memory only with their type and stride");
        a.grad = grad->data;
        a.gstride = grad->stride;
        a.gtype = grad->dtype;
        a.nt = rows * C * (int64_t)elem_size(grad->dtype) > kStreamBytes;
    }
    a.z = d->logits.data;
    a.t = d->teacher.data;
    a.ttype = d->teacher.dtype;
    a.classes = d->classes;
    a.labels = d->labels;
    a.weight = d->weight;
    a.wide = d->index_dtype == AGNES_INT64;
    a.zstride = d->logits.stride;
    a.tstride = d->teacher.stride;
    a.cstride = d->classes_stride;
    a.rows = rows;
    a.C = (int32_t)C;
    a.k = (int32_t)k;
    a.temp = d->temperature;
    a.ct = kLog2e / d->temperature;
    a.soft = d->soft;
    a.hard = d->labels ? d->hard : 0.f;
    return a;
}

// The n rows from row r on.
template <typename T> static DistillArgs rows_from(const DistillArgs& a, int64_t r, int64_t n) {
    DistillArgs b = a;
    b.z = (const T*)a.z + r * a.zstride;
    b.t = (const char*)a.t + r * a.tstride * (int64_t)elem_size(a.ttype);
    b.classes = (const char*)a.classes + r * a.cstride * (a.wide ? 8 : 4);
    if (a.labels) b.labels = (const char*)a.labels + r * (a.wide ? 8 : 4);
    if (a.weight) b.weight = a.weight + r;
    if (a.loss) b.loss = a.loss + r;
    if (a.stats) b.stats = a.stats + 3 * r;
    if (a.stats_in) b.stats_in = a.stats_in + 3 * r;
    if (a.grad) b.grad = (char*)a.grad + r * a.gstride * (int64_t)elem_size(a.gtype);
    b.rows = n;
    return b;
}

template <typename T, int MODE> static void launch(const DistillArgs& a, void* ws, hipStream_t st) {
    constexpr int E = 16 / (int)sizeof(T);
    const int64_t pieces = (a.C + E - 1) / E, rows = a.rows;
    if (pieces <= kLanePieces && a.k <= kLaneEntries) {
        // at least a lane per teacher entry: their comparisons grow with the entries of a lane
        int L = kLanesMin;
        while (L * 4 < pieces || L < a.k) L *= 2;
        const int P = pieces <= L ? 1 : pieces <= 2 * L ? 2 : 4;
        const int per = kBlock / L;
        const dim3 grid((unsigned)std::min<int64_t>((rows + per - 1) / per, kLaneGroups));
        const size_t lds = (size_t)kBlock * P * E * 4 + (size_t)per * 2 * a.k * 4;
        if (P == 1) AGNES_LAUNCH((k_distill_lanes<T, 1, MODE>), grid, dim3(kBlock), lds, st, a, L);
        else if (P == 2) AGNES_LAUNCH((k_distill_lanes<T, 2, MODE>), grid, dim3(kBlock), lds, st, a, L);
        else AGNES_LAUNCH((k_distill_lanes<T, 4, MODE>), grid, dim3(kBlock), lds, st, a, L);
        return;
    }
    int64_t span = 0;
    int parts = parts_of(rows, a.C, sizeof(T), span);
    if (a.stats_in && span == 0) {               // the gradient alone needs no sums: parts of any length do
        span = 4 * kPartThreads * E;
        parts = (int)((a.C + span - 1) / span);
    }
    if (span) {
        // blockIdx.y holds at most 65535 rows
        for (int64_t r = 0; r < rows; r += 65535) {
            const int64_t n = std::min<int64_t>(65535, rows - r);
            const DistillArgs b = rows_from<T>(a, r, n);
            Part* p = (Part*)ws + r * parts;
            const dim3 grid((unsigned)parts, (unsigned)n);
            if (!a.stats_in) AGNES_LAUNCH((k_distill_part<T, MODE>), grid, dim3(kPartThreads), 0, st, b, span, p);
            // without a gradient only a row's first part has anything to do
            AGNES_LAUNCH((k_distill_apply<T, MODE>), dim3(a.grad ? (unsigned)parts : 1u, (unsigned)n),
                         dim3(kPartThreads), 0, st, b, span, parts, (const Part*)p);
        }
        return;
    }
    for (int64_t r = 0; r < rows; r += kLaunchRows) {
        const int64_t n = std::min(kLaunchRows, rows - r);
        const DistillArgs b = rows_from<T>(a, r, n);
        const dim3 grid((unsigned)n);
        if (pieces <= 4 * 256) AGNES_LAUNCH((k_distill_block<T, 256, 4, MODE>), grid, dim3(256), 0, st, b);
        else if (pieces <= 8 * 256) AGNES_LAUNCH((k_distill_block<T, 256, 8, MODE>), grid, dim3(256), 0, st, b);
        else if (pieces <= 8 * 512) AGNES_LAUNCH((k_distill_block<T, 512, 8, MODE>), grid, dim3(512), 0, st, b);
        else if (pieces <= 8 * 1024) AGNES_LAUNCH((k_distill_block<T, 1024, 8, MODE>), grid, dim3(1024), 0, st, b);
        else AGNES_LAUNCH((k_distill_block<T, 1024, 16, MODE>), grid, dim3(1024), 0, st, b);
    }
}

static void run(const agnes_distill* d, const DistillArgs& a, void* ws, hipStream_t st) {
    if (a.rows == 0) return;
    with_float(d->logits.dtype, [&](auto t) {
        typedef decltype(t) T;
        // one exponential does for a single term, and for both at T = 1
        if (a.hard == 0.f || a.temp == 1.f) launch<T, kOne>(a, ws, st);
        else if (a.temp == 2.f) launch<T, kSquare>(a, ws, st);
        else launch<T, kTwo>(a, ws, st);
    });
}

void distill_loss(const agnes_distill* d, float* loss, float* stats, const agnes_matrix* grad, void* ws,
                  uint64_t ws_bytes, hipStream_t st) {
    DistillArgs a = check_distill(d, grad);
    AGNES_REQUIRE(loss || a.rows == 0, AGNES_ERR_INVALID, "loss must not be NULL");
    check_workspace(ws, ws_bytes, distill_bytes(a.rows, a.C));
    a.loss = loss;
    a.stats = stats;
    run(d, a, ws, st);
}

void distill_grad(const agnes_distill* d, const float* stats, const agnes_matrix* grad, hipStream_t st) {
    AGNES_REQUIRE(grad, AGNES_ERR_INVALID, "grad must not be NULL");
    DistillArgs a = check_distill(d, grad);
    AGNES_REQUIRE(stats || a.rows == 0, AGNES_ERR_INVALID, "stats must not be NULL");
    a.stats_in = stats;
    run(d, a, nullptr, st);
}

}  // namespace agnes
