// The clipped policy loss of drawn actions with a penalty for leaving a
// reference policy, and its gradient.
//
// With m = max_j z_j and S = sum_j exp((z_j - m) / T):
//   logp   = (z_y - m) / T - ln S,   r = exp(logp - old),   d = ref - logp
//   loss   = w [ -min(r A, clip(r) A) + kl (exp d - d - 1) ]
//   grad_j = g ([j = y] - exp((z_j - m) / T) / S),   g = w / T dL / dlogp
// Whether a row is clipped hangs on the last digits of logp, and exp d - d - 1
// cancels where the policies are close, so what a row needs once is computed
// in 64 bits; m, S and the gradient in 32.
//
// A row of logits is read once, stays in registers between its sum and its
// gradient, and its gradient is written once.  Variants, by the number of
// 16-byte pieces of a row:
//   up to 256      some lanes of a wave per row (a whole wave from 33 pieces on)
//   up to 16384    a workgroup of 256 to 1024 threads per row
//   above, or above 1024 with too few rows to fill the chip: the row is split
//     over workgroups; a first launch leaves each part's maximum and sum and the action's
//     logit, a second one joins them and writes the gradient (a second read of
//     the row).
// The gradient from statistics is the second launch alone, or the lanes' kernel.
// Bound by memory where there is enough of it: 8192 x 65536 bfloat16 375 us (5.7
// TB/s); 2048 x 47 float32 5.3 us, 8 x 100003 float16 4.9 us for the parts, 3.5 to join
// them for the loss and 6.8 for the gradient.
#include <algorithm>
#include <cmath>
#include <limits>

#include "logits.hpp"

namespace agnes {

// The descriptor as the kernels take it.
struct PolicyArgs {
    const void* z;
    const void* actions;
    const float *advantage, *old_logp, *ref_logp, *weight;
    const float* stats_in;         // the rows' statistics, or NULL: from the logits
    float *loss, *logp, *stats;
    void* grad;
    int64_t zstride, gstride, rows;
    int32_t C;
    agnes_dtype gtype;
    bool wide;                     // 64-bit actions
    bool nt;                       // gradient past the caches
    float temp, kl;                // T
    double low, high;              // 1 - clip_low, 1 + clip_high
    float ct, ct_low;              // log2(e) / T = ct + ct_low, both positive: exp(x / T) = 2^(x ct + x ct_low)
};

// exp(d / T) for d <= 0.  A single factor's rounding would move all of a row's terms,
// and with them its logp, one way; with positive parts -inf stays -inf.
__device__ __forceinline__ float exp_t(const PolicyArgs& a, float d) { return pow2(fmaf(d, a.ct, d * a.ct_low)); }

// What a row asks for, as loaded.
struct Decision {
    int64_t y;
    float w, A, old, ref;
};
__device__ __forceinline__ Decision load_decision(const PolicyArgs& a, int64_t r) {
    Decision d;
    d.y = load_index(a.actions, a.wide, r);
    d.w = a.weight ? a.weight[r] : 1.f;
    d.A = a.advantage ? a.advantage[r] : 0.f;
    d.old = a.old_logp ? a.old_logp[r] : 0.f;
    d.ref = a.ref_logp ? a.ref_logp[r] : 0.f;
    return d;
}
__device__ __forceinline__ bool skipped(const PolicyArgs& a, const Decision& d) {
    return d.w == 0.f || d.y < 0 || d.y >= a.C;
}

// What the row's largest logit, its sum and its action's logit give: the loss,
// logp and the gradient's factor g.
struct Outcome {
    float loss, logp, g;
};
__device__ __forceinline__ Outcome outcome(const PolicyArgs& a, const Decision& d, float m, float sum, float zy) {
    const double lp = zy == -INFINITY && sum == sum ? -INFINITY : ((double)zy - (double)m) / a.temp - log((double)sum);
    const bool never = lp == -INFINITY;          // the action cannot be drawn
    const double A = d.A, r = never ? 0.0 : exp(lp - (double)d.old);
    const double bound = A > 0.0 ? a.high : a.low;
    const bool clipped = (A > 0.0 && r > bound) || (A < 0.0 && r < bound);
    double loss = A == 0.0 ? 0.0 : -(clipped ? bound : r) * A;
    double slope = A == 0.0 || clipped ? 0.0 : -r * A;
    if (a.kl > 0.f) {
        const double away = (double)d.ref - lp, e = exp(away);
        loss += never ? INFINITY : a.kl * (e - 1.0 - away);
        slope += a.kl * (1.0 - e);
    }
    if (lp != lp) loss = slope = lp;             // also where the terms above need no logp
    return {(float)(d.w * loss), (float)lp, never ? 0.f : (float)(d.w * slope / a.temp)};
}

// E gradients from column c on, those before column hi, of the row whose first element is number `at`.
template <int E>
__device__ __forceinline__ void store_grad(const PolicyArgs& a, int64_t at, int c, int hi, const float (&x)[E]) {
    if (a.gtype == AGNES_FLOAT32) store_typed<E>((float*)a.grad + at, c, hi, x, a.nt);
    else if (a.gtype == AGNES_FLOAT16) store_typed<E>((_Float16*)a.grad + at, c, hi, x, a.nt);
    else store_typed<E>((__bf16*)a.grad + at, c, hi, x, a.nt);
}

// Maximum and sum of part of a row, relative to that maximum (to 0 where it is -inf).
struct Sum {
    float m, s;
};

// Adds E logits (-inf where there are none), none above x.m.  A NaN or +inf
// logit makes the sum NaN, and with it everything that follows.
template <int E, typename Raw> __device__ __forceinline__ void add_piece(const PolicyArgs& a, Sum& x, const Raw& v) {
    const float base = x.m == -INFINITY ? 0.f : x.m;
#pragma unroll
    for (int q = 0; q < E; q++) x.s += exp_t(a, (float)v[q] - base);
}
// Brings a sum to the maximum m of a larger part.
__device__ __forceinline__ void rebase(const PolicyArgs& a, Sum& x, float m) {
    if (m == -INFINITY) return;                    // the sum is 0 (or NaN)
    x.s *= exp_t(a, x.m - m);
    x.m = m;
}
__device__ __forceinline__ Sum lanes_join(const PolicyArgs& a, Sum x) {
    rebase(a, x, lanes_max(x.m, kWave));
    x.s = lanes_sum(x.s, kWave);
    return x;
}

// The gradient of logits [c, c + E): k = g / S.
template <int E, typename Raw>
__device__ __forceinline__ void grad_piece(const PolicyArgs& a, const Raw& v, int c, float m, float k, float g, int y, float (&x)[E]) {
#pragma unroll
    for (int q = 0; q < E; q++) {
        x[q] = -k * exp_t(a, (float)v[q] - m);
        if (c + q == y) x[q] += g;
    }
}

__device__ __forceinline__ void store_row(const PolicyArgs& a, int64_t r, const Outcome& o, float m, float s, float zy) {
    if (a.loss) a.loss[r] = o.loss;
    if (a.logp) a.logp[r] = o.logp;
    if (a.stats) {
        a.stats[3 * r] = m;
        a.stats[3 * r + 1] = s;
        a.stats[3 * r + 2] = zy;
    }
}

// ----------------------------------------------------------------- lanes of a wave per row

// L lanes per row, P pieces per lane; a group takes several rows and loads the
// next one before the present one's arithmetic.
constexpr int kLanesMin = 8;
constexpr int kLaneGroups = 2048;                // workgroups, about what the chip holds at once

template <typename T, int P> struct PolicyRow {
    typename Vec<T, 16 / (int)sizeof(T)>::type v[P];
    Decision d;
};

template <typename T, int P> __global__ __launch_bounds__(kBlock) void k_policy_lanes(PolicyArgs a, int L) {
    constexpr int E = 16 / (int)sizeof(T);
    const int groups = kBlock / L, g = threadIdx.x / L, gl = threadIdx.x % L;
    const int64_t step = (int64_t)gridDim.x * groups;
    int64_t r = (int64_t)blockIdx.x * groups + g;
    auto load = [&](int64_t i) {
        PolicyRow<T, P> x;
        const T* zr = (const T*)a.z + i * a.zstride;
#pragma unroll
        for (int p = 0; p < P; p++) x.v[p] = logits_piece<T, E>(zr, (gl + p * L) * E, a.C);
        x.d = load_decision(a, i);
        return x;
    };
    PolicyRow<T, P> next;
    if (r < a.rows) next = load(r);
    for (; r < a.rows; r += step) {                         // per group; nothing below crosses a group
        PolicyRow<T, P> x = next;
        if (r + step < a.rows) next = load(r + step);
        const int64_t at = r * a.gstride;
        if (skipped(a, x.d)) {
            if (gl == 0) store_row(a, r, Outcome{0.f, 0.f, 0.f}, 0.f, 0.f, 0.f);
            if (a.grad) {
                const float zero[E] = {};
#pragma unroll
                for (int p = 0; p < P; p++) store_grad<E>(a, at, (gl + p * L) * E, a.C, zero);
            }
            continue;
        }
        const int y = (int)x.d.y;
        Sum s{-INFINITY, 0.f};
        float zy;
        if (a.stats_in) {
            s = Sum{a.stats_in[3 * r], a.stats_in[3 * r + 1]};
            zy = a.stats_in[3 * r + 2];
        } else {
            uint32_t named = 0;                             // the action's logit, in the lane that holds it
#pragma unroll
            for (int p = 0; p < P; p++)
#pragma unroll
                for (int e = 0; e < E; e++) {
                    const float z = (float)x.v[p][e];
                    s.m = fmaxf(s.m, z);
                    if ((gl + p * L) * E + e == y) named = __float_as_uint(z);
                }
            s.m = lanes_max(s.m, L);
#pragma unroll
            for (int p = 0; p < P; p++) {
                keep_packed(x.v[p]);
                add_piece<E>(a, s, x.v[p]);
                __builtin_amdgcn_sched_barrier(0);
            }
            s.s = lanes_sum(s.s, L);
            zy = lanes_reduce(__uint_as_float(named), L, [](float u, float v) {
                return __uint_as_float(__float_as_uint(u) | __float_as_uint(v));
            });
        }
        const Outcome o = outcome(a, x.d, s.m, s.s, zy);
        if (gl == 0) store_row(a, r, o, s.m, s.s, zy);
        if (!a.grad) continue;
        const float k = o.g == 0.f ? 0.f : o.g / s.s;
#pragma unroll
        for (int p = 0; p < P; p++) {
            float w[E] = {};
            keep_packed(x.v[p]);
            if (o.g != 0.f) grad_piece<E>(a, x.v[p], (gl + p * L) * E, s.m, k, o.g, y, w);
            store_grad<E>(a, at, (gl + p * L) * E, a.C, w);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// ----------------------------------------------------------------- a workgroup per row

template <typename T, int THREADS, int P>
__global__ __launch_bounds__(THREADS, THREADS == 1024 && P == 8 ? 8 : 4) void k_policy_block(PolicyArgs a) {
    constexpr int E = 16 / (int)sizeof(T), WAVES = THREADS / kWave;
    typedef typename Vec<T, E>::type Raw;
    __shared__ Sum red[WAVES];
    __shared__ float named;
    const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;
    const int64_t r = blockIdx.x;
    const T* zr = (const T*)a.z + r * a.zstride;
    const int64_t at = r * a.gstride;
    const Decision d = load_decision(a, r);
    if (skipped(a, d)) {
        if (tid == 0) store_row(a, r, Outcome{0.f, 0.f, 0.f}, 0.f, 0.f, 0.f);
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
    if (tid == 0) named = to_float(zr[d.y]);       // read before anything is stored, also where grad is over the logits
    Sum s{-INFINITY, 0.f};
#pragma unroll
    for (int i = 0; i < P; i++)
        if (i * THREADS * E < a.C) {
#pragma unroll
            for (int x = 0; x < E; x++) s.m = fmaxf(s.m, (float)v[i][x]);
        }
    s.m = lanes_max(s.m, kWave);
#pragma unroll
    for (int i = 0; i < P; i++)
        if (i * THREADS * E < a.C) {               // no work for rounds that lie behind the row
            keep_packed(v[i]);
            add_piece<E>(a, s, v[i]);
            __builtin_amdgcn_sched_barrier(0);     // one piece's values at a time: registers decide the occupancy
        }
    s.s = lanes_sum(s.s, kWave);
    if (lane == 0) red[wave] = s;
    __syncthreads();
    s = lane < WAVES ? red[lane] : Sum{-INFINITY, 0.f};
    s = lanes_join(a, s);
    const Outcome o = outcome(a, d, s.m, s.s, named);
    if (tid == 0) store_row(a, r, o, s.m, s.s, named);
    if (!a.grad) return;
    const float k = o.g == 0.f ? 0.f : o.g / s.s;
#pragma unroll
    for (int i = 0; i < P; i++) {
        if (i * THREADS * E < a.C) {
            const int c = (tid + i * THREADS) * E;
            float x[E] = {};
            keep_packed(v[i]);
            if (o.g != 0.f) grad_piece<E>(a, v[i], c, s.m, k, o.g, (int)d.y, x);
            store_grad<E>(a, at, c, a.C, x);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// ----------------------------------------------------------------- a row over several workgroups

// Part of a row: its maximum and sum, and the action's logit if it lies in it (else 0).
struct PolicyPart {
    float m, s, zy, pad;
};

constexpr int kPartThreads = 256;

// blockIdx: (part, row).  A part is `span` logits, a multiple of a piece.
template <typename T>
__global__ __launch_bounds__(kPartThreads) void k_policy_part(PolicyArgs a, int64_t span, PolicyPart* __restrict__ parts) {
    constexpr int E = 16 / (int)sizeof(T), U = 4;
    typedef typename Vec<T, E>::type Raw;
    __shared__ Sum red[kPartThreads / kWave];
    const int tid = threadIdx.x, lane = lane_id(), wave = wave_id();
    const int64_t r = blockIdx.y;
    const T* zr = (const T*)a.z + r * a.zstride;
    const Decision d = load_decision(a, r);
    if (skipped(a, d)) return;                     // the second launch skips the row too
    const int lo = (int)(blockIdx.x * span), hi = (int)min((int64_t)a.C, lo + span);
    Sum s{-INFINITY, 0.f};
    for (int c0 = lo; c0 < hi; c0 += kPartThreads * E * U) {
        Raw v[U];
#pragma unroll
        for (int i = 0; i < U; i++) v[i] = logits_piece<T, E>(zr, c0 + (tid + i * kPartThreads) * E, hi);
        float m = s.m;
#pragma unroll
        for (int i = 0; i < U; i++)
#pragma unroll
            for (int x = 0; x < E; x++) m = fmaxf(m, (float)v[i][x]);
        rebase(a, s, m);
#pragma unroll
        for (int i = 0; i < U; i++) add_piece<E>(a, s, v[i]);
    }
    s = lanes_join(a, s);
    if (lane == 0) red[wave] = s;
    __syncthreads();
    if (wave != 0) return;
    s = lane < kPartThreads / kWave ? red[lane] : Sum{-INFINITY, 0.f};
    s = lanes_join(a, s);
    if (lane == 0) {
        const float zy = d.y >= lo && d.y < hi ? to_float(zr[d.y]) : 0.f;
        parts[r * gridDim.x + blockIdx.x] = PolicyPart{s.m, s.s, zy, 0.f};
    }
}

// The row's sum from its parts (or from stats_in), then the loss, by the first
// workgroup, and the gradient of [lo, hi).  The action's logit comes with them:
// where grad is over the logits another workgroup may have written there.
template <typename T>
__global__ __launch_bounds__(kPartThreads) void k_policy_apply(PolicyArgs a, int64_t span, int nparts, const PolicyPart* __restrict__ parts) {
    constexpr int E = 16 / (int)sizeof(T), U = 4;
    typedef typename Vec<T, E>::type Raw;
    const int tid = threadIdx.x, lane = lane_id();
    const int64_t r = blockIdx.y;
    const T* zr = (const T*)a.z + r * a.zstride;
    const int64_t at = r * a.gstride;
    const int lo = (int)(blockIdx.x * span), hi = (int)min((int64_t)a.C, lo + span);
    const bool first = blockIdx.x == 0;
    const Decision d = load_decision(a, r);
    if (skipped(a, d)) {
        if (first && tid == 0) store_row(a, r, Outcome{0.f, 0.f, 0.f}, 0.f, 0.f, 0.f);
        if (a.grad) {
            const float zero[E] = {};
            for (int c = lo + tid * E; c < hi; c += kPartThreads * E) store_grad<E>(a, at, c, hi, zero);
        }
        return;
    }
    Raw v[U];
    if (a.grad) {                                  // on their way while the parts are joined
#pragma unroll
        for (int i = 0; i < U; i++) v[i] = logits_piece<T, E>(zr, lo + (tid + i * kPartThreads) * E, hi);
    }
    Sum s{-INFINITY, 0.f};
    float zy = 0.f;
    if (a.stats_in) {
        s = Sum{a.stats_in[3 * r], a.stats_in[3 * r + 1]};
        zy = a.stats_in[3 * r + 2];
    } else {
        const PolicyPart* p = parts + r * nparts;
        for (int i = lane; i < nparts; i += kWave) s.m = fmaxf(s.m, p[i].m);
        s.m = lanes_max(s.m, kWave);
        for (int i = lane; i < nparts; i += kWave) {
            Sum x{p[i].m, p[i].s};
            rebase(a, x, s.m);
            s.s += x.s;
        }
        s.s = lanes_sum(s.s, kWave);
        zy = p[d.y / span].zy;
    }
    const Outcome o = outcome(a, d, s.m, s.s, zy);
    if (first && tid == 0) store_row(a, r, o, s.m, s.s, zy);
    if (!a.grad) return;
    const float k = o.g == 0.f ? 0.f : o.g / s.s;
    for (int c0 = lo; c0 < hi; c0 += kPartThreads * E * U) {
        if (c0 != lo) {
#pragma unroll
            for (int i = 0; i < U; i++) v[i] = logits_piece<T, E>(zr, c0 + (tid + i * kPartThreads) * E, hi);
        }
#pragma unroll
        for (int i = 0; i < U; i++) {
            const int c = c0 + (tid + i * kPartThreads) * E;
            float x[E] = {};
            if (o.g != 0.f) grad_piece<E>(a, v[i], c, s.m, k, o.g, (int)d.y, x);
            store_grad<E>(a, at, c, hi, x);
        }
    }
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

uint64_t policy_bytes(int64_t rows, int64_t classes) {
    AGNES_REQUIRE(rows >= 0 && classes >= 0 && rows < ((int64_t)1 << 31) && classes < ((int64_t)1 << 31),
                  AGNES_ERR_INVALID, "rows and classes must be in [0, 2^31)");
    if (rows == 0 || classes == 0) return 0;
    int64_t span = 0, most = 0;
    for (int64_t size : {2, 4}) {                // either size of logits
        const int n = parts_of(rows, classes, size, span);
        if (span) most = std::max<int64_t>(most, rows * n * (int64_t)sizeof(PolicyPart));
    }
    return (uint64_t)most;
}

static PolicyArgs check_policy(const agnes_policy* p, bool alone, const agnes_matrix* grad) {
    AGNES_REQUIRE(p, AGNES_ERR_INVALID, "the descriptor must not be NULL");
    check_matrix(&p->logits, false, "logits");
    const int64_t rows = p->logits.rows, C = p->logits.cols;
    AGNES_REQUIRE(C >= 1, AGNES_ERR_INVALID, "there must be at least one class");
    AGNES_REQUIRE(C < ((int64_t)1 << 31) - (1 << 16), AGNES_ERR_INVALID, "there must be fewer than 2^31 - 2^16 classes");
    AGNES_REQUIRE(is_index(p->index_dtype), AGNES_ERR_INVALID, "actions must be int32 or int64");
    AGNES_REQUIRE(p->actions || rows == 0, AGNES_ERR_INVALID, "actions must not be NULL");
    AGNES_REQUIRE(std::isfinite(p->temperature) && p->temperature > 0.f && std::isfinite(kLog2e / p->temperature),
                  AGNES_ERR_INVALID, "the temperature must be positive and finite, and so must log2(e) / temperature");
    PolicyArgs a{};
    if (!alone) {
        AGNES_REQUIRE((p->advantage && p->old_logp) || rows == 0, AGNES_ERR_INVALID,
                      "advantage and old_logp must not be NULL");
        AGNES_REQUIRE(std::isfinite(p->clip_low) && p->clip_low >= 0.f && p->clip_low <= 1.f, AGNES_ERR_INVALID,
                      "clip_low must be in [0, 1]");
        AGNES_REQUIRE(std::isfinite(p->clip_high) && p->clip_high >= 0.f, AGNES_ERR_INVALID,
                      "clip_high must be finite and not negative");
        AGNES_REQUIRE(std::isfinite(p->kl) && p->kl >= 0.f, AGNES_ERR_INVALID, "kl must be finite and not negative");
        AGNES_REQUIRE(p->ref_logp || p->kl == 0.f || rows == 0, AGNES_ERR_INVALID, "kl > 0 needs ref_logp");
        a.advantage = p->advantage;
        a.old_logp = p->old_logp;
        a.ref_logp = p->kl > 0.f ? p->ref_logp : nullptr;
        a.low = 1.0 - (double)p->clip_low;
        a.high = 1.0 + (double)p->clip_high;
        a.kl = p->kl;
    }
    if (grad) {
        check_matrix(grad, true, "grad");
        AGNES_REQUIRE(grad->rows == rows && grad->cols == C, AGNES_ERR_INVALID, "grad must have the logits' shape");
        AGNES_REQUIRE(grad->data != p->logits.data || rows == 0 ||
                          (grad->dtype == p->logits.dtype && (rows == 1 || grad->stride == p->logits.stride)),
                      AGNES_ERR_INVALID, "grad may share the logits' memory only with their type and stride");
        a.grad = grad->data;
        a.gstride = grad->stride;
        a.gtype = grad->dtype;
        a.nt = rows * C * (int64_t)elem_size(grad->dtype) > kStreamBytes;
    }
    a.z = p->logits.data;
    a.actions = p->actions;
    a.weight = p->weight;
    a.wide = p->index_dtype == AGNES_INT64;
    a.zstride = p->logits.stride;
    a.rows = rows;
    a.C = (int32_t)C;
    a.temp = p->temperature;
    const double ct = M_LOG2E / (double)p->temperature;
    a.ct = (float)ct;
    if (a.ct > ct) a.ct = std::nextafter(a.ct, 0.f);
    a.ct_low = std::max((float)(ct - a.ct), std::numeric_limits<float>::denorm_min());
    return a;
}

// The n rows from row r on.
template <typename T> static PolicyArgs rows_from(const PolicyArgs& a, int64_t r, int64_t n) {
    PolicyArgs b = a;
    b.z = (const T*)a.z + r * a.zstride;
    b.actions = (const char*)a.actions + r * (a.wide ? 8 : 4);
    for (const float** p : {&b.advantage, &b.old_logp, &b.ref_logp, &b.weight})
        if (*p) *p += r;
    if (a.stats_in) b.stats_in = a.stats_in + 3 * r;
    if (a.loss) b.loss = a.loss + r;
    if (a.logp) b.logp = a.logp + r;
    if (a.stats) b.stats = a.stats + 3 * r;
    if (a.grad) b.grad = (char*)a.grad + r * a.gstride * (int64_t)elem_size(a.gtype);
    b.rows = n;
    return b;
}

template <typename T> static void launch(const PolicyArgs& a, void* ws, hipStream_t st) {
    constexpr int E = 16 / (int)sizeof(T);
    const int64_t pieces = (a.C + E - 1) / E, rows = a.rows;
    if (pieces <= kLanePieces) {
        int L = kLanesMin;
        while (L * 4 < pieces) L *= 2;
        const int per = kBlock / L;
        const dim3 grid((unsigned)std::min<int64_t>((rows + per - 1) / per, kLaneGroups));
        if (pieces <= L) AGNES_LAUNCH((k_policy_lanes<T, 1>), grid, dim3(kBlock), 0, st, a, L);
        else if (pieces <= 2 * L) AGNES_LAUNCH((k_policy_lanes<T, 2>), grid, dim3(kBlock), 0, st, a, L);
        else AGNES_LAUNCH((k_policy_lanes<T, 4>), grid, dim3(kBlock), 0, st, a, L);
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
            const PolicyArgs b = rows_from<T>(a, r, n);
            PolicyPart* p = (PolicyPart*)ws + r * parts;
            const dim3 grid((unsigned)parts, (unsigned)n);
            if (!a.stats_in) AGNES_LAUNCH((k_policy_part<T>), grid, dim3(kPartThreads), 0, st, b, span, p);
            // without a gradient only a row's first part has anything to do
            AGNES_LAUNCH((k_policy_apply<T>), dim3(a.grad ? (unsigned)parts : 1u, (unsigned)n), dim3(kPartThreads), 0, st, b,
                         span, parts, (const PolicyPart*)p);
        }
        return;
    }
    for (int64_t r = 0; r < rows; r += kLaunchRows) {
        const int64_t n = std::min(kLaunchRows, rows - r);
        const PolicyArgs b = rows_from<T>(a, r, n);
        const dim3 grid((unsigned)n);
        if (pieces <= 4 * 256) AGNES_LAUNCH((k_policy_block<T, 256, 4>), grid, dim3(256), 0, st, b);
        else if (pieces <= 8 * 256) AGNES_LAUNCH((k_policy_block<T, 256, 8>), grid, dim3(256), 0, st, b);
        else if (pieces <= 8 * 512) AGNES_LAUNCH((k_policy_block<T, 512, 8>), grid, dim3(512), 0, st, b);
        else if (pieces <= 8 * 1024) AGNES_LAUNCH((k_policy_block<T, 1024, 8>), grid, dim3(1024), 0, st, b);
        else AGNES_LAUNCH((k_policy_block<T, 1024, 16>), grid, dim3(1024), 0, st, b);
    }
}

static void run(agnes_dtype t, const PolicyArgs& a, void* ws, hipStream_t st) {
    if (a.rows == 0) return;
    with_float(t, [&](auto v) { launch<decltype(v)>(a, ws, st); });
}

void policy_logprob(const agnes_policy* p, float* logp, void* ws, uint64_t ws_bytes, hipStream_t st) {
    PolicyArgs a = check_policy(p, true, nullptr);
    AGNES_REQUIRE(logp || a.rows == 0, AGNES_ERR_INVALID, "logp must not be NULL");
    check_workspace(ws, ws_bytes, policy_bytes(a.rows, a.C));
    a.logp = logp;
    run(p->logits.dtype, a, ws, st);
}

void policy_loss(const agnes_policy* p, float* loss, float* logp, float* stats, const agnes_matrix* grad, void* ws,
                 uint64_t ws_bytes, hipStream_t st) {
    PolicyArgs a = check_policy(p, false, grad);
    AGNES_REQUIRE((loss && logp) || a.rows == 0, AGNES_ERR_INVALID, "loss and logp must not be NULL");
    check_workspace(ws, ws_bytes, policy_bytes(a.rows, a.C));
    a.loss = loss;
    a.logp = logp;
    a.stats = stats;
    run(p->logits.dtype, a, ws, st);
}

void policy_grad(const agnes_policy* p, const float* stats, const agnes_matrix* grad, hipStream_t st) {
    AGNES_REQUIRE(grad, AGNES_ERR_INVALID, "grad must not be NULL");
    PolicyArgs a = check_policy(p, false, grad);
    AGNES_REQUIRE(stats || a.rows == 0, AGNES_ERR_INVALID, "stats must not be NULL");
    a.stats_in = stats;
    run(p->logits.dtype, a, nullptr, st);
}

}  // namespace agnes
