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
#include <algorithm>
#include <cmath>

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
    float ct;                      // log2(e) / T: exp(x / T) = 2^(x ct)
};

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

// A workgroup per row, which it reads for the maximum, for the sum and for the gradient.
template <typename T> __global__ __launch_bounds__(kBlock) void k_policy_row(PolicyArgs a) {
    __shared__ float red[kWavesPerBlock];
    const int64_t r = blockIdx.x;
    const T* zr = (const T*)a.z + r * a.zstride;
    const Decision d = load_decision(a, r);
    const int tid = threadIdx.x;
    if (skipped(a, d)) {
        if (tid == 0) {
            if (a.loss) a.loss[r] = 0.f;
            if (a.logp) a.logp[r] = 0.f;
            if (a.stats) a.stats[2 * r] = a.stats[2 * r + 1] = 0.f;
        }
        if (a.grad)
            for (int64_t c = tid; c < a.C; c += kBlock) store_any(a.grad, a.gtype, r * a.gstride + c, 0.f);
        return;
    }
    const float zy = to_float(zr[d.y]);
    float m = -INFINITY, s = 0.f;
    if (a.stats_in) {
        m = a.stats_in[2 * r];
        s = a.stats_in[2 * r + 1];
        __syncthreads();                         // zy is read before the gradient is stored
    } else {
        for (int64_t c = tid; c < a.C; c += kBlock) m = fmaxf(m, to_float(zr[c]));
        m = lanes_max(m, kWave);
        if (lane_id() == 0) red[wave_id()] = m;
        __syncthreads();
        for (int w = 0; w < kWavesPerBlock; w++) m = fmaxf(m, red[w]);
        __syncthreads();
        const float base = m == -INFINITY ? 0.f : m;
        for (int64_t c = tid; c < a.C; c += kBlock) s += pow2((to_float(zr[c]) - base) * a.ct);
        s = lanes_sum(s, kWave);
        if (lane_id() == 0) red[wave_id()] = s;
        __syncthreads();
        s = 0.f;
        for (int w = 0; w < kWavesPerBlock; w++) s += red[w];
    }
    const Outcome o = outcome(a, d, m, s, zy);
    if (tid == 0) {
        if (a.loss) a.loss[r] = o.loss;
        if (a.logp) a.logp[r] = o.logp;
        if (a.stats) {
            a.stats[2 * r] = m;
            a.stats[2 * r + 1] = s;
        }
    }
    if (!a.grad) return;
    const float k = o.g == 0.f ? 0.f : o.g / s;
    for (int64_t c = tid; c < a.C; c += kBlock) {
        float x = 0.f;
        if (o.g != 0.f) {
            x = -k * pow2((to_float(zr[c]) - m) * a.ct);
            if (c == d.y) x += o.g;
        }
        store_any(a.grad, a.gtype, r * a.gstride + c, x);
    }
}

// ----------------------------------------------------------------- host

constexpr int64_t kLaunchRows = 1 << 21;         // rows per launch of a workgroup each: a launch holds fewer than 2^32 threads

uint64_t policy_bytes(int64_t rows, int64_t classes) {
    AGNES_REQUIRE(rows >= 0 && classes >= 0 && rows < ((int64_t)1 << 31) && classes < ((int64_t)1 << 31),
                  AGNES_ERR_INVALID, "rows and classes must be in [0, 2^31)");
    return 0;
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
    a.ct = kLog2e / p->temperature;
    return a;
}

// The n rows from row r on.
template <typename T> static PolicyArgs rows_from(const PolicyArgs& a, int64_t r, int64_t n) {
    PolicyArgs b = a;
    b.z = (const T*)a.z + r * a.zstride;
    b.actions = (const char*)a.actions + r * (a.wide ? 8 : 4);
    for (const float** p : {&b.advantage, &b.old_logp, &b.ref_logp, &b.weight})
        if (*p) *p += r;
    if (a.stats_in) b.stats_in = a.stats_in + 2 * r;
    if (a.loss) b.loss = a.loss + r;
    if (a.logp) b.logp = a.logp + r;
    if (a.stats) b.stats = a.stats + 2 * r;
    if (a.grad) b.grad = (char*)a.grad + r * a.gstride * (int64_t)elem_size(a.gtype);
    b.rows = n;
    return b;
}

template <typename T> static void launch(const PolicyArgs& a, void* ws, hipStream_t st) {
    for (int64_t r = 0; r < a.rows; r += kLaunchRows) {
        const int64_t n = std::min(kLaunchRows, a.rows - r);
        AGNES_LAUNCH(k_policy_row<T>, dim3((unsigned)n), dim3(kBlock), 0, st, rows_from<T>(a, r, n));
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
