// Loss of a student's logits against a teacher's top logits, and its gradient.
//
// With m = max_j z_j, S_T = sum_j exp((z_j - m) / T) and S_1 = sum_j exp(z_j - m):
//   ln q_j = (z_j - m) / T - ln S_T
//   loss   = w [ a T^2 sum_e p_e (ln p_e - ln q_{c_e}) + b (ln S_1 - (z_y - m)) ]
//   grad_j = w [ a T (P q_j - sum_{c_e = j} p_e) + b (exp(z_j - m) / S_1 - [j = y]) ]
// p is the softmax of the row's valid teacher logits, P = 1 if there are any.
#include <algorithm>
#include <cmath>

#include "ops.hpp"

namespace agnes {

// The descriptor as the kernels take it.
struct DistillArgs {
    const void* classes;
    const void* labels;
    const float* weight;
    int64_t zstride, tstride, cstride;
    int64_t rows;
    int32_t C, k;
    float inv_t, soft, hard;       // 1 / T, a, b
    float temp;
};

__device__ __forceinline__ float block_max(float x, float* lds) {
    for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d, kWave));
    __syncthreads();
    if (lane_id() == 0) lds[wave_id()] = x;
    __syncthreads();
    float r = lds[0];
    for (int w = 1; w < kWavesPerBlock; w++) r = fmaxf(r, lds[w]);
    return r;
}

__device__ __forceinline__ float block_sum(float x, float* lds) {
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, kWave);
    __syncthreads();
    if (lane_id() == 0) lds[wave_id()] = x;
    __syncthreads();
    float r = lds[0];
    for (int w = 1; w < kWavesPerBlock; w++) r += lds[w];
    return r;
}

// One workgroup per row, three passes over it: maximum, sums, gradient.
// stats_in: take the row's statistics from there.
template <typename T, typename TT, typename TG, typename IdT>
__global__ __launch_bounds__(kBlock) void k_distill(const T* z, const TT* __restrict__ t, DistillArgs a,
                                                    const float* __restrict__ stats_in, float* __restrict__ loss,
                                                    float* __restrict__ stats, TG* grad, int64_t gstride) {
    __shared__ float lds[kWavesPerBlock];
    __shared__ int32_t cls[AGNES_DISTILL_MAX_K];
    __shared__ float prob[AGNES_DISTILL_MAX_K];
    const int64_t r = blockIdx.x;
    const T* zr = z + r * a.zstride;
    TG* gr = grad + r * gstride;
    const int C = a.C, tid = threadIdx.x;
    const float w = a.weight ? a.weight[r] : 1.f;
    if (w == 0.f) {
        if (tid == 0 && loss) loss[r] = 0.f;
        if (tid == 0 && stats) stats[3 * r] = stats[3 * r + 1] = stats[3 * r + 2] = 0.f;
        if (grad)
            for (int64_t j = tid; j < C; j += kBlock) gr[j] = from_float<TG>(0.f);
        return;
    }
    // the teacher's distribution
    float tm = -INFINITY;
    for (int e = tid; e < a.k; e += kBlock) {
        const int64_t c = (int64_t)((const IdT*)a.classes)[r * a.cstride + e];
        const bool ok = c >= 0 && c < C;
        const float x = ok ? to_float(t[r * a.tstride + e]) * a.inv_t : -INFINITY;
        cls[e] = ok ? (int)c : -1;
        prob[e] = x;
        tm = x > tm || x != x ? x : tm;
    }
    const bool tnan = block_sum(tm != tm ? 1.f : 0.f, lds) > 0.f;
    tm = tnan ? NAN : block_max(tm, lds);
    const bool some = !(tm == -INFINITY) && a.soft > 0.f;
    float ts = 0.f;
    if (some)
        for (int e = tid; e < a.k; e += kBlock) ts += expf(prob[e] - tm);
    ts = block_sum(ts, lds);
    const int64_t y = a.labels ? (int64_t)((const IdT*)a.labels)[r] : -1;
    const bool named = y >= 0 && y < C && a.hard > 0.f;
    // the student's statistics
    float m, st, s1;
    if (stats_in) {
        m = stats_in[3 * r];
        st = stats_in[3 * r + 1];
        s1 = stats_in[3 * r + 2];
    } else {
        float x = -INFINITY, bad = 0.f;
        for (int64_t j = tid; j < C; j += kBlock) {
            const float v = to_float(zr[j]);
            if (v != v) bad = 1.f;
            x = fmaxf(x, v);
        }
        m = block_sum(bad, lds) > 0.f ? NAN : block_max(x, lds);
        float u = 0.f, v = 0.f;
        if (m != -INFINITY)
            for (int64_t j = tid; j < C; j += kBlock) {
                const float d = to_float(zr[j]) - m;
                u += expf(d * a.inv_t);
                v += expf(d);
            }
        st = block_sum(u, lds);
        s1 = block_sum(v, lds);
    }
    const bool empty = m == -INFINITY;             // every logit is -inf
    const float lt = logf(st), l1 = logf(s1), ltt = logf(ts);
    float part = 0.f;
    for (int e = tid; e < a.k; e += kBlock) {
        float p = 0.f;
        if (some) {
            const float x = prob[e] - tm;
            p = expf(x) / ts;
            if (p != 0.f) {
                const float lnq = empty ? -INFINITY : (to_float(zr[cls[e]]) - m) * a.inv_t - lt;
                part += p * ((x - ltt) - lnq);
            }
        }
        prob[e] = p;
    }
    part = block_sum(part, lds);
    if (tid == 0) {
        if (loss) {
            float L = some ? a.soft * a.temp * a.temp * part : 0.f;
            if (named) L += a.hard * (empty ? INFINITY : l1 - (to_float(zr[y]) - m));
            loss[r] = w * L;
        }
        if (stats) {
            stats[3 * r] = m;
            stats[3 * r + 1] = st;
            stats[3 * r + 2] = s1;
        }
    }
    if (!grad) return;
    __syncthreads();                                // prob is complete
    const float ca = some ? w * a.soft * a.temp : 0.f, cb = named ? w * a.hard : 0.f;
    for (int64_t j = tid; j < C; j += kBlock) {
        if (empty) {
            gr[j] = from_float<TG>(0.f);
            continue;
        }
        const float d = to_float(zr[j]) - m;
        float x = 0.f;
        if (some) {
            float p = 0.f;
            for (int e = 0; e < a.k; e++)
                if (cls[e] == j) p += prob[e];
            x += ca * (expf(d * a.inv_t) / st - p);
        }
        if (named) x += cb * (expf(d) / s1 - (j == y ? 1.f : 0.f));
        gr[j] = from_float<TG>(x);
    }
}

uint64_t distill_bytes(int64_t rows, int64_t classes) {
    AGNES_REQUIRE(rows >= 0 && classes >= 0 && rows < ((int64_t)1 << 31) && classes < ((int64_t)1 << 31),
                  AGNES_ERR_INVALID, "rows and classes must be in [0, 2^31)");
    return 0;
}

static DistillArgs check_distill(const agnes_distill* d, const agnes_matrix* grad) {
    AGNES_REQUIRE(d, AGNES_ERR_INVALID, "the descriptor must not be NULL");
    check_matrix(&d->logits, false, "logits");
    check_matrix(&d->teacher, false, "teacher");
    const int64_t rows = d->logits.rows, C = d->logits.cols, k = d->teacher.cols;
    AGNES_REQUIRE(C >= 1, AGNES_ERR_INVALID, "there must be at least one class");
    AGNES_REQUIRE(d->teacher.rows == rows, AGNES_ERR_INVALID, "teacher and logits must have equal rows");
    AGNES_REQUIRE(k <= AGNES_DISTILL_MAX_K, AGNES_ERR_INVALID, "the teacher may have at most 1024 entries per row");
    AGNES_REQUIRE(is_index(d->index_dtype), AGNES_ERR_INVALID, "classes and labels must be int32 or int64");
    AGNES_REQUIRE(d->classes || k == 0 || rows == 0, AGNES_ERR_INVALID, "classes must not be NULL");
    AGNES_REQUIRE(d->classes_stride >= 0, AGNES_ERR_INVALID, "classes_stride must not be negative");
    AGNES_REQUIRE(std::isfinite(d->temperature) && d->temperature > 0.f && std::isfinite(1.f / d->temperature),
                  AGNES_ERR_INVALID, "the temperature must be positive and finite");
    AGNES_REQUIRE(std::isfinite(d->soft) && d->soft >= 0.f && std::isfinite(d->hard) && d->hard >= 0.f,
                  AGNES_ERR_INVALID, "soft and hard must be finite and not negative");
    if (grad) {
        check_matrix(grad, true, "grad");
        AGNES_REQUIRE(grad->rows == rows && grad->cols == C, AGNES_ERR_INVALID, "grad must have the logits' shape");
        AGNES_REQUIRE(grad->data != d->logits.data || rows == 0 ||
                          (grad->dtype == d->logits.dtype && (rows == 1 || grad->stride == d->logits.stride)),
                      AGNES_ERR_INVALID, "grad may share the logits' memory only with their type and stride");
    }
    DistillArgs a{};
    a.classes = d->classes;
    a.labels = d->labels;
    a.weight = d->weight;
    a.zstride = d->logits.stride;
    a.tstride = d->teacher.stride;
    a.cstride = d->classes_stride;
    a.rows = rows;
    a.C = (int32_t)C;
    a.k = (int32_t)k;
    a.temp = d->temperature;
    a.inv_t = 1.f / d->temperature;
    a.soft = d->soft;
    a.hard = d->hard;
    return a;
}

static void launch(const agnes_distill* d, const DistillArgs& a, const float* stats_in, float* loss, float* stats,
                   const agnes_matrix* grad, hipStream_t st) {
    if (a.rows == 0) return;
    with_float(d->logits.dtype, [&](auto tz) {
        with_float(d->teacher.dtype, [&](auto tt) {
            with_float(grad ? grad->dtype : d->logits.dtype, [&](auto tg) {
                with_index(d->index_dtype, [&](auto id) {
                    typedef decltype(tz) TZ;
                    typedef decltype(tt) TT;
                    typedef decltype(tg) TG;
                    typedef decltype(id) IdT;
                    AGNES_LAUNCH((k_distill<TZ, TT, TG, IdT>), dim3((unsigned)a.rows), dim3(kBlock), 0, st,
                                 (const TZ*)d->logits.data, (const TT*)d->teacher.data, a, stats_in, loss, stats,
                                 grad ? (TG*)grad->data : nullptr, grad ? grad->stride : 0);
                });
            });
        });
    });
}

void distill_loss(const agnes_distill* d, float* loss, float* stats, const agnes_matrix* grad, void* ws,
                  uint64_t ws_bytes, hipStream_t st) {
    const DistillArgs a = check_distill(d, grad);
    AGNES_REQUIRE(loss || a.rows == 0, AGNES_ERR_INVALID, "loss must not be NULL");
    check_workspace(ws, ws_bytes, distill_bytes(a.rows, a.C));
    launch(d, a, nullptr, loss, stats, grad, st);
}

void distill_grad(const agnes_distill* d, const float* stats, const agnes_matrix* grad, hipStream_t st) {
    AGNES_REQUIRE(grad, AGNES_ERR_INVALID, "grad must not be NULL");
    const DistillArgs a = check_distill(d, grad);
    AGNES_REQUIRE(stats || a.rows == 0, AGNES_ERR_INVALID, "stats must not be NULL");
    launch(d, a, stats, nullptr, nullptr, grad, st);
}

}  // namespace agnes
