// Embedding lookup and its gradient.
//
// Lookup: out[i] = scale * table[ids[i]].  Gradient: dTable[v] = scale * sum of
// grad_out[i] over the i with ids[i] = v, ascending in i.  The ids are sorted
// stably, so a table row's contributions form one run of the sorted list, and
// each run is summed in its order: no atomics, the same bits on every run.
#include <algorithm>

#include "ops.hpp"

namespace agnes {

// ----------------------------------------------------------------- lookup

template <typename TI, typename TO, typename IdT>
__global__ __launch_bounds__(kBlock) void k_embed_lookup(const TI* __restrict__ table, int64_t tstride, int64_t V,
                                                         int64_t D, const IdT* __restrict__ ids, int64_t n,
                                                         float scale, TO* __restrict__ out, int64_t ostride) {
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int64_t v = (int64_t)ids[i];
        const bool named = v >= 0 && v < V;
        for (int64_t c = threadIdx.x; c < D; c += kBlock)
            out[i * ostride + c] = from_float<TO>(named ? scale * to_float(table[v * tstride + c]) : 0.f);
    }
}

static void check_lookup(const agnes_matrix* table, const void* ids, agnes_dtype ids_dtype, const agnes_matrix* out) {
    check_matrix(table, false, "table");
    check_matrix(out, true, "out");
    AGNES_REQUIRE(is_index(ids_dtype), AGNES_ERR_INVALID, "ids must be int32 or int64");
    AGNES_REQUIRE(ids || out->rows == 0, AGNES_ERR_INVALID, "ids must not be NULL");
    AGNES_REQUIRE(out->cols == table->cols, AGNES_ERR_INVALID, "out must have the table's columns");
    AGNES_REQUIRE(table->rows < INT32_MAX, AGNES_ERR_INVALID, "the table must have fewer than 2^31 - 1 rows");
}

void embedding_lookup(const agnes_matrix* table, const void* ids, agnes_dtype ids_dtype, float scale,
                      const agnes_matrix* out, hipStream_t st) {
    check_lookup(table, ids, ids_dtype, out);
    const int64_t n = out->rows, D = out->cols;
    if (n == 0 || D == 0) return;
    with_float(table->dtype, [&](auto ti) {
        with_float(out->dtype, [&](auto to) {
            with_index(ids_dtype, [&](auto id) {
                typedef decltype(ti) TI;
                typedef decltype(to) TO;
                typedef decltype(id) IdT;
                AGNES_LAUNCH((k_embed_lookup<TI, TO, IdT>), dim3((unsigned)std::min<int64_t>(n, 1 << 16)), dim3(kBlock),
                             0, st, (const TI*)table->data, table->stride, table->rows, D, (const IdT*)ids, n, scale,
                             (TO*)out->data, out->stride);
            });
        });
    });
}

// ----------------------------------------------------------------- gradient

// Sort keys: the id, or V for padding (sorted behind every id).
template <typename IdT>
__global__ __launch_bounds__(kBlock) void k_embed_keys(const IdT* __restrict__ ids, int64_t n, int64_t V,
                                                       uint32_t* __restrict__ keys, int64_t* n_dev) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i == 0) *n_dev = n;
    if (i >= n) return;
    const int64_t v = (int64_t)ids[i];
    keys[i] = (uint32_t)(v >= 0 && v < V ? v : V);
}

// 1 where a run of equal ids begins.
__global__ __launch_bounds__(kBlock) void k_embed_heads(const uint32_t* __restrict__ keys, int64_t n, uint32_t V,
                                                        int32_t* __restrict__ heads) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i >= n) return;
    heads[i] = keys[i] < V && (i == 0 || keys[i - 1] != keys[i]);
}

__global__ __launch_bounds__(kBlock) void k_embed_clear_ids(int32_t* row_ids, int64_t max_rows) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i < max_rows) row_ids[i] = -1;
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_embed_clear_rows(T* out, int64_t stride, int64_t rows, int64_t D) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < D; c += kBlock) out[r * stride + c] = from_float<T>(0.f);
}

// One workgroup per run.  compact: the run's place among all runs (rank: heads
// before every position) is its output row, otherwise its id is.
template <typename TI, typename TO>
__global__ __launch_bounds__(kBlock) void k_embed_sum(const TI* __restrict__ g, int64_t gstride, int64_t D,
                                                      const uint32_t* __restrict__ keys,
                                                      const uint32_t* __restrict__ perm, int64_t n, uint32_t V,
                                                      const int64_t* __restrict__ rank, float scale, bool accumulate,
                                                      bool compact, int32_t* row_ids, int64_t max_rows, TO* __restrict__ out,
                                                      int64_t ostride) {
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const uint32_t v = keys[i];
        if (v >= V) break;
        if (i > 0 && keys[i - 1] == v) continue;
        int64_t row = v;
        if (compact) {
            row = rank[i];
            if (row >= max_rows) continue;
            if (threadIdx.x == 0) row_ids[row] = (int32_t)v;
        }
        for (int64_t c = threadIdx.x; c < D; c += kBlock) {
            float acc = 0.f;
            for (int64_t j = i; j < n && keys[j] == v; j++) acc += to_float(g[(int64_t)perm[j] * gstride + c]);
            acc *= scale;
            TO* p = out + row * ostride + c;
            if (accumulate) acc += to_float(*p);
            *p = from_float<TO>(acc);
        }
    }
}

struct GradPlan {
    uint32_t *keys[2], *vals[2], *hist, *dtot;
    int64_t *n_dev, *rank, *partials;
    int32_t* heads;
    size_t bytes;
};

static GradPlan plan_grad(int64_t n, int64_t num_rows, int64_t dim, void* ws) {
    AGNES_REQUIRE(n >= 0 && n < INT32_MAX, AGNES_ERR_RANGE, "the number of ids must be in [0, 2^31 - 1)");
    AGNES_REQUIRE(num_rows >= 0 && num_rows < INT32_MAX, AGNES_ERR_INVALID,
                  "the table must have fewer than 2^31 - 1 rows");
    AGNES_REQUIRE(dim >= 0 && dim < ((int64_t)1 << 31), AGNES_ERR_INVALID, "dim must be in [0, 2^31)");
    GradPlan p{};
    Carve c(ws);
    p.n_dev = c.take<int64_t>(1);
    for (int k = 0; k < 2; k++) {
        p.keys[k] = c.take<uint32_t>(n);
        p.vals[k] = c.take<uint32_t>(n);
    }
    p.hist = c.take<uint32_t>(radix_hist_entries(n));
    p.dtot = c.take<uint32_t>(radix_dtot_entries());
    p.heads = c.take<int32_t>(n);
    p.rank = c.take<int64_t>(n + 1);
    p.partials = c.take<int64_t>(scan_partials_needed());
    p.bytes = c.used;
    return p;
}

uint64_t embedding_grad_bytes(int64_t n, int64_t num_rows, int64_t dim) {
    return plan_grad(n, num_rows, dim, nullptr).bytes;
}

static void check_grad(const agnes_matrix* g, const void* ids, agnes_dtype ids_dtype, int64_t num_rows,
                       const agnes_matrix* out, const void* ws, uint64_t ws_bytes) {
    check_matrix(g, false, "grad_out");
    check_matrix(out, true, "the gradient");
    AGNES_REQUIRE(is_index(ids_dtype), AGNES_ERR_INVALID, "ids must be int32 or int64");
    AGNES_REQUIRE(ids || g->rows == 0, AGNES_ERR_INVALID, "ids must not be NULL");
    AGNES_REQUIRE(out->cols == g->cols, AGNES_ERR_INVALID, "the gradient must have grad_out's columns");
    check_workspace(ws, ws_bytes, embedding_grad_bytes(g->rows, num_rows, g->cols));
}

// The gradient in either form: compact: the distinct rows alone.
static void grad(const agnes_matrix* g, const void* ids, agnes_dtype ids_dtype, float scale, bool accumulate,
                 bool compact, int64_t num_rows, int32_t* row_ids, const agnes_matrix* out, int64_t* count, void* ws,
                 hipStream_t st) {
    const int64_t n = g->rows, D = g->cols;
    const GradPlan p = plan_grad(n, num_rows, D, ws);
    const int G = (int)std::max<int64_t>(1, (n + kBlock - 1) / kBlock);
    with_index(ids_dtype, [&](auto id) {
        typedef decltype(id) IdT;
        AGNES_LAUNCH((k_embed_keys<IdT>), dim3(G), dim3(kBlock), 0, st, (const IdT*)ids, n, num_rows, p.keys[0],
                     p.n_dev);
    });
    int bits = 1;
    while (((int64_t)1 << bits) <= num_rows) bits++;
    const int at = radix_sort_pairs32(p.keys[0], p.vals[0], p.keys[1], p.vals[1], p.n_dev, n, bits, p.hist, p.dtot,
                                      st, true);
    if (compact) {
        AGNES_LAUNCH(k_embed_heads, dim3(G), dim3(kBlock), 0, st, p.keys[at], n, (uint32_t)num_rows, p.heads);
        scan_counts(p.heads, p.rank, p.n_dev, n, count, p.partials, st);
        AGNES_LAUNCH(k_embed_clear_ids, dim3((unsigned)((out->rows + kBlock - 1) / kBlock + 1)), dim3(kBlock), 0, st,
                     row_ids, out->rows);
    }
    with_float(out->dtype, [&](auto to) {
        typedef decltype(to) TO;
        if (!compact && !accumulate && out->rows > 0 && D > 0)
            AGNES_LAUNCH((k_embed_clear_rows<TO>), dim3((unsigned)std::min<int64_t>(out->rows, 1 << 16)), dim3(kBlock),
                         0, st, (TO*)out->data, out->stride, out->rows, D);
        if (n == 0) return;
        with_float(g->dtype, [&](auto ti) {
            typedef decltype(ti) TI;
            AGNES_LAUNCH((k_embed_sum<TI, TO>), dim3((unsigned)std::min<int64_t>(n, 1 << 16)), dim3(kBlock), 0, st,
                         (const TI*)g->data, g->stride, D, p.keys[at], p.vals[at], n, (uint32_t)num_rows, p.rank,
                         scale, accumulate, compact, row_ids, out->rows, (TO*)out->data, out->stride);
        });
    });
}

void embedding_grad(const agnes_matrix* grad_out, const void* ids, agnes_dtype ids_dtype, float scale,
                    bool accumulate, const agnes_matrix* grad_table, void* ws, uint64_t ws_bytes, hipStream_t st) {
    AGNES_REQUIRE(grad_table, AGNES_ERR_INVALID, "the gradient must not be NULL");
    check_grad(grad_out, ids, ids_dtype, grad_table->rows, grad_table, ws, ws_bytes);
    if (grad_table->rows == 0 || grad_table->cols == 0) return;
    grad(grad_out, ids, ids_dtype, scale, accumulate, false, grad_table->rows, nullptr, grad_table, nullptr, ws, st);
}

void embedding_grad_rows(const agnes_matrix* grad_out, const void* ids, agnes_dtype ids_dtype, float scale,
                         int64_t num_rows, int32_t* row_ids, const agnes_matrix* rows, int64_t* count, void* ws,
                         uint64_t ws_bytes, hipStream_t st) {
    check_grad(grad_out, ids, ids_dtype, num_rows, rows, ws, ws_bytes);
    AGNES_REQUIRE(count, AGNES_ERR_INVALID, "count must not be NULL");
    AGNES_REQUIRE(row_ids || rows->rows == 0, AGNES_ERR_INVALID, "row_ids must not be NULL");
    grad(grad_out, ids, ids_dtype, scale, false, true, num_rows, row_ids, rows, count, ws, st);
}

// ----------------------------------------------------------------- a batch's nodes

// Orders `st` behind the batch's gather and behind an earlier reader on another
// stream, so that the event recorded after the work covers both.
static int64_t enter_batch(Batch& b, hipStream_t st) {
    AGNES_REQUIRE(b.state == kGathering || b.state == kDone, AGNES_ERR_INVALID, "the batch holds no finished hyperbatch");
    AGNES_CHECK_HIP(hipStreamWaitEvent(st, b.gathered_at, 0));
    if (b.sage_pending) AGNES_CHECK_HIP(hipStreamWaitEvent(st, b.sage_done, 0));
    return b.node_off[b.H];
}

static void leave_batch(Batch& b, hipStream_t st) {
    AGNES_CHECK_HIP(hipEventRecord(b.sage_done, st));
    b.sage_pending = true;
}

void batch_embedding_lookup(Batch& b, const agnes_matrix* table, float scale, const agnes_matrix* out,
                            hipStream_t st) {
    AGNES_REQUIRE(table && out, AGNES_ERR_INVALID, "table and out must not be NULL");
    AGNES_REQUIRE(b.store && table->rows == b.store->num_nodes, AGNES_ERR_INVALID,
                  "the table must have one row per node");
    const int64_t n = enter_batch(b, st);
    AGNES_REQUIRE(out->rows == n, AGNES_ERR_INVALID, "out must have one row per node of the batch");
    embedding_lookup(table, b.nodes.ptr, AGNES_INT32, scale, out, st);
    leave_batch(b, st);
}

void batch_embedding_grad_rows(Batch& b, const agnes_matrix* grad_out, float scale, int32_t* row_ids,
                               const agnes_matrix* rows, int64_t* count, void* ws, uint64_t ws_bytes, hipStream_t st) {
    AGNES_REQUIRE(grad_out && rows, AGNES_ERR_INVALID, "grad_out and rows must not be NULL");
    const int64_t n = enter_batch(b, st);
    AGNES_REQUIRE(grad_out->rows == n, AGNES_ERR_INVALID, "grad_out must have one row per node of the batch");
    embedding_grad_rows(grad_out, b.nodes.ptr, AGNES_INT32, scale, b.store->num_nodes, row_ids, rows, count, ws,
                        ws_bytes, st);
    leave_batch(b, st);
}

}  // namespace agnes
