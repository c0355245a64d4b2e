// Embedding lookup and its gradient.
//
// Lookup: out[i] = scale * table[ids[i]].  Gradient: dTable[v] = scale * sum of
// grad_out[i] over the i with ids[i] = v, ascending in i.  The ids are sorted
// stably, so a table row's contributions form one run of the sorted list, and
// each run is summed in its order: no atomics, the same bits on every run.
#include <algorithm>

#include "ops.hpp"

namespace agnes {

// A row is handled by a group of lanes (a power of two, at most a wave), each
// holding E consecutive elements of it; wider rows take several tiles.
struct RowShape {
    int lanes;       // per group
    int tiles;       // column tiles of lanes * E elements
};
static RowShape row_shape(int64_t D, int E) {
    const int64_t pieces = (D + E - 1) / E;
    int lanes = 1;
    while (lanes < pieces && lanes < kWave) lanes *= 2;
    return {lanes, (int)((pieces + lanes - 1) / lanes)};
}

// E elements at column c of a row of D, as many as there are.
template <typename T, int E>
__device__ __forceinline__ void load_piece(const T* row, int64_t c, int64_t D, float (&x)[E]) {
    if (c + E <= D) {
        Vec<T, E>::load(row + c, x);
    } else {
#pragma unroll
        for (int q = 0; q < E; q++) x[q] = c + q < D ? to_float(row[c + q]) : 0.f;
    }
}
// The same without the conversion, for pieces that wait in registers.
template <typename T, int E>
__device__ __forceinline__ typename Vec<T, E>::type raw_piece(const T* row, int64_t c, int64_t D) {
    if (c + E <= D) return Vec<T, E>::raw(row + c);
    typename Vec<T, E>::type v;
#pragma unroll
    for (int q = 0; q < E; q++) v[q] = c + q < D ? row[c + q] : (T)0.f;
    return v;
}
template <typename T, int E>
__device__ __forceinline__ void store_piece(T* row, int64_t c, int64_t D, const float (&x)[E], bool nt) {
    if (c + E <= D) {
        Vec<T, E>::store(row + c, x, nt);
    } else {
#pragma unroll
        for (int q = 0; q < E; q++)
            if (c + q < D) row[c + q] = from_float<T>(x[q]);
    }
}

// ----------------------------------------------------------------- lookup

// A group of lanes copies kLookupRows rows at a time: their ids, then all their
// pieces, then the stores, so that many row reads are in flight per wave.
// Bound by memory: 2000003 ids over 2^20 rows of 128 float32, to bfloat16:
// 218 us, 1.0 GB read and 0.5 GB written.
constexpr int kLookupRows = 4;

template <typename TI, typename TO, typename IdT>
__global__ __launch_bounds__(kBlock) void k_embed_lookup(const TI* __restrict__ table, int64_t tstride, int64_t V,
                                                         int64_t D, const IdT* __restrict__ ids, int64_t n,
                                                         float scale, TO* __restrict__ out, int64_t ostride,
                                                         int lanes, bool nt) {
    constexpr int E = 16 / (int)(sizeof(TI) < sizeof(TO) ? sizeof(TI) : sizeof(TO)), U = kLookupRows;
    const int groups = kBlock / lanes, g = threadIdx.x / lanes, gl = threadIdx.x % lanes;
    for (int64_t i0 = (int64_t)blockIdx.x * groups * U + g; i0 < n; i0 += (int64_t)gridDim.x * groups * U) {
        int64_t v[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t i = i0 + (int64_t)u * groups;
            v[u] = i < n ? (int64_t)ids[i] : -1;
        }
        for (int64_t c = (int64_t)gl * E; c < D; c += (int64_t)lanes * E) {
            float x[U][E];
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (v[u] >= 0 && v[u] < V) {
                    load_piece<TI, E>(table + v[u] * tstride, c, D, x[u]);
                } else {
#pragma unroll
                    for (int q = 0; q < E; q++) x[u][q] = 0.f;
                }
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int64_t i = i0 + (int64_t)u * groups;
                if (i >= n) continue;
#pragma unroll
                for (int q = 0; q < E; q++) x[u][q] *= scale;
                store_piece<TO, E>(out + i * ostride, c, D, x[u], nt);
            }
        }
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
                const int lanes = row_shape(D, 16 / (int)std::min(sizeof(TI), sizeof(TO))).lanes;
                const int64_t per = (int64_t)(kBlock / lanes) * kLookupRows;
                AGNES_LAUNCH((k_embed_lookup<TI, TO, IdT>), dim3((unsigned)std::min<int64_t>((n + per - 1) / per, 1 << 22)),
                             dim3(kBlock), 0, st, (const TI*)table->data, table->stride, table->rows, D, (const IdT*)ids, n, scale,
                             (TO*)out->data, out->stride, lanes, n * D * (int64_t)sizeof(TO) > kStreamBytes);
            });
        });
    });
}

// ----------------------------------------------------------------- gradient: sorted ids

// Up to kRankSort ids are sorted by counting, in one launch: an id's place is
// the number of ids before it in (id, position) order.  Every workgroup holds
// all keys in LDS; 16 lanes share one id's comparisons.  More ids take the
// device-wide radix sort (three launches per digit).  Whole gradient of 8192
// ids: 20 us less by counting; of 16384 ids: 45 us more.  Padding gets the key V
// and so comes last.  Both kernels also clear the list of distinct ids.
constexpr int kRankSort = 8192;
constexpr int kRankLanes = 16;

template <typename IdT>
__device__ __forceinline__ uint32_t sort_key(IdT id, int64_t V) {
    return (uint32_t)((int64_t)id >= 0 && (int64_t)id < V ? (int64_t)id : V);
}

__device__ __forceinline__ void clear_row_ids(int32_t* row_ids, int64_t max_rows) {
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < max_rows; i += (int64_t)gridDim.x * kBlock)
        row_ids[i] = -1;
}

template <typename IdT>
__global__ __launch_bounds__(kBlock) void k_embed_rank_sort(const IdT* __restrict__ ids, int n, int64_t V,
                                                            uint32_t* __restrict__ keys, uint32_t* __restrict__ perm,
                                                            int32_t* row_ids, int64_t max_rows) {
    __shared__ __attribute__((aligned(16))) int32_t k[kRankSort];
    const int quads = (n + 3) / 4;
    for (int i = threadIdx.x; i < quads * 4; i += kBlock)
        k[i] = i < n ? (int32_t)sort_key(ids[i], V) : INT32_MAX;      // V < 2^31 - 1: behind every key
    clear_row_ids(row_ids, max_rows);
    __syncthreads();
    const int part = threadIdx.x % kRankLanes;
    const int i = blockIdx.x * (kBlock / kRankLanes) + threadIdx.x / kRankLanes;
    const int mine = i < n ? k[i] : 0;
    int place = 0;
    // an equal key counts if its position is smaller: key <= mine - 1 behind position i, key <= mine before it
    for (int q = part; q < quads; q += kRankLanes) {
        const int4 x = *(const int4*)&k[4 * q];
        place += x.x <= mine - (4 * q + 0 >= i);
        place += x.y <= mine - (4 * q + 1 >= i);
        place += x.z <= mine - (4 * q + 2 >= i);
        place += x.w <= mine - (4 * q + 3 >= i);
    }
#pragma unroll
    for (int d = 1; d < kRankLanes; d <<= 1) place += __shfl_xor(place, d, kWave);
    if (part == 0 && i < n) {
        keys[place] = (uint32_t)mine;
        perm[place] = (uint32_t)i;
    }
}

template <typename IdT>
__global__ __launch_bounds__(kBlock) void k_embed_keys(const IdT* __restrict__ ids, int64_t n, int64_t chunks,
                                                       int64_t V, uint32_t* __restrict__ keys, int64_t* sizes,
                                                       int32_t* row_ids, int64_t max_rows) {
    clear_row_ids(row_ids, max_rows);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        sizes[0] = n;
        sizes[1] = chunks;
    }
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += (int64_t)gridDim.x * kBlock)
        keys[i] = sort_key(ids[i], V);
}

// No ids at all: an empty list.
__global__ __launch_bounds__(kBlock) void k_embed_no_ids(int32_t* row_ids, int64_t max_rows, int64_t* count) {
    clear_row_ids(row_ids, max_rows);
    if (blockIdx.x == 0 && threadIdx.x == 0) *count = 0;
}

// ----------------------------------------------------------------- gradient: runs

// The sorted list is cut into chunks of fixed length, whatever the runs: a
// group of lanes sums a chunk's rows in order and
//   - writes the gradient of every run that lies inside the chunk, or begins in
//     it and has at most kFollow rows in the next, whose group passes over them;
//   - leaves the sum of a first piece that continues the chunk before in the
//     chunk's entry 2c ("head"), and that of a last piece that goes on in the
//     next chunk in its entry 2c + 1 ("tail"; a chunk inside one run has a
//     head only), with the run's output row in `part_row` (-1: no entry).
// The entries are again a list of runs, each begun by a tail and continued by
// heads, and are summed the same way, level by level, until few are left; the
// last level follows each run to its end.  So the work of a run is split evenly
// however often an id occurs, and the order of every sum depends on the list
// alone.  A level has about 1/16 (first) or 1/8 (later) as many entries as the
// one before had rows.
// Most runs are short: passing over them at a chunk's start saves their entries,
// written and read (1500007 rows of 256 bfloat16: 399 -> 364 us; with 16 rows
// for kFollow the same).  A group of a later level waits for one batch of entries
// after the other, so it takes few (131072 x 1024 with hot ids: 159 us with 32,
// 148 us with 16).
constexpr int kRows = 4;                    // rows per batch
constexpr int kFollow = 8;                  // at most a chunk, and a multiple of kRows
constexpr int kSmall = 4096;                // up to so many ids
constexpr int kChunkSmall = 16;             // chunks are shorter, for more groups,
constexpr int kChunk = 32;                  // than above
constexpr int kJoinChunk = 16;              // entries per group of a later level
constexpr int64_t kJoinLast = 512;          // entries that the last level may have

static int chunk_of(int64_t n) { return n <= kSmall ? kChunkSmall : kChunk; }

// Where a run's sum goes.
template <typename TO> struct Sink {
    TO* out;
    int64_t ostride, D;
    int64_t max_rows;                       // rows of out
    float scale;
    bool accumulate;
    float* part;                            // [entries][dpad] partial sums
    int32_t* part_row;                      // [entries]
    int64_t dpad;
    bool nt;                                // stores past the caches

    template <int E> __device__ __forceinline__ void finish(int64_t row, int64_t c, float (&acc)[E]) const {
        if (c >= D || row >= max_rows) return;
        TO* p = out + row * ostride;
#pragma unroll
        for (int q = 0; q < E; q++) acc[q] *= scale;
        if (accumulate) {
            float old[E];
            load_piece<TO, E>(p, c, D, old);
#pragma unroll
            for (int q = 0; q < E; q++) acc[q] += old[q];
        }
        store_piece<TO, E>(p, c, D, acc, nt);
    }
    template <int E> __device__ __forceinline__ void leave(int64_t entry, int64_t c, const float (&acc)[E]) const {
        if (c < D) Vec<float, E>::store(part + entry * dpad + c, acc);      // dpad is a multiple of E
    }
};

// Heads (first positions of runs) in chunk c.
__device__ __forceinline__ int chunk_heads(const uint32_t* keys, int64_t n, uint32_t V, int64_t c, int chunk) {
    const int64_t q0 = c * chunk, q1 = min(n, q0 + chunk);
    uint32_t prev = q0 > 0 && q0 < n ? keys[q0 - 1] : V;
    int heads = 0;
    for (int64_t q = q0; q < q1; q++) {
        const uint32_t k = keys[q];
        heads += k != prev && k < V;        // keys ascend: once V, always V
        prev = k;
    }
    return heads;
}

// The heads of every chunk of kChunk = 32: a wave reads 64 keys, two chunks, at once.
__global__ __launch_bounds__(kBlock) void k_embed_heads(const uint32_t* __restrict__ keys, int64_t n, uint32_t V,
                                                        int64_t chunks, int32_t* __restrict__ heads) {
    static_assert(kChunk == 32, "half a wave per chunk");
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    bool head = false;
    if (i < n) {
        const uint32_t k = keys[i];
        head = k < V && (i == 0 || keys[i - 1] != k);
    }
    const uint64_t m = __ballot(head);
    const int64_t c = i / kChunk;
    if (i % kChunk == 0 && c < chunks) heads[c] = __popc((uint32_t)(lane_id() ? m >> 32 : m));
}

// What the first level reads.
template <typename TI> struct Sorted {
    const TI* g;
    int64_t gstride;
    const uint32_t *keys, *perm;
    int64_t n;
    uint32_t V;
    int chunk;
    int64_t chunks;
    bool compact;                           // output row = the run's place among all runs, not its id
    const int64_t* rank;                    // heads before every chunk; NULL: counted here (few ids)
    int32_t* row_ids;
    int64_t* count;
};

// Zeroes the rows of [v0, v0 + R) that no key names; R <= kBlock.
template <typename TO>
__device__ __forceinline__ void clear_unnamed(const uint32_t* keys, int64_t n, int64_t v0, int R, int64_t V, TO* out,
                                              int64_t ostride, int64_t D, int lanes, bool nt) {
    constexpr int E = 16 / (int)sizeof(TO);
    __shared__ bool named[kBlock];
    // the keys of these rows: one half of the wave finds where they begin, the other where they end
    const uint32_t bound = (uint32_t)(lane_id() < 32 ? v0 : min(V, v0 + R));
    const int64_t at = group_partition_point<32>(0, n, [&](int64_t i) { return keys[i] < bound; });
    const int64_t lo = (int64_t)shfl64((uint64_t)at, 0), hi = (int64_t)shfl64((uint64_t)at, 32);
    const int t = threadIdx.x;
    if (t < R) {
        int64_t a = lo, b = hi;
        const uint32_t v = (uint32_t)(v0 + t);
        while (a < b) {
            const int64_t m = (a + b) >> 1;
            if (keys[m] < v) a = m + 1; else b = m;
        }
        named[t] = a < hi && keys[a] == v;
    }
    __syncthreads();
    const int groups = kBlock / lanes, g = t / lanes, gl = t % lanes;
    float zero[E];
#pragma unroll
    for (int q = 0; q < E; q++) zero[q] = 0.f;
    for (int r = g; r < R; r += groups) {
        if (named[r] || v0 + r >= V) continue;
        for (int64_t c = (int64_t)gl * E; c < D; c += (int64_t)lanes * E)
            store_piece<TO, E>(out + (v0 + r) * ostride, c, D, zero, nt);
    }
}

// Workgroups [0, sum_blocks) sum chunks, column tile by column tile; the rest
// clear the rows that no id names, fill_rows at a time.  Bound by memory, which
// rows are read from in the ids' order: 1500007 rows of 256 bfloat16 into 0.7M
// distinct ones 246 us (4.6 TB/s); the sort before it takes 90 us.
template <typename TI, typename TO>
__global__ __launch_bounds__(kBlock) void k_embed_sum(Sorted<TI> s, Sink<TO> o, int lanes, int tiles,
                                                      int64_t sum_blocks, int fill_rows, int fill_lanes) {
    constexpr int E = 16 / (int)sizeof(TI);
    if ((int64_t)blockIdx.x >= sum_blocks) {
        clear_unnamed<TO>(s.keys, s.n, ((int64_t)blockIdx.x - sum_blocks) * fill_rows, fill_rows, s.V, o.out,
                          o.ostride, o.D, fill_lanes, o.nt);
        return;
    }
    const int groups = kBlock / lanes, g = threadIdx.x / lanes, gl = threadIdx.x % lanes;
    const int64_t c0 = (int64_t)blockIdx.x / tiles * groups;        // the workgroup's first chunk
    const int tile = blockIdx.x % tiles;
    const int64_t c = c0 + g;
    int64_t rank = 0;                                               // heads before the chunk
    if (s.compact && !s.rank) {
        __shared__ int lds[kWavesPerBlock];
        __shared__ int base[kBlock];
        int before = 0;
        for (int64_t q = threadIdx.x; q < c0 * s.chunk; q += kBlock)
            before += s.keys[q] < s.V && (q == 0 || s.keys[q - 1] != s.keys[q]);
        int total, mine = 0, all;
        (void)block_exclusive_scan(before, lds, total);
        if ((int)threadIdx.x < groups) mine = chunk_heads(s.keys, s.n, s.V, c0 + threadIdx.x, s.chunk);
        const int ex = block_exclusive_scan(mine, lds, all);
        base[threadIdx.x] = total + ex;
        __syncthreads();
        rank = base[g];
        if (c0 + groups >= s.chunks && tile == 0 && threadIdx.x == 0) *s.count = total + all;
    } else if (s.compact && c < s.chunks) {
        rank = s.rank[c];
    }
    // The keys and places of all the workgroup's chunks, so that only the rows
    // themselves are waited for: two batches of kRows are in flight.
    extern __shared__ uint32_t staged[];
    const int pitch = s.chunk + 1;                                  // odd: the groups' reads fall into different banks
    uint32_t* const skey = staged + g * pitch;
    const uint32_t* const sperm = skey + (groups + 1) * pitch;
    for (int i = threadIdx.x; i < groups * s.chunk + kFollow; i += kBlock) {
        const int64_t q = c0 * s.chunk + i;
        const int at = i / s.chunk * pitch + i % s.chunk;
        staged[at] = q < s.n ? s.keys[q] : s.V;
        staged[(groups + 1) * pitch + at] = q < s.n ? s.perm[q] : 0u;
    }
    __syncthreads();
    if (c >= s.chunks) return;
    const int64_t col = ((int64_t)tile * lanes + gl) * E;
    const int64_t q0 = c * s.chunk, q1 = min(s.n, q0 + s.chunk);
    const bool lead = tile == 0 && gl == 0, live = col < o.D;
    uint32_t cur = q0 > 0 ? s.keys[q0 - 1] : s.V;                   // the open run's id
    // Whether the run that ends in front of, or goes over, position q began in the
    // chunk before q and has at most kFollow rows from q on.
    auto followed = [&](int64_t q, uint32_t key) {
        return (q - s.chunk == 0 || s.keys[q - s.chunk - 1] != key) && (q + kFollow >= s.n || s.keys[q + kFollow] != key);
    };
    const uint32_t done = q0 > 0 && followed(q0, cur) ? cur : s.V;  // summed by the group before
    bool continued = true;                                          // it began in an earlier chunk
    bool any = false;                                               // it has rows here
    int64_t row = s.compact ? rank - 1 : (int64_t)cur;
    int32_t head = -1, tail = -1;
    float acc[E];
#pragma unroll
    for (int q = 0; q < E; q++) acc[q] = 0.f;
    typedef typename Vec<TI, E>::type Raw;
    auto fetch = [&](int q, Raw (&x)[kRows]) {
#pragma unroll
        for (int j = 0; j < kRows; j++)
            if (live && skey[q + j] < s.V && skey[q + j] != done)
                x[j] = raw_piece<TI, E>(s.g + (int64_t)sperm[q + j] * s.gstride, col, o.D);
    };
    auto add = [&](int q, const Raw (&x)[kRows]) {
#pragma unroll
        for (int j = 0; j < kRows; j++) {
            const uint32_t key = skey[q + j];
            if (key >= s.V || key == done) continue;
            if (key != cur) {
                if (any) {
                    if (continued) {
                        o.leave(2 * c, col, acc);
                        head = (int32_t)row;
                    } else {
                        o.finish(row, col, acc);
                    }
                }
                cur = key;
                continued = false;
                row = s.compact ? rank++ : (int64_t)cur;
                if (s.compact && lead && row < o.max_rows) s.row_ids[row] = (int32_t)cur;
#pragma unroll
                for (int e = 0; e < E; e++) acc[e] = 0.f;
            }
            any = true;
#pragma unroll
            for (int e = 0; e < E; e++) acc[e] += (float)x[j][e];
        }
    };
    Raw xa[kRows] = {}, xb[kRows] = {};                             // lanes behind the last column load nothing
    fetch(0, xa);
    for (int q = 0; q < s.chunk; q += 2 * kRows) {                  // chunk is a multiple of 2 kRows
        fetch(q + kRows, xb);
        add(q, xa);
        if (q + 2 * kRows < s.chunk) fetch(q + 2 * kRows, xa);
        add(q + kRows, xb);
    }
    if (any) {
        const bool on = q1 < s.n && skey[pitch] == cur;             // goes on in the next chunk
        if (on && !continued && followed(q1, cur)) {
            const uint32_t *fkey = skey + pitch, *fperm = sperm + pitch;
#pragma unroll
            for (int q = 0; q < kFollow; q += kRows) {
#pragma unroll
                for (int j = 0; j < kRows; j++)
                    if (live && fkey[q + j] == cur)
                        xa[j] = raw_piece<TI, E>(s.g + (int64_t)fperm[q + j] * s.gstride, col, o.D);
#pragma unroll
                for (int j = 0; j < kRows; j++) {
                    if (fkey[q + j] != cur) continue;
#pragma unroll
                    for (int e = 0; e < E; e++) acc[e] += (float)xa[j][e];
                }
            }
            o.finish(row, col, acc);
        } else if (on) {
            o.leave(continued ? 2 * c : 2 * c + 1, col, acc);
            (continued ? head : tail) = (int32_t)row;
        } else if (continued) {
            o.leave(2 * c, col, acc);
            head = (int32_t)row;
        } else {
            o.finish(row, col, acc);
        }
    }
    if (lead && o.part_row) {
        o.part_row[2 * c] = head;
        o.part_row[2 * c + 1] = tail;
    }
}

// A later level over `entries` entries (rows in/in_row).  last: a group follows
// every run that a tail of its chunk begins to the run's end.
template <typename TO>
__global__ __launch_bounds__(kBlock) void k_embed_join(const float* __restrict__ in, const int32_t* __restrict__ in_row,
                                                       int64_t entries, int chunk, bool last, Sink<TO> o, int lanes,
                                                       int tiles) {
    constexpr int E = 4;
    const int groups = kBlock / lanes, g = threadIdx.x / lanes, gl = threadIdx.x % lanes;
    const int64_t c = (int64_t)blockIdx.x / tiles * groups + g;
    const int tile = blockIdx.x % tiles;
    const int64_t q0 = c * chunk;
    const int64_t col = ((int64_t)tile * lanes + gl) * E;
    if (q0 >= entries || col >= o.D) return;                        // D > 0, and lanes do not exchange anything
    const int64_t q1 = min(entries, q0 + chunk);
    int32_t cur = -1, head = -1, tail = -1;
    bool continued = false, open = true;
    float acc[E] = {0.f, 0.f, 0.f, 0.f};
    constexpr int R = 8;                                            // entries per batch; chunk is a multiple
    for (int64_t q = q0; open && q < (last ? entries : q1); q += R) {
        int32_t row[R];
        float x[R][E];
#pragma unroll
        for (int j = 0; j < R; j++) row[j] = q + j < entries ? in_row[q + j] : -1;
#pragma unroll
        for (int j = 0; j < R; j++)
            if (row[j] >= 0) Vec<float, E>::load(in + (q + j) * o.dpad + col, x[j]);
#pragma unroll
        for (int j = 0; j < R; j++) {
            if (!open) continue;
            const bool begins = (q + j) & 1;                        // a tail begins a run, a head continues one
            if (last && q + j >= q1 && (row[j] < 0 ? !begins || cur < 0 : begins)) {
                open = false;                                       // past the chunk, the followed run has ended
                continue;
            }
            if (row[j] < 0) continue;
            if (begins) {
                if (cur >= 0) {
                    if (continued) {
                        o.leave(2 * c, col, acc);
                        head = cur;
                    } else {
                        o.finish(cur, col, acc);
                    }
                }
                cur = row[j];
                continued = false;
#pragma unroll
                for (int e = 0; e < E; e++) acc[e] = 0.f;
            } else if (cur < 0) {
                if (last) continue;                                 // begun by another group's chunk
                cur = row[j];
                continued = true;
            }
#pragma unroll
            for (int e = 0; e < E; e++) acc[e] += x[j][e];
        }
    }
    if (cur >= 0) {
        if (!last && q1 < entries && in_row[q1] >= 0) {             // its next head is in the next chunk
            o.leave(continued ? 2 * c : 2 * c + 1, col, acc);
            (continued ? head : tail) = cur;
        } else if (continued) {
            o.leave(2 * c, col, acc);
            head = cur;
        } else {
            o.finish(cur, col, acc);
        }
    }
    if (!last && tile == 0 && gl == 0) {
        o.part_row[2 * c] = head;
        o.part_row[2 * c + 1] = tail;
    }
}

// ----------------------------------------------------------------- gradient: host

constexpr int kLevels = 8;                  // 2^31 ids: 2^27 entries, then 1/8 of them at each level, 2^9 at the seventh
struct GradPlan {
    uint32_t *keys[2], *perm[2], *hist, *dtot;
    int64_t *sizes, *rank, *partials;
    int32_t* heads;
    int64_t chunks, dpad;
    int levels;                             // levels after the first
    int64_t entries[kLevels];               // that each of them reads
    float* part[kLevels];
    int32_t* part_row[kLevels];
    size_t bytes;
};

static GradPlan plan_grad(int64_t n, int64_t num_rows, int64_t dim, void* ws) {
    AGNES_REQUIRE(n < INT32_MAX, AGNES_ERR_RANGE, "the number of ids must be below 2^31 - 1");
    AGNES_REQUIRE(n >= 0, AGNES_ERR_INVALID, "the number of ids must not be negative");
    AGNES_REQUIRE(num_rows >= 0 && num_rows < INT32_MAX, AGNES_ERR_INVALID,
                  "the table must have fewer than 2^31 - 1 rows");
    AGNES_REQUIRE(dim >= 0 && dim < ((int64_t)1 << 31), AGNES_ERR_INVALID, "dim must be in [0, 2^31)");
    GradPlan p{};
    Carve c(ws);
    const bool radix = n > kRankSort;
    p.chunks = (n + chunk_of(n) - 1) / chunk_of(n);
    p.sizes = c.take<int64_t>(2);
    for (int k = 0; k < (radix ? 2 : 1); k++) {
        p.keys[k] = c.take<uint32_t>(n);
        p.perm[k] = c.take<uint32_t>(n);
    }
    if (radix) {
        p.hist = c.take<uint32_t>(radix_hist_entries(n));
        p.dtot = c.take<uint32_t>(radix_dtot_entries());
        p.heads = c.take<int32_t>(p.chunks);
        p.rank = c.take<int64_t>(p.chunks + 1);
        p.partials = c.take<int64_t>(scan_partials_needed());
    }
    p.dpad = (dim + 7) / 8 * 8;
    for (int64_t e = p.chunks > 1 ? 2 * p.chunks : 0; e > 0 && p.levels < kLevels;) {
        p.entries[p.levels] = e;
        p.part[p.levels] = c.take<float>(e * p.dpad);
        p.part_row[p.levels] = c.take<int32_t>(e);
        p.levels++;
        if (e <= kJoinLast) break;
        e = 2 * ((e + kJoinChunk - 1) / kJoinChunk);
    }
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

static unsigned blocks_for(int64_t n, int64_t per) {
    const int64_t g = (n + per - 1) / per;
    AGNES_REQUIRE(g < (1 << 24), AGNES_ERR_RANGE, "the gradient is too large for one launch");
    return (unsigned)g;
}

// The gradient in either form: compact: the distinct rows alone.
static void grad(const agnes_matrix* g, const void* ids, agnes_dtype ids_dtype, float scale, bool accumulate,
                 bool compact, int64_t num_rows, int32_t* row_ids, const agnes_matrix* out, int64_t* count, void* ws,
                 hipStream_t st) {
    const int64_t n = g->rows, D = g->cols, max_rows = out->rows;
    if (n == 0 && compact) {
        AGNES_LAUNCH(k_embed_no_ids, dim3(grid_for(max_rows, 1024)), dim3(kBlock), 0, st, row_ids, max_rows, count);
        return;
    }
    const GradPlan p = plan_grad(n, num_rows, D, ws);
    const uint32_t V = (uint32_t)num_rows;
    const int chunk = chunk_of(n);
    const uint32_t *keys = p.keys[0], *perm = p.perm[0];
    if (n > 0)
        with_index(ids_dtype, [&](auto id) {
            typedef decltype(id) IdT;
            if (n <= kRankSort) {
                AGNES_LAUNCH((k_embed_rank_sort<IdT>), dim3(blocks_for(n, kBlock / kRankLanes)), dim3(kBlock), 0, st,
                             (const IdT*)ids, (int)n, num_rows, p.keys[0], p.perm[0], row_ids,
                             compact ? max_rows : 0);
                return;
            }
            AGNES_LAUNCH((k_embed_keys<IdT>), dim3(grid_for(n, 2048)), dim3(kBlock), 0, st, (const IdT*)ids, n,
                         p.chunks, num_rows, p.keys[0], p.sizes, row_ids, compact ? max_rows : 0);
            int bits = 1;
            while (((int64_t)1 << bits) <= num_rows) bits++;
            const int at = radix_sort_pairs32(p.keys[0], p.perm[0], p.keys[1], p.perm[1], p.sizes, n, bits, p.hist,
                                              p.dtot, st, true);
            keys = p.keys[at];
            perm = p.perm[at];
            if (compact) {
                AGNES_LAUNCH(k_embed_heads, dim3(blocks_for(n, kBlock)), dim3(kBlock), 0, st, keys, n, V, p.chunks,
                             p.heads);
                scan_counts(p.heads, p.rank, p.sizes + 1, p.chunks, count, p.partials, st);
            }
        });
    with_float(out->dtype, [&](auto to) {
        typedef decltype(to) TO;
        const bool nt = max_rows * D * (int64_t)sizeof(TO) > kStreamBytes;
        with_float(g->dtype, [&](auto ti) {
            typedef decltype(ti) TI;
            const RowShape shape = row_shape(std::max<int64_t>(D, 1), 16 / (int)sizeof(TI));
            const int fill_lanes = row_shape(D, 16 / (int)sizeof(TO)).lanes;
            // fewer rows per clearing workgroup where rows are long or few, so that there are enough of them
            const int fill_rows = D * (int64_t)sizeof(TO) >= 512 || num_rows < (1 << 18) ? 64 : kBlock;
            const bool clear = !compact && !accumulate;
            const int64_t sum_blocks = (p.chunks + kBlock / shape.lanes - 1) / (kBlock / shape.lanes) * shape.tiles;
            Sorted<TI> s{(const TI*)g->data, g->stride, keys, perm, n, V, chunk, p.chunks, compact, p.rank, row_ids,
                         count};
            Sink<TO> o{(TO*)out->data, out->stride, D, max_rows, scale, accumulate, p.part[0], p.part_row[0], p.dpad, nt};
            const int64_t all = sum_blocks + (clear ? (num_rows + fill_rows - 1) / fill_rows : 0);
            if (all == 0) return;
            const size_t lds = (size_t)(kBlock / shape.lanes + 1) * (chunk + 1) * 2 * sizeof(uint32_t);
            AGNES_LAUNCH((k_embed_sum<TI, TO>), dim3(blocks_for(all, 1)), dim3(kBlock), lds, st, s, o, shape.lanes,
                         shape.tiles, sum_blocks, fill_rows, fill_lanes);
        });
        if (D == 0) return;
        const RowShape shape = row_shape(p.dpad, 4);
        for (int l = 0; l < p.levels; l++) {
            const bool last = l + 1 == p.levels;
            // the last level: a group per few entries, since it follows each run to its end
            const int chunk = last ? 8 : kJoinChunk;
            const int64_t groups = (p.entries[l] + chunk - 1) / chunk;
            Sink<TO> o{(TO*)out->data, out->stride,          D,        max_rows,
                       scale,          accumulate,           last ? nullptr : p.part[l + 1],
                       last ? nullptr : p.part_row[l + 1], p.dpad,   nt};
            AGNES_LAUNCH((k_embed_join<TO>), dim3(blocks_for(groups, kBlock / shape.lanes) * shape.tiles), dim3(kBlock),
                         0, st, p.part[l], p.part_row[l], p.entries[l], chunk, last, o, shape.lanes, shape.tiles);
        }
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
// stream, so that the event recorded after the work covers both.  Neither can be
// captured: the gather's event lies outside the graph, and one recorded inside
// it says nothing about a replay.
static int64_t enter_batch(Batch& b, hipStream_t st) {
    AGNES_REQUIRE(b.state == kGathering || b.state == kDone, AGNES_ERR_INVALID, "the batch holds no finished hyperbatch");
    int dev = 0;
    AGNES_CHECK_HIP(hipGetDevice(&dev));
    AGNES_REQUIRE(dev == b.store->device, AGNES_ERR_INVALID, "the current device is not the batch's device");
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    AGNES_CHECK_HIP(hipStreamIsCapturing(st, &cs));
    AGNES_REQUIRE(cs == hipStreamCaptureStatusNone, AGNES_ERR_INVALID,
                  "a batch's embedding calls cannot be captured in a graph; take its node list and the calls on ids");
    AGNES_CHECK_HIP(hipStreamWaitEvent(st, b.gathered_at, 0));
    if (b.lookup_pending) AGNES_CHECK_HIP(hipStreamWaitEvent(st, b.lookup_done, 0));
    return b.node_off[b.H];
}

static void leave_batch(Batch& b, hipStream_t st) {
    AGNES_CHECK_HIP(hipEventRecord(b.lookup_done, st));
    b.lookup_pending = true;
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
