// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//   y[t] = scale table[ids[t]]            dtable[v] = scale sum over ids[t] = v of dy[t] + c[v]
//
// Both are bound by memory.  The gradient's sums must not depend on scheduling, so no value is added with an atomic: the tokens are
// sorted by id, stably, and the sorted list is cut into tiles of kTile tokens.  A wave takes a tile and 64 pieces of its columns
// and walks the tokens in order; the sum of an id whose tokens all lie in the tile is a row of the result, and the sums of an
// id that reaches over the tile's edges are kept and joined in the order of the tiles by a last pass.  So an
// id that half of the tokens have costs as little as a rare one.  Other waves of that last pass fill the rows without tokens.
//
// Sorting: runs of tokens are sorted in LDS, one workgroup each, and merged in one step: a token's place in the whole list is
// the number of tokens in front of it in every run, found by bisection.
#include "row_ops.hpp"

#include <algorithm>

namespace fg {
namespace {

constexpr int kTile = 16;                   // sorted tokens per tile
constexpr int kDigit = 6;                   // bits that one pass of the sort takes

// ---- lookup -----------------------------------------------------------------------------------------
// A wave takes rows << shift lanes: 64 >> shift rows at a time, 2^shift lanes each.
template <class T>
__global__ __launch_bounds__(256) void embedding(const T *table, int64_t ld, const void *ids, bool wide, float scale, T *y, int64_t ldy, int64_t tokens,
                                                 int vocab, int dim, int shift, int64_t group0) {
    constexpr int N = RowPiece<T>::N, AHEAD = 4;
    const int lane = threadIdx.x & 63, at = lane & ((1 << shift) - 1), rows = 64 >> shift, pieces = (dim + N - 1) / N;
    const int chunks = (pieces + (AHEAD << shift) - 1) / (AHEAD << shift);
    const int64_t wave = (group0 + blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int64_t t = wave / chunks * rows + (lane >> shift);
    const int first = (int)(wave % chunks) * (AHEAD << shift) + at;
    if (t >= tokens) return;
    const int id = load_index(ids, wide, t, vocab);
    const T *row = table + (int64_t)(id < 0 ? 0 : id) * ld;
    float v[AHEAD][N];
#pragma unroll
    for (int c = 0; c < AHEAD; ++c)
        if (first + (c << shift) < pieces) {
            if (id >= 0) load_piece(row, first + (c << shift), dim, v[c]);
            else
#pragma unroll
                for (int i = 0; i < N; ++i) v[c][i] = 0.f;
        }
#pragma unroll
    for (int c = 0; c < AHEAD; ++c)
        if (first + (c << shift) < pieces) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[c][i] = id >= 0 ? v[c][i] * scale : 0.f;
            store_piece(y + t * ldy, first + (c << shift), dim, v[c]);
        }
}

// ---- sorting ----------------------------------------------------------------------------------------
// Sorts run blockIdx.x of ITEMS * 64 WAVES tokens by id, stably; ids that name no row count as `vocab` and come last.  Also clears the
// marks of the rows that have tokens, and the count of open ids; a single run is the whole list, and its rows' marks are set here.
// A pass counts, per wave, the tokens of each of 64 digits, token by token in order (lanes with the same digit find each other by ballots), turns the counts
// into places, digits first and then waves, and moves the tokens.
template <int WAVES, int ITEMS>
__global__ __launch_bounds__(64 * WAVES) void embedding_sort(const void *ids, bool wide, int tokens, int vocab, int passes, uint32_t *keys, uint32_t *order, uint4 *present,
                                                             uint32_t *open_count) {
    constexpr int THREADS = 64 * WAVES, RUN = ITEMS * THREADS;
    __shared__ uint32_t key[RUN];
    __shared__ uint16_t pos[RUN];
    __shared__ uint32_t count[WAVES][1 << kDigit], total[WAVES];
    static_assert(WAVES << kDigit == THREADS, "one thread per counter");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = blockIdx.x * RUN, n = min(tokens - first, RUN);
    for (int64_t w = (int64_t)blockIdx.x * THREADS + threadIdx.x; w < (vocab + 15) / 16; w += (int64_t)gridDim.x * THREADS) present[w] = make_uint4(0, 0, 0, 0);
    if (blockIdx.x == 0 && threadIdx.x == 0) *open_count = 0;
#pragma unroll
    for (int r = 0; r < ITEMS; ++r) {
        const int i = (wave * ITEMS + r) * 64 + lane;
        const int id = i < n ? load_index(ids, wide, first + i, vocab) : -1;
        key[i] = i >= n ? (uint32_t)vocab + 1 : id < 0 ? (uint32_t)vocab : (uint32_t)id;
        pos[i] = (uint16_t)i;
    }
    for (int pass = 0; pass < passes; ++pass) {
        count[wave][lane] = 0;              // (a wave's own counters: LDS operations of a wave take place in order)
        __syncthreads();
        uint32_t k[ITEMS], at[ITEMS];
        int place[ITEMS];
        volatile uint32_t *mine = count[wave];
#pragma unroll
        for (int r = 0; r < ITEMS; ++r) {
            const int i = (wave * ITEMS + r) * 64 + lane;
            k[r] = key[i];
            at[r] = pos[i];
            const uint32_t digit = (k[r] >> (pass * kDigit)) & ((1 << kDigit) - 1);
            uint64_t same = ~0ull;          // lanes with the same digit
#pragma unroll
            for (int b = 0; b < kDigit; ++b) {
                const uint64_t set = __ballot((digit >> b) & 1);
                same &= (digit >> b) & 1 ? set : ~set;
            }
            const uint32_t before = (uint32_t)__popcll(same & ((1ull << lane) - 1)), base = mine[digit];
            __builtin_amdgcn_wave_barrier();
            if (before == 0) mine[digit] = base + (uint32_t)__popcll(same);
            __builtin_amdgcn_wave_barrier();
            place[r] = (int)(base + before);
        }
        __syncthreads();
        // where the tokens of (digit, wave) begin: the sum of all counters in front of it, digits first
        const int d = threadIdx.x / WAVES, w = threadIdx.x % WAVES;
        const uint32_t own = count[w][d];
        uint32_t sum = own;
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            const uint32_t other = __shfl_up(sum, s);
            if (lane >= s) sum += other;
        }
        if (lane == 63) total[wave] = sum;
        __syncthreads();
        uint32_t front = lane < wave ? total[lane] : 0;                 // of the waves in front (at most 16)
#pragma unroll
        for (int s = 8; s > 0; s /= 2) front += __shfl_xor(front, s);
        count[w][d] = sum - own + (uint32_t)__builtin_amdgcn_readfirstlane(front);
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ITEMS; ++r) {
            const uint32_t to = count[wave][(k[r] >> (pass * kDigit)) & ((1 << kDigit) - 1)] + place[r];
            key[to] = k[r];
            pos[to] = (uint16_t)at[r];
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < n; i += THREADS) {
        keys[first + i] = key[i];
        order[first + i] = first + pos[i];
        if (gridDim.x == 1 && key[i] < (uint32_t)vocab && (i == 0 || key[i - 1] != key[i])) ((uint8_t *)present)[key[i]] = 1;      // (cleared barriers ago)
    }
}

// Token i of the sorted runs goes to its place in the whole list: behind all smaller ids, and behind equal ones of earlier runs.  SIDE runs are
// searched side by side, a fixed number of steps: 8 where there are more than 4 (20624 tokens, six runs: 9.4 us, 11.7 four at a time).  Bound by the latency
// of the steps, one load each.
template <int SIDE>
__global__ __launch_bounds__(256) void embedding_merge(const uint32_t *keys, const uint32_t *order, int tokens, int run, uint32_t *all_keys, uint32_t *all_order,
                                                      int vocab, uint8_t *present) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= tokens) return;
    const int own = i / run, runs = (tokens + run - 1) / run;
    const uint32_t k = keys[i];
    int place = i - own * run;
    for (int r0 = 0; r0 < runs; r0 += SIDE) {
        int before[SIDE] = {};              // keys of the run that are in front
        for (int step = run; step > 0; step /= 2) {                     // (a power of two)
            uint32_t at[SIDE];
#pragma unroll
            for (int s = 0; s < SIDE; ++s) {
                const int r = r0 + s, to = before[s] + step;
                // (what is not there counts as behind)
                at[s] = r < runs && r != own && to <= min(run, tokens - r * run) ? keys[r * run + to - 1] : ~0u;
            }
#pragma unroll
            for (int s = 0; s < SIDE; ++s)
                if (at[s] < k || (at[s] == k && r0 + s < own)) before[s] += step;
        }
#pragma unroll
        for (int s = 0; s < SIDE; ++s) place += before[s];
    }
    all_keys[place] = k;
    all_order[place] = order[i];
    if (k < (uint32_t)vocab && (i == own * run || keys[i - 1] != k)) present[k] = 1;
}

// ---- sums -------------------------------------------------------------------------------------------
struct EmbeddingGradArgs {
    const void *dy;
    const void *c;
    void *out;
    const uint32_t *keys, *order;
    const uint8_t *present;                 // a byte for each row: it has tokens.  (Bits would be set by atomics, which the XCDs take one after another: 20624
                                            // tokens of 4993 ids 29 us in embedding_merge, 9.4 so.)
    float *open;                            // tile t: the sum of the id that comes in over its front at 2 t dim, of the one that goes out at (2 t + 1) dim
    uint32_t *open_count, *open_tiles;      // tiles that an id which began there goes out of, in any order
    int64_t lddy, ldc, ldo;
    int tokens, vocab, dim, tiles, chunks;  // chunks: of 64 pieces, that cover the columns
    int64_t join_groups;                    // workgroups that join sums, in front of those that fill rows
    int64_t group0;                         // the launch's first workgroup
    int shift;                              // lanes of a row to fill
    float scale;
};

// Piece p of what is there in row id.
template <class D, int N>
__device__ __forceinline__ typename RowPiece<D, N>::vec embedding_there(const EmbeddingGradArgs &a, uint32_t id, int p) {
    return load_raw<D, N>((const D *)a.c + (int64_t)id * a.ldc, p, a.dim);
}
// A row's sum becomes the result: scaled, what is there added, rounded once.
template <class D, bool ADD, int N>
__device__ __forceinline__ void embedding_finish(const EmbeddingGradArgs &a, uint32_t id, int p, const typename RowPiece<D, N>::vec &there, float (&sum)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = ADD ? sum[i] * a.scale + (float)there[i] : sum[i] * a.scale;
    store_piece((D *)a.out + (int64_t)id * a.ldo, p, a.dim, sum);
}

// ADD: there is a matrix to add to.  Its rows are requested with those of dy (when each was read at the end of its sum: 9999 tokens of 1001 FP32
// 38.9 us, 33.1 so).
template <class T, class D, bool ADD>
__global__ __launch_bounds__(256) void embedding_sums(const EmbeddingGradArgs a) {
    constexpr int N = RowPiece<T>::N;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), pieces = (a.dim + N - 1) / N;
    const int64_t item = (a.group0 + blockIdx.x) * 4 + wave;
    const int tile = (int)(item / a.chunks), p = (int)(item % a.chunks) * 64 + lane;
    if (tile >= a.tiles) return;
    const int i0 = tile * kTile, n = min(kTile, a.tokens - i0);
    const bool on = p < pieces;             // (lanes without columns hold tokens all the same)
    // the tokens of the tile, one per lane; and whether the ids at its edges reach beyond it
    const uint32_t key_of_lane = a.keys[i0 + min(lane, n - 1)], token_of_lane = a.order[i0 + min(lane, n - 1)];
    const bool comes_in = i0 > 0 && a.keys[i0 - 1] == a.keys[i0], goes_out = i0 + n < a.tokens && a.keys[i0 + n] == a.keys[i0 + n - 1];
    // the tokens that end an id's sum, and those of them whose sum is all of the tile's
    const uint32_t next_of_lane = __shfl_down(key_of_lane, 1);
    const uint64_t ends = __ballot(lane < n && key_of_lane < (uint32_t)a.vocab && (lane + 1 == n || next_of_lane != key_of_lane));
    uint64_t closed = ends;
    if (comes_in) closed &= ~(ends & -ends);                            // (the first)
    if (goes_out) closed &= ~(1ull << (n - 1));
    float sum[N] = {};
    typename RowPiece<T>::vec v[kTile];     // (as stored: as FP32 they take the registers of three waves per SIMD)
    typename RowPiece<D, N>::vec there[ADD ? kTile : 1];
#pragma unroll
    for (int e = 0; e < kTile; ++e)
        if (ADD && on && (closed >> e & 1)) there[ADD ? e : 0] = embedding_there<D, N>(a, __builtin_amdgcn_readlane(key_of_lane, e), p);
#pragma unroll
    for (int e = 0; e < kTile; ++e)
        if (e < n && on) v[e] = load_raw<T, N>((const T *)a.dy + (int64_t)(uint32_t)__builtin_amdgcn_readlane(token_of_lane, e) * a.lddy, p, a.dim);
    bool in = comes_in;                     // the current id began in an earlier tile
#pragma unroll
    for (int e = 0; e < kTile; ++e) {
        const uint32_t id = __builtin_amdgcn_readlane(key_of_lane, e);
        if (e < n && id < (uint32_t)a.vocab) {                          // (ids that name no row are the last)
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] += (float)v[e][i];
            if (ends >> e & 1) {
                if (on) {
                    if (closed >> e & 1) embedding_finish<D, ADD>(a, id, p, there[ADD ? e : 0], sum);
                    else store_piece(a.open + ((int64_t)tile * 2 + (in ? 0 : 1)) * a.dim, p, a.dim, sum);
                    if (!in && e + 1 == n && goes_out && p == 0) a.open_tiles[atomicAdd(a.open_count, 1u)] = tile;
                }
                in = false;
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] = 0.f;
            }
        }
    }
}

// Rows without tokens: zeros, or what is there.  A lane looks at the marks of ROWS rows at once: 4 where it only stores (65536 rows of 4096 bfloat16 74 us, 79 one
// by one, 77 with 16), one where it loads too (50001 of 1001 FP32 73 us, 81 with 4: rows follow each other).
template <bool ADD> constexpr int kFillRows = ADD ? 1 : 4;
template <class T, class D, bool ADD>
__device__ __forceinline__ void embedding_fill(const EmbeddingGradArgs &a, int64_t item, int lane, int pieces) {
    constexpr int N = RowPiece<T>::N, AHEAD = 4, ROWS = kFillRows<ADD>;
    const int at = lane & ((1 << a.shift) - 1), rows = 64 >> a.shift, chunks = (pieces + (AHEAD << a.shift) - 1) / (AHEAD << a.shift);
    const int64_t row0 = (item / chunks * rows + (lane >> a.shift)) * ROWS;
    const int first = (int)(item % chunks) * (AHEAD << a.shift) + at;
    if (row0 >= a.vocab) return;
    const uint32_t marks = ROWS == 1 ? a.present[row0] : ((const uint32_t *)a.present)[row0 / 4];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int64_t row = row0 + r;
        if (row >= a.vocab || (marks >> r * 8 & 1)) continue;
        float v[AHEAD][N] = {};
        if (ADD) {
#pragma unroll
            for (int c = 0; c < AHEAD; ++c)
                if (first + (c << a.shift) < pieces) load_piece((const D *)a.c + row * a.ldc, first + (c << a.shift), a.dim, v[c]);
        }
#pragma unroll
        for (int c = 0; c < AHEAD; ++c)
            if (first + (c << a.shift) < pieces) store_piece((D *)a.out + row * a.ldo, first + (c << a.shift), a.dim, v[c]);
    }
}

// Joins the sums of an id that goes out of a tile it began in: that tile's, then those of the tiles that it comes into.  A workgroup takes one such id
// at a time and 64 pieces of its columns; its waves add up a quarter of the tiles each, and the quarters are added in order.  That is a chain of
// latencies (20 us for 16384 tokens in a launch of its own), which the filling of rows in the other workgroups covers.
template <class T, class D, bool ADD>
__global__ __launch_bounds__(256) void embedding_join(const EmbeddingGradArgs a) {
    constexpr int N = RowPiece<T>::N, AHEAD = 8, WAVES = 4;
    __shared__ float part[WAVES][N][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), pieces = (a.dim + N - 1) / N;
    const int64_t group = a.group0 + blockIdx.x;
    if (group >= a.join_groups) {
        embedding_fill<T, D, ADD>(a, (group - a.join_groups) * WAVES + wave, lane, pieces);
        return;
    }
    const int p = (int)(group % a.chunks) * 64 + lane;
    const uint32_t ids = *a.open_count;
    for (int64_t n = group / a.chunks; n < ids; n += a.join_groups / a.chunks) {
        const int tile = a.open_tiles[n];
        const uint32_t id = a.keys[(int64_t)tile * kTile + kTile - 1];
        // how many tiles it comes into: those behind, as long as they begin with it
        int into = 0;
        for (int stride = 64; stride > 0; stride /= 64)
            for (;;) {
                const int64_t t = tile + into + (int64_t)stride * (lane + 1);
                const uint64_t same = __ballot(t < a.tiles && a.keys[t * kTile] == id);
                const int more = same == ~0ull ? 64 : __builtin_ctzll(~same);
                into += more * stride;
                if (more < 64) break;
            }
        const int each = (into + WAVES - 1) / WAVES, first = wave * each, last = min(first + each, into);
        float sum[N] = {};
        if (p < pieces) {
            if (wave == 0) load_piece(a.open + ((int64_t)tile * 2 + 1) * a.dim, p, a.dim, sum);
            for (int t0 = first; t0 < last; t0 += AHEAD) {
                float v[AHEAD][N];
#pragma unroll
                for (int t = 0; t < AHEAD; ++t)
                    if (t0 + t < last) load_piece(a.open + (int64_t)(tile + 1 + t0 + t) * 2 * a.dim, p, a.dim, v[t]);
#pragma unroll
                for (int t = 0; t < AHEAD; ++t)
                    if (t0 + t < last)
#pragma unroll
                        for (int i = 0; i < N; ++i) sum[i] += v[t][i];
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) part[wave][i][lane] = sum[i];
        __syncthreads();
        if (wave == 0 && p < pieces) {
#pragma unroll
            for (int w = 1; w < WAVES; ++w)
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] += part[w][i][lane];
            typename RowPiece<D, N>::vec there = {};
            if (ADD) there = embedding_there<D, N>(a, id, p);
            embedding_finish<D, ADD>(a, id, p, there, sum);
        }
        __syncthreads();
    }
}

// ---- host ----------------------------------------------------------------------------------------------
// Lanes of a row: as many as have a piece each, at most a wave (as a power of two).
int lanes_shift(int pieces) {
    int s = 0;
    while (s < 6 && (1 << s) < pieces) ++s;
    return s;
}
// Tokens of a run (powers of two: embedding_merge).  Few tokens are sorted by few waves or few items a lane: up to 256 tokens 4.5 us, and 11.6 in a run of 4096;
// 1024 tokens 7.2 us and 11.
int run_of(int64_t tokens) { return tokens <= 256 ? 256 : tokens <= 1024 ? 1024 : tokens <= 65536 ? 4096 : 16384; }

// The workspace: sorted runs, the whole list, the rows that have tokens, open sums.
struct EmbeddingSpace {
    int64_t keys, order, all_keys, all_order, present, open_count, open_tiles, open, bytes;
    EmbeddingSpace(int64_t tokens, int64_t vocab, int64_t dim) {
        auto up = [](int64_t b) { return (b + 255) / 256 * 256; };
        keys = 0;
        order = keys + up(4 * tokens);
        all_keys = order + up(4 * tokens);
        all_order = all_keys + up(4 * tokens);
        present = all_order + up(4 * tokens);
        open_count = present + up(vocab);
        open_tiles = open_count + 256;
        open = open_tiles + up((tokens + kTile - 1) / kTile * 4);
        bytes = open + (tokens + kTile - 1) / kTile * 2 * dim * 4;
    }
};

template <class F> void with_element(int dtype, F &&f) {
    switch (dtype) {
        case FG_F16: f(f16_t{}); break;
        case FG_BF16: f(bf16_t{}); break;
        default: f(float{});
    }
}

fg_status check_embedding(int64_t tokens, int64_t vocab, int64_t dim, const void *ids, int32_t index_dtype) {
    if (tokens < 0 || vocab < 0 || dim < 0) return fail(FG_ERR_SHAPE, "negative size: %lld tokens, %lld rows of %lld", (long long)tokens, (long long)vocab, (long long)dim);
    if (tokens > (1 << 30) || vocab > (1 << 30) || dim > (1 << 24)) return fail(FG_ERR_UNSUPPORTED, "sizes above 2^30 (rows of more than 2^24) are not supported");
    return check_indices("ids", ids, index_dtype, tokens);
}

}  // namespace

hipError_t load_embedding_kernels() {
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)embedding<float>);
}

}  // namespace fg

using namespace fg;

extern "C" {

fg_status fg_embedding(int64_t tokens, int64_t vocab, int64_t dim, const fg_matrix *table, const void *ids, int32_t index_dtype, float scale,
                       const fg_matrix *Y, void *hip_stream) {
    if (fg_status st = check_embedding(tokens, vocab, dim, ids, index_dtype)) return st;
    if (fg_status st = check_rows("table", table, vocab, dim)) return st;
    if (fg_status st = check_rows("Y", Y, tokens, dim)) return st;
    if (table->dtype != Y->dtype) return fail(FG_ERR_UNSUPPORTED, "the table and Y must have the same element type");
    if (tokens == 0 || dim == 0) return FG_OK;
    Launches enqueue(hip_stream);
    with_element(Y->dtype, [&](auto t) {
        using T = decltype(t);
        const int pieces = (int)((dim + RowPiece<T>::N - 1) / RowPiece<T>::N), shift = lanes_shift((pieces + 3) / 4);
        const int64_t waves = (tokens + (64 >> shift) - 1) / (64 >> shift) * ((pieces + (4 << shift) - 1) / (4 << shift));
        in_parts((waves + 3) / 4, [&](int64_t first, dim3 grid) {
            enqueue(embedding<T>, grid, dim3(256), (const T *)table->re, table->ld, ids, index_dtype == FG_I64, scale,
                               (T *)Y->re, Y->ld, tokens, (int)vocab, (int)dim, shift, first);
        });
    });
    return enqueue.status("embedding");
}

int64_t fg_embedding_grad_workspace(int64_t tokens, int64_t vocab, int64_t dim) {
    if (tokens < 0 || vocab <= 0 || dim <= 0) return 0;
    return EmbeddingSpace(tokens, vocab, dim).bytes;
}

fg_status fg_embedding_grad(int64_t tokens, int64_t vocab, int64_t dim, const fg_matrix *dY, const void *ids, int32_t index_dtype, float scale,
                            const fg_matrix *Cin, const fg_matrix *dtable, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (fg_status st = check_embedding(tokens, vocab, dim, ids, index_dtype)) return st;
    if (fg_status st = check_rows("dY", dY, tokens, dim, true)) return st;
    if (fg_status st = check_rows("dtable", dtable, vocab, dim)) return st;
    if (dtable->dtype != dY->dtype && dtable->dtype != FG_F32) return fail(FG_ERR_UNSUPPORTED, "dtable must be FG_F32 or of the type of dY");
    if (Cin) {
        if (fg_status st = check_rows("Cin", Cin, vocab, dim)) return st;
        if (Cin->dtype != dtable->dtype) return fail(FG_ERR_UNSUPPORTED, "Cin and dtable must have the same element type");
        if (Cin->re == dtable->re && Cin->ld != dtable->ld) return fail(FG_ERR_LAYOUT, "Cin in the place of dtable must have its leading dimension");
    }
    if (vocab == 0 || dim == 0) return FG_OK;
    const EmbeddingSpace at(tokens, vocab, dim);
    if (fg_status st = check_workspace(workspace, workspace_bytes, at.bytes)) return st;
    char *w = (char *)workspace;
    uint32_t *keys = (uint32_t *)(w + at.keys), *order = (uint32_t *)(w + at.order);
    uint8_t *present = (uint8_t *)(w + at.present);
    uint32_t *open_count = (uint32_t *)(w + at.open_count), *open_tiles = (uint32_t *)(w + at.open_tiles);
    uint32_t *all_keys = (uint32_t *)(w + at.all_keys), *all_order = (uint32_t *)(w + at.all_order);
    Launches enqueue(hip_stream);
    int passes = 1;
    while (((vocab + 1) >> (passes * kDigit)) != 0) ++passes;             // the largest key is vocab + 1
    const bool wide = index_dtype == FG_I64;
    const int run = run_of(tokens);
    const unsigned runs = (unsigned)std::max<int64_t>(1, (tokens + run - 1) / run);
    auto sort = [&](auto waves, auto items) {
        constexpr int WAVES = decltype(waves)::value, ITEMS = decltype(items)::value;
        enqueue(embedding_sort<WAVES, ITEMS>, dim3(runs), dim3(64 * WAVES), ids, wide, (int)tokens, (int)vocab, passes, runs == 1 ? all_keys : keys,
                           runs == 1 ? all_order : order, (uint4 *)present, open_count);
    };
    using std::integral_constant;
    if (run == 256) sort(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    else if (run == 1024) sort(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (run == 4096) sort(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    else sort(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    auto merge = [&](auto side) {
        enqueue(embedding_merge<decltype(side)::value>, dim3((unsigned)((tokens + 255) / 256)), dim3(256), keys, order, (int)tokens, run, all_keys,
                           all_order, (int)vocab, present);
    };
    if (runs > 4) merge(integral_constant<int, 8>{});
    else if (runs > 1) merge(integral_constant<int, 4>{});
    if (fg_status st = enqueue.status("embedding_sort")) return st;
    const bool in_place = Cin && Cin->re == dtable->re;
    auto launch = [&](auto t, auto d) {
        using T = decltype(t);
        using D = decltype(d);
        const int64_t pieces = (dim + RowPiece<T>::N - 1) / RowPiece<T>::N, tiles = (tokens + kTile - 1) / kTile, chunks = (pieces + 63) / 64;
        const int shift = lanes_shift((int)((pieces + 3) / 4));
        const int64_t joins = tiles > 1 ? std::min<int64_t>(tiles - 1, 512) * chunks : 0;
        EmbeddingGradArgs a = {dY->re, Cin ? Cin->re : nullptr, dtable->re, all_keys, all_order, present, (float *)(w + at.open), open_count, open_tiles, dY->ld,
                                     Cin ? Cin->ld : 0, dtable->ld, (int)tokens, (int)vocab, (int)dim, (int)tiles, (int)chunks, joins, 0, shift, scale};
        auto run = [&](auto tag) {
            constexpr bool ADD = decltype(tag)::value;
            const int64_t rows = (64 >> shift) * kFillRows<ADD>, fills = in_place ? 0 : (vocab + rows - 1) / rows * ((pieces + (4 << shift) - 1) / (4 << shift));
            const int64_t rest = joins + (fills + 3) / 4;
            in_parts((tiles * chunks + 3) / 4, [&](int64_t first, dim3 grid) {
                a.group0 = first;
                enqueue(embedding_sums<T, D, ADD>, grid, dim3(256), a);
            });
            in_parts(rest, [&](int64_t first, dim3 grid) {
                a.group0 = first;
                enqueue(embedding_join<T, D, ADD>, grid, dim3(256), a);
            });
        };
        if (Cin) run(std::true_type{});
        else run(std::false_type{});
    };
    with_element(dY->dtype, [&](auto t) {
        if (dtable->dtype == FG_F32) launch(t, float{});
        else launch(t, t);
    });
    return enqueue.status("embedding_grad");
}

}  // extern "C"
