// Embedding lookup with scaling, and its gradient.
//
//   mgwfbp_embed        out[t,:] = sum over tables k, in order, of scale_k * table_k[id_k[t], :]
//   mgwfbp_embed_grad   grad[r,:] = scale * sum over the tokens t with id[t] = r of dy[t,:]   (+ grad[r,:])
//
// Sums are binary32 and rounded once.  An id outside the table stands for no row.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "device_types.h"
#include "mgwfbp_layers.h"

namespace {

using namespace ops;

thread_local int g_last_hip_error = 0;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256;
constexpr int64_t MOST_TOKENS = int64_t(1) << 26, MOST_DIM = int64_t(1) << 23;

// ---------------------------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------------------------

struct Table {
    const void* rows;
    const void* ids;
    int64_t n_rows, stride;
    float scale;
    int32_t id_type;
};
struct EmbedArgs {
    Table table[MGWFBP_MAX_TABLES];
    void* out;
    int64_t out_stride, tokens, dim;
    uint32_t vecs;             // vectors of a row
    uint32_t page;             // tokens per blockIdx.y, so that a page's vectors are counted in 32 bits
};

__device__ __forceinline__ int64_t id_at(const void* ids, int32_t id_type, int64_t t) {
    return id_type == MGWFBP_I64 ? static_cast<const int64_t*>(ids)[t] : static_cast<const int32_t*>(ids)[t];
}

// One lane for eight columns of a token.  Lanes run over the vectors of a token and on into the next token, so that
// narrow tables fill wavefronts too.  All of a token's ids, then all its rows are asked for at once: two waits for memory, which is
// what bounds a short call (1 token of 1024 columns from three binary32 tables: 1.8 us).  4096 tokens: 6.3 us, 27 MB at 4.4 TB/s.
template <typename TabT, typename OutT, int K>
__global__ __launch_bounds__(THREADS) void embed_kernel(EmbedArgs A) {
    const uint32_t at = blockIdx.x * THREADS + threadIdx.x;
    const uint32_t in_page = at / A.vecs, v = at - in_page * A.vecs;
    const int64_t t = static_cast<int64_t>(blockIdx.y) * A.page + in_page;
    if (in_page >= A.page || t >= A.tokens) return;
    const int64_t col = static_cast<int64_t>(v) * VEC;
    const int n = static_cast<int>(min(A.dim - col, static_cast<int64_t>(VEC)));
    int64_t id[K];
    bool here[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        id[k] = id_at(A.table[k].ids, A.table[k].id_type, t);
        here[k] = static_cast<uint64_t>(id[k]) < static_cast<uint64_t>(A.table[k].n_rows);
    }
    Raw8<TabT> row[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
        row[k] = load8(static_cast<const TabT*>(A.table[k].rows) + (here[k] ? id[k] : 0) * A.table[k].stride + col, here[k] ? n : 0);
    float sum[VEC] = {};
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float x = here[k] ? A.table[k].scale * get(row[k], i) : 0.f;
            sum[i] = k == 0 ? x : sum[i] + x;
        }
    store8(static_cast<OutT*>(A.out) + t * A.out_stride + col, sum, n);
}

// ---------------------------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------------------------
//
// Up to FEW_TOKENS_MOST tokens need no order: every row looks for its own (direct_kernel; one launch, see its rule).
// A table of up to FEW_ROWS rows (token types) needs none either: every lane keeps a sum for each row (few_rows_kernel, and
// few_join_kernel where there are several chunks of tokens).  4096 tokens of 1024 bfloat16 columns and 2 rows: 8 us, and 21
// the other way.  For the rest:
// 1. Tokens are ordered by (row, token).  Up to RANKED_TOKENS tokens a token's place is the number of tokens before it,
//    counted by comparing it with every other one (rank_kernel): one launch, no dependence between workgroups.  Beyond that,
//    a radix sort by 8 bits at a time.  Tokens without a row come last.
// 2. The ordered tokens are cut into chunks of a fixed length; lanes sum a chunk's stretches of one row each
//    (sum_kernel).  Rows of one or two chunks are written to the gradient, longer ones in stretches to the workspace.  In the
//    same launch, rows that are not among the ordered tokens are cleared.
// 3. The stretches of longer rows are joined, in order (join_kernel).
//
// The order of every sum follows from the sizes and ids alone: the same call gives the same bits.

struct GradArgs {
    const void* ids;
    const void* dy;
    void* grad;
    int64_t dy_stride, grad_stride, n_rows, dim, padding_row;
    int64_t tokens;
    uint32_t* order;           // [tokens] token at a place of the order
    int32_t* row;              // [tokens] its row, n_rows if it has none
    float* partial;            // [2 * chunks][dim_padded]: a chunk's first and its last stretch
    u32x2* joins;              // [1 + chunks] how many rows have to be joined; the chunks they begin in and the rows, in any order
    uint32_t* other_order;     // radix sort: the other side of a pass, and the counts of every workgroup
    int32_t* other_row;
    uint32_t* counts;          // [blocks][256]
    int64_t dim_padded;
    float scale;
    int32_t id_type, accumulate;
    uint32_t chunk, chunks;    // tokens per chunk, number of chunks
    uint32_t vecs, page;       // vectors of a row; chunks per blockIdx.y
    uint32_t sum_blocks;       // workgroups that sum; the rest clear clear_rows rows each
    uint32_t clear_rows;
    uint32_t join_width;       // lanes side by side that join a row
    uint32_t items, shift, from_ids;   // radix sort: tokens per workgroup, first bit of the digit, first pass
};

__device__ __forceinline__ int32_t row_of(const GradArgs& A, int64_t id) {
    return static_cast<uint64_t>(id) < static_cast<uint64_t>(A.n_rows) && id != A.padding_row ? static_cast<int32_t>(id)
                                                                                              : static_cast<int32_t>(A.n_rows);
}

// The first place of the order with a row of r or more, by a wavefront: 64 places looked at in a turn, so that two turns find
// one of 4096 and three one of 260 thousand.
__device__ __forceinline__ uint32_t first_place(const GradArgs& A, int32_t r) {
    const uint32_t lane = threadIdx.x % 64;
    uint32_t lo = 0, hi = static_cast<uint32_t>(A.tokens);               // it is one of lo .. hi
    while (lo < hi) {
        const uint32_t step = (hi - lo + 63) / 64, at = lo + lane * step;
        const uint32_t below = __popcll(__ballot(at < hi && A.row[min(at, hi - 1)] < r));
        if (below == 0) break;
        hi = min(lo + below * step, hi);
        lo += (below - 1) * step + 1;
    }
    return lo;
}

// Clears those rows from first on, at most A.clear_rows, that are not among the ordered tokens.  It looks at every place of these rows, which
// is nothing beside the sums but for very many tokens in very few rows: a million in 8 rows of 1024 bfloat16 columns 2.0 ms, of which
// the sums are 0.42; in 100 rows 0.68.
template <typename GradT> __device__ void clear_absent_rows(const GradArgs& A, int64_t first) {
    __shared__ uint8_t absent[THREADS];
    __shared__ uint32_t place[2];
    const int rows = static_cast<int>(min(A.n_rows - first, static_cast<int64_t>(A.clear_rows)));
    absent[threadIdx.x] = 1;
    const uint32_t wave = threadIdx.x / 64;
    if (wave < 2) {                                                  // the places of the first row and of the first row behind
        const uint32_t at = first_place(A, static_cast<int32_t>(first) + (wave == 0 ? 0 : rows));
        if (threadIdx.x % 64 == 0) place[wave] = at;
    }
    __syncthreads();
    for (uint32_t at = place[0] + threadIdx.x; at < place[1]; at += THREADS) absent[A.row[at] - first] = 0;
    __syncthreads();
    const float zeros[VEC] = {};
    const uint32_t at_once = min(A.vecs, static_cast<uint32_t>(THREADS)), beside = THREADS / at_once;
    const uint32_t beside_no = threadIdx.x / at_once;
    if (beside_no >= beside) return;
    for (int i = beside_no; i < rows; i += beside) {
        if (!absent[i]) continue;
        GradT* const g = static_cast<GradT*>(A.grad) + (first + i) * A.grad_stride;
        for (uint32_t v = threadIdx.x - beside_no * at_once; v < A.vecs; v += at_once)
            store8(g + static_cast<int64_t>(v) * VEC, zeros, static_cast<int>(min(A.dim - static_cast<int64_t>(v) * VEC, static_cast<int64_t>(VEC))));
    }
}

constexpr int RANK_EACH = 8;               // tokens that a workgroup ranks
constexpr int RANK_AHEAD = 16;             // ids that a lane has on their way
constexpr int64_t RANKED_TOKENS = 8192;
constexpr int64_t NARROW_ROWS = (int64_t(1) << 18) - 1;      // (row, token) of so many rows fits 31 bits

// The place of a token is the number of pairs (row, token) below its own.  A wavefront compares 64 others at a time with
// each of the workgroup's tokens; a comparison is one vector instruction and the count of its mask two scalar ones.  4096
// tokens are 16 M comparisons, 260 thousand instructions: a microsecond of the chip.  What takes its time is that ids come
// from memory, all at once.
template <typename Key, typename IdT> __global__ __launch_bounds__(THREADS) void rank_kernel(GradArgs A) {
    constexpr int TOKEN_BITS = sizeof(Key) == 4 ? 13 : 32;
    static_assert(RANKED_TOKENS <= 1 << 13, "tokens of narrow keys");
    if (blockIdx.x == 0 && threadIdx.x == 0) A.joins[0] = u32x2{0, 0};
    __shared__ uint32_t below[THREADS / 64][RANK_EACH];
    __shared__ int32_t own_row[RANK_EACH];
    const uint32_t n = static_cast<uint32_t>(A.tokens);
    const uint32_t first = blockIdx.x * RANK_EACH;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const IdT* const ids = static_cast<const IdT*>(A.ids);
    auto key_of = [&](IdT id, uint32_t t) { return static_cast<Key>(static_cast<uint32_t>(row_of(A, id))) << TOKEN_BITS | t; };
    IdT other[RANK_AHEAD];                                   // ids of the next turn
    auto look = [&](uint32_t s0) {
#pragma unroll
        for (int j = 0; j < RANK_AHEAD; ++j) other[j] = ids[min(s0 + j * THREADS + lane, n - 1)];
    };
    look(wave * 64);
    IdT mine[RANK_EACH];
#pragma unroll
    for (int r = 0; r < RANK_EACH; ++r) mine[r] = ids[min(first + r, n - 1)];
    Key own[RANK_EACH];
    uint32_t count[RANK_EACH];
#pragma unroll
    for (int r = 0; r < RANK_EACH; ++r) {
        own[r] = key_of(mine[r], min(first + r, n - 1));
        count[r] = 0;
        if (threadIdx.x == 0) own_row[r] = static_cast<int32_t>(own[r] >> TOKEN_BITS);
    }
    for (uint32_t s0 = wave * 64; s0 < n; s0 += RANK_AHEAD * THREADS) {
        Key key[RANK_AHEAD];
#pragma unroll
        for (int j = 0; j < RANK_AHEAD; ++j) {
            const uint32_t s = s0 + j * THREADS + lane;
            const Key k = key_of(other[j], min(s, n - 1));
            key[j] = s < n ? k : ~Key(0);
        }
        if (s0 + RANK_AHEAD * THREADS < n) look(s0 + RANK_AHEAD * THREADS);
#pragma unroll
        for (int j = 0; j < RANK_AHEAD; ++j)
#pragma unroll
            for (int r = 0; r < RANK_EACH; ++r) count[r] += __popcll(__ballot(key[j] < own[r]));
    }
    if (lane == 0)
#pragma unroll
        for (int r = 0; r < RANK_EACH; ++r) below[wave][r] = count[r];
    __syncthreads();
    const uint32_t t = first + threadIdx.x;
    if (threadIdx.x < RANK_EACH && t < n) {
        uint32_t place = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) place += below[w][threadIdx.x];
        A.order[place] = t;
        A.row[place] = own_row[threadIdx.x];
    }
}

// ---- radix sort: a pass orders by one digit of the row and keeps the order of equal digits ----
constexpr int DIGITS = 256;
constexpr int WAVES = THREADS / 64;

__device__ __forceinline__ int32_t sort_row(const GradArgs& A, int64_t at) { return A.from_ids ? row_of(A, id_at(A.ids, A.id_type, at)) : A.other_row[at]; }

// How often each digit occurs among a workgroup's tokens.  (Counted for the next pass by the move before it, with atomic additions
// in memory, it saves a launch of 5 us and costs 10.)
__global__ __launch_bounds__(THREADS) void digit_kernel(GradArgs A) {
    if (blockIdx.x == 0 && threadIdx.x == 0) A.joins[0] = u32x2{0, 0};
    __shared__ uint32_t count[DIGITS];
    count[threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = static_cast<int64_t>(blockIdx.x) * A.items, end = min(first + A.items, A.tokens);
#pragma unroll 4
    for (int64_t at = first + threadIdx.x; at < end; at += THREADS)
        atomicAdd(&count[(static_cast<uint32_t>(sort_row(A, at)) >> A.shift) % DIGITS], 1u);
    __syncthreads();
    A.counts[static_cast<int64_t>(blockIdx.x) * DIGITS + threadIdx.x] = count[threadIdx.x];
}

// Moves a workgroup's tokens to their places: behind every smaller digit, behind the same digit of the workgroups and
// wavefronts before, in order within the wavefront.
__global__ __launch_bounds__(THREADS) void move_kernel(GradArgs A) {
    __shared__ uint32_t scan[DIGITS];
    __shared__ uint32_t place[WAVES][DIGITS];
    const uint32_t d = threadIdx.x, lane = d % 64, wave = d / 64;
    uint32_t before = 0, all = 0;
#pragma unroll 16
    for (uint32_t b = 0; b < gridDim.x; ++b) {
        const uint32_t c = A.counts[static_cast<int64_t>(b) * DIGITS + d];
        before += b < blockIdx.x ? c : 0;
        all += c;
    }
    scan[d] = all;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) place[w][d] = 0;
    __syncthreads();
    for (uint32_t step = 1; step < DIGITS; step *= 2) {
        const uint32_t add = d >= step ? scan[d - step] : 0;
        __syncthreads();
        scan[d] += add;
        __syncthreads();
    }
    const int64_t part = A.items / WAVES;                    // a multiple of 64
    const int64_t first = static_cast<int64_t>(blockIdx.x) * A.items + wave * part, end = min(first + part, A.tokens);
    for (int64_t at = first + lane; at < end; at += 64)
        atomicAdd(&place[wave][(static_cast<uint32_t>(sort_row(A, at)) >> A.shift) % DIGITS], 1u);
    __syncthreads();
    uint32_t next = scan[d] - all + before;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const uint32_t c = place[w][d];
        place[w][d] = next;
        next += c;
    }
    __syncthreads();
    for (int64_t at0 = first; at0 < end; at0 += 64) {        // the same number of turns for every lane of the wavefront
        const int64_t at = at0 + lane;
        const bool here = at < end;
        const int32_t r = here ? sort_row(A, at) : 0;
        const uint32_t digit = (static_cast<uint32_t>(r) >> A.shift) % DIGITS;
        uint64_t same = __ballot(here);
#pragma unroll
        for (int bit = 0; bit < 8; ++bit) {
            const bool set = (digit >> bit & 1) != 0;
            const uint64_t mask = __ballot(set);
            same &= set ? mask : ~mask;
        }
        if (here) {
            const uint32_t ahead = __popcll(same & ((uint64_t(1) << lane) - 1));
            const uint32_t to = place[wave][digit] + ahead;
            A.order[to] = A.from_ids ? static_cast<uint32_t>(at) : A.other_order[at];
            A.row[to] = r;
        }
        // the places are read by lanes that others have written for: no barrier between the lanes of a wavefront, but an order
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (here && (same >> lane) == 1) place[wave][digit] += __popcll(same);      // the last lane of each digit
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// ---- sums ----

template <typename GradT, bool ACCUMULATE>
__device__ __forceinline__ void write_row(const GradArgs& A, int32_t r, int64_t col, int n, const float (&sum)[VEC]) {
    GradT* const g = static_cast<GradT*>(A.grad) + r * A.grad_stride + col;
    float x[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = sum[i] * A.scale;
    if constexpr (ACCUMULATE) {
        const Raw8<GradT> had = load8(g, n);
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[i] += get(had, i);
    }
    store8(g, x, n);
}

__device__ __forceinline__ void write_partial(const GradArgs& A, uint32_t which, int64_t col, const float (&sum)[VEC]) {
    float* const p = A.partial + which * A.dim_padded + col;
    *reinterpret_cast<f32x4*>(p) = f32x4{sum[0], sum[1], sum[2], sum[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{sum[4], sum[5], sum[6], sum[7]};
}

// One lane for eight columns of a chunk.  A row that begins in a chunk and ends in the next one is summed by the lanes of the
// first alone; only rows that reach further are joined.  65543 tokens of 1024 binary32 columns into 30522 rows, 0.4 GB: 88 us, 4.5
// TB/s, the rate of a copy.  4096 bfloat16 tokens into as many rows: 13 us, of which writing 62 MB takes 9.  What stands once for every
// token in the code is kept small (the stretch from before the chunk and the one that goes on behind it are written at the end): with everything in place, the
// instructions of a short launch came from memory for longer than its data.
template <typename DyT, typename GradT, bool ACCUMULATE> __global__ __launch_bounds__(THREADS) void sum_kernel(GradArgs A) {
    if (blockIdx.x >= A.sum_blocks) {
        if (blockIdx.y == 0) clear_absent_rows<GradT>(A, static_cast<int64_t>(blockIdx.x - A.sum_blocks) * A.clear_rows);
        return;
    }
    const uint32_t at = blockIdx.x * THREADS + threadIdx.x;
    const uint32_t in_page = at / A.vecs, v = at - in_page * A.vecs;
    const uint32_t c = blockIdx.y * A.page + in_page;
    if (in_page >= A.page || c >= A.chunks) return;
    const int64_t col = static_cast<int64_t>(v) * VEC;
    const int n = static_cast<int>(min(A.dim - col, static_cast<int64_t>(VEC)));
    const int64_t first = static_cast<int64_t>(c) * A.chunk, end = min(first + A.chunk, A.tokens), further = min(end + A.chunk, A.tokens);
    const DyT* const dy = static_cast<const DyT*>(A.dy) + col;
    const int32_t none = static_cast<int32_t>(A.n_rows);
    constexpr int AHEAD = sizeof(DyT) == 4 ? 8 : 16;             // 64 registers of dy on their way
    u32x4 order[AHEAD / 4];                                      // the next places, asked for early: whole fours, padded to 256 bytes
    i32x4 rows[AHEAD / 4];
    auto look = [&](int64_t p) {
#pragma unroll
        for (int j = 0; j < AHEAD / 4; ++j) {
            order[j] = *reinterpret_cast<const u32x4*>(A.order + p + 4 * j);
            rows[j] = *reinterpret_cast<const i32x4*>(A.row + p + 4 * j);
        }
    };
    look(first);
    const int32_t front = A.row[first], back = A.row[end - 1];
    const int32_t before = first > 0 ? A.row[first - 1] : none, long_before = first > A.chunk ? A.row[first - A.chunk - 1] : none;
    const int32_t after = end < A.tokens ? A.row[end] : none, long_after = further < A.tokens ? A.row[further] : none;
    if (front == none) return;
    const bool goes_on = back != none && after == back;         // the last stretch, behind the chunk
    const bool came = before == front;                          // the first stretch, from before the chunk
    const bool through = came && goes_on && front == back;
    const bool skips = came && !through && long_before != front;            // the chunk before has summed it
    const bool extends = goes_on && !through && long_after != back;
    const int64_t stop = extends ? further : end;
    float sum[VEC] = {}, head[VEC] = {};
    int32_t current = none;
    for (int64_t p0 = first; p0 < stop; p0 += AHEAD) {
        Raw8<DyT> x[AHEAD];
        int32_t r[AHEAD];
        uint32_t token[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int64_t p = p0 + j;
            const int32_t row = rows[j / 4][j % 4];
            const bool counts = p < end ? !(skips && row == front) : p < stop && row == back;
            r[j] = counts ? row : none;
            token[j] = r[j] != none ? order[j / 4][j % 4] : 0;
        }
        if (n == VEC) {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) x[j] = load8(dy + static_cast<int64_t>(token[j]) * A.dy_stride);
        } else {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) x[j] = load8(dy + static_cast<int64_t>(token[j]) * A.dy_stride, n);
        }
        if (p0 + AHEAD < stop) look(p0 + AHEAD);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (r[j] != current) {                              // a stretch has ended
                if (came && current == front)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) head[i] = sum[i];
                else if (current != none)
                    write_row<GradT, ACCUMULATE>(A, current, col, n, sum);
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
                current = r[j];
            }
            if (r[j] != none)
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[i] += get(x[j], i);
        }
    }
    // The last stretch is still in sum if it reaches the end; one that ends in tokens without a row has been written.
    const bool front_last = came && current == front;
    if (came && !skips) write_partial(A, 2 * c, col, front_last ? sum : head);
    if (current != none && !front_last) {
        if (goes_on && !extends && current == back) write_partial(A, 2 * c + 1, col, sum);
        else write_row<GradT, ACCUMULATE>(A, current, col, n, sum);
    }
    if (v == 0 && goes_on && !through && !extends)              // begins here: to be joined
        A.joins[1 + atomicAdd(reinterpret_cast<uint32_t*>(A.joins), 1u)] = u32x2{c, static_cast<uint32_t>(back)};
}

// Rows whose tokens reach over several chunks, one at a time by a workgroup.  A lane has four columns, join_width lanes a row's
// stretch; slot i of the workgroup's adds the stretches i, i + slots, ..., then the slots' sums are added in order.  All of it
// is waiting for memory, so what can be asked for at once is: the first row of the list before its length is known, and the
// beginnings of four chunks a lane to find the row's last one.
template <typename GradT> __global__ __launch_bounds__(THREADS) void join_kernel(GradArgs A) {
    __shared__ f32x4 sums[THREADS];
    const uint32_t lane = threadIdx.x % 64;
    const uint32_t slot = threadIdx.x / A.join_width, slots = THREADS / A.join_width, place = threadIdx.x % A.join_width;
    const int64_t col = (static_cast<int64_t>(blockIdx.y) * A.join_width + place) * 4;
    const uint32_t rows_to_join = A.joins[0].x;
    u32x2 join = A.joins[1 + blockIdx.x];                                        // within the list, whatever its length
    for (uint32_t no = blockIdx.x; no < rows_to_join;) {
        const uint32_t c = join.x;
        const int32_t r = static_cast<int32_t>(join.y);
        uint32_t pieces = 1;                                                     // chunks behind c that begin with the row have one, too
        for (;;) {
            uint64_t begins[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t q = c + pieces + j * 64 + lane;
                begins[j] = __ballot(q < A.chunks && A.row[static_cast<int64_t>(min(q, A.chunks - 1)) * A.chunk] == r);
            }
            uint32_t more = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (more == j * 64u) more += ~begins[j] != 0 ? __builtin_ctzll(~begins[j]) : 64;
            pieces += more;
            if (more < 256) break;
        }
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        if (col < A.dim) {
            if (slot == 0) sum = *reinterpret_cast<const f32x4*>(A.partial + (2 * static_cast<int64_t>(c) + 1) * A.dim_padded + col);
#pragma unroll 16
            for (uint32_t i = slot == 0 ? slots : slot; i < pieces; i += slots)
                sum += *reinterpret_cast<const f32x4*>(A.partial + 2 * static_cast<int64_t>(c + i) * A.dim_padded + col);
        }
        no += gridDim.x;
        if (no < rows_to_join) join = A.joins[1 + no];
        sums[threadIdx.x] = sum;
        __syncthreads();
        if (slot == 0 && col < A.dim) {
            for (uint32_t w = 1; w < min(slots, pieces); ++w) sum += sums[w * A.join_width + place];
            GradT* const g = static_cast<GradT*>(A.grad) + r * A.grad_stride + col;
            const int n = static_cast<int>(min(A.dim - col, int64_t(4)));
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = sum[i] * A.scale;
                if (A.accumulate && i < n) x[i] += static_cast<float>(g[i]);
            }
            store_some(g, x, n);
        }
        __syncthreads();
    }
}

// ---- few tokens: no order, every row looks for its own ----

constexpr int64_t FEW_TOKENS_MOST = 256;
constexpr int FEW_ROWS = 4;              // for which there is a form of their own, below
constexpr int DIRECT_WAVES = THREADS / 64;

// Lanes hold the ids, LANE_IDS each; a row's tokens are the bits of as many comparisons.  A wavefront takes one row after the other,
// and 512 columns: zeros where there are no tokens, else their sum in order, AHEAD of them on their way at a time.  Rows of more than LONG_ROW
// tokens are left for the end, where all wavefronts take a part of each.  Bound by writing the table (30522 rows of 1024
// bfloat16: 12 us, 5.2 TB/s), or by a launch (512 rows: 3 us).
//
// The rule.  256 tokens spread over 100 rows of 64 columns 4 us, of frequencies like words' 7, all in one row 8, and 15, 17 and 12 with an
// order; 30522 rows of 1024 columns 12, 18, 15 and 19, 19, 20.  With 512 tokens (and sixteen comparisons) 30522 rows take 17, 26,
// 21 and 20, 20, 21.  A row costs a wavefront its comparisons however short it is: 65536 rows of 64 columns 7 and 14 us, 200
// thousand 16 and 16, of 512 columns 28 and 36.  Up to FEW_ROWS rows a sum for each is better: 2 rows of 1024 columns 6, here 9.
constexpr int64_t DIRECT_ROWS = 131072, DIRECT_DIM = 256;
bool is_direct(int64_t tokens, int64_t n_rows, int64_t dim) {
    return tokens <= FEW_TOKENS_MOST && n_rows > FEW_ROWS && (n_rows <= DIRECT_ROWS || dim >= DIRECT_DIM);
}

template <typename DyT, typename GradT> __global__ __launch_bounds__(THREADS) void direct_kernel(GradArgs A) {
    constexpr int LANE_IDS = FEW_TOKENS_MOST / 64;
    constexpr int AHEAD = sizeof(DyT) == 4 ? 8 : 16;
    constexpr int LONG_ROW = 32, LONG_ROWS = LANE_IDS * 64 / LONG_ROW;
    __shared__ int32_t long_row[DIRECT_WAVES][LONG_ROWS];
    __shared__ uint32_t long_rows[DIRECT_WAVES];
    __shared__ f32x4 part[DIRECT_WAVES][2][64];
    static_assert(LANE_IDS == DIRECT_WAVES, "of a long row, a wavefront takes the mask of its number");
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t n = static_cast<uint32_t>(A.tokens);
    int32_t row[LANE_IDS];
#pragma unroll
    for (int k = 0; k < LANE_IDS; ++k) {
        const uint32_t t = k * 64 + lane;
        row[k] = row_of(A, id_at(A.ids, A.id_type, min(t, n - 1)));
        if (t >= n) row[k] = static_cast<int32_t>(A.n_rows);
    }
    const int64_t col = (static_cast<int64_t>(blockIdx.y) * 64 + lane) * VEC;
    const int width = static_cast<int>(max(int64_t(0), min(A.dim - col, static_cast<int64_t>(VEC))));
    // Lanes behind the last column read what the slice's first one reads: with nothing to read they would take another branch.
    const int64_t in_col = width > 0 ? col : static_cast<int64_t>(blockIdx.y) * 64 * VEC;
    const int in_width = static_cast<int>(min(A.dim - in_col, static_cast<int64_t>(VEC)));
    const DyT* const dy = static_cast<const DyT*>(A.dy) + in_col;
    // Adds the tokens of the k-th 64 that are set in `rest`.
    auto add = [&](float (&sum)[VEC], uint32_t k, uint64_t rest) {
        auto take = [&](auto many) {                             // the next ones: the lowest bits that are left
            constexpr int N = decltype(many)::value;
            Raw8<DyT> x[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                x[j] = load8(dy + static_cast<int64_t>(k * 64 + __builtin_ctzll(rest)) * A.dy_stride, in_width);
                rest &= rest - 1;
            }
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[i] += get(x[j], i);
        };
        uint32_t left = __popcll(rest);
        for (; left >= AHEAD; left -= AHEAD) take(std::integral_constant<int, AHEAD>());
        for (; left >= 4; left -= 4) take(std::integral_constant<int, 4>());
        for (; left > 0; --left) take(std::integral_constant<int, 1>());
    };
    // Adds the tokens of those masks that are set in `which`.  (Lane k holds the k-th mask: in a loop there is one copy of
    // the code above.)
    auto add_all = [&](float (&sum)[VEC], const uint64_t (&mine)[LANE_IDS], uint64_t which) {
        uint32_t low = 0, high = 0;
#pragma unroll
        for (int k = 0; k < LANE_IDS; ++k) {
            low = lane == k ? static_cast<uint32_t>(mine[k]) : low;
            high = lane == k ? static_cast<uint32_t>(mine[k] >> 32) : high;
        }
        for (uint64_t words = __ballot((low | high) != 0) & which; words != 0; words &= words - 1) {
            const uint32_t k = __builtin_ctzll(words);
            add(sum, k, static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(high, k))) << 32 |
                            static_cast<uint32_t>(__builtin_amdgcn_readlane(low, k)));
        }
    };
    auto write = [&](int64_t r, const float (&sum)[VEC]) {
        if (width <= 0) return;
        if (A.accumulate) write_row<GradT, true>(A, static_cast<int32_t>(r), col, width, sum);
        else write_row<GradT, false>(A, static_cast<int32_t>(r), col, width, sum);
    };
    const int64_t first = static_cast<int64_t>(blockIdx.x) * A.clear_rows, end = min(first + A.clear_rows, A.n_rows);
    uint32_t found = 0;                                          // long rows
    for (int64_t r = first + wave; r < end; r += DIRECT_WAVES) {
        uint64_t mine[LANE_IDS], any = 0;
#pragma unroll
        for (int k = 0; k < LANE_IDS; ++k) any |= mine[k] = __ballot(row[k] == static_cast<int32_t>(r));
        float sum[VEC] = {};
        if (any == 0) {
            if (!A.accumulate && width > 0) store8(static_cast<GradT*>(A.grad) + r * A.grad_stride + col, sum, width);
            continue;
        }
        uint32_t count = 0;
#pragma unroll
        for (int k = 0; k < LANE_IDS; ++k) count += __popcll(mine[k]);
        if (count > LONG_ROW) {
            if (lane == 0) long_row[wave][found] = static_cast<int32_t>(r);
            ++found;
            continue;
        }
        add_all(sum, mine, ~uint64_t(0));
        write(r, sum);
    }
    if (lane == 0) long_rows[wave] = found;
    __syncthreads();
    for (int w = 0; w < DIRECT_WAVES; ++w)
        for (uint32_t i = 0; i < long_rows[w]; ++i) {            // by all wavefronts, 64 of the ids each
            const int32_t r = long_row[w][i];
            float sum[VEC] = {};
            uint64_t mine[LANE_IDS];
#pragma unroll
            for (int k = 0; k < LANE_IDS; ++k) mine[k] = __ballot(row[k] == r);
            add_all(sum, mine, uint64_t(1) << wave);
            part[wave][0][lane] = f32x4{sum[0], sum[1], sum[2], sum[3]};
            part[wave][1][lane] = f32x4{sum[4], sum[5], sum[6], sum[7]};
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int other = 1; other < DIRECT_WAVES; ++other)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum[e] += part[other][e / 4][lane][e % 4];
                write(r, sum);
            }
            __syncthreads();
        }
}

// ---- few rows: no order, a sum for each row in every lane ----

constexpr int FEW_LANES = 16, FEW_TOKENS = THREADS / FEW_LANES, FEW_AHEAD = 8;       // 128 columns of 16 tokens at a time

// 128 columns of a chunk of tokens by a workgroup.  A token's vector is added to its row's sum and nothing to the others (a
// selection, no product: what a token without a row holds does not matter).  Two launches of 4.4 and 3.5 us for 4096 tokens of 1024
// bfloat16 columns, which are 8 MB: waits for memory and the launches themselves.
template <typename DyT, typename GradT, int ROWS> __global__ __launch_bounds__(THREADS) void few_rows_kernel(GradArgs A) {
    __shared__ float sums[FEW_TOKENS][FEW_LANES * VEC + 4];
    const uint32_t lane = threadIdx.x % FEW_LANES, place = threadIdx.x / FEW_LANES;
    const int64_t col = (static_cast<int64_t>(blockIdx.x) * FEW_LANES + lane) * VEC;
    const int n = static_cast<int>(max(int64_t(0), min(A.dim - col, static_cast<int64_t>(VEC))));
    const int64_t first = static_cast<int64_t>(blockIdx.y) * A.chunk, end = min(first + A.chunk, A.tokens);
    const DyT* const dy = static_cast<const DyT*>(A.dy) + col;
    float sum[ROWS][VEC] = {};
    for (int64_t t0 = first + place; t0 < end; t0 += FEW_TOKENS * FEW_AHEAD) {
        Raw8<DyT> x[FEW_AHEAD];
        int64_t id[FEW_AHEAD];
#pragma unroll
        for (int j = 0; j < FEW_AHEAD; ++j) {
            const int64_t t = min(t0 + FEW_TOKENS * j, end - 1);
            x[j] = load8(dy + t * A.dy_stride, n);
            id[j] = id_at(A.ids, A.id_type, t);
        }
#pragma unroll
        for (int j = 0; j < FEW_AHEAD; ++j) {
            if (t0 + FEW_TOKENS * j >= end || id[j] == A.padding_row) id[j] = -1;
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[r][i] += id[j] == r ? get(x[j], i) : 0.f;
        }
    }
    for (int r = 0; r < ROWS; ++r) {
        if (r >= A.n_rows) break;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < ROWS; ++q)
            if (q == r)
#pragma unroll
                for (int i = 0; i < VEC; ++i) sums[place][lane * VEC + i] = sum[q][i];
        __syncthreads();
        const int64_t c = static_cast<int64_t>(blockIdx.x) * FEW_LANES * VEC + threadIdx.x;
        if (threadIdx.x >= FEW_LANES * VEC || c >= A.dim) continue;
        float all = 0.f;
#pragma unroll
        for (int w = 0; w < FEW_TOKENS; ++w) all += sums[w][threadIdx.x];
        if (A.chunks > 1) {
            A.partial[(static_cast<int64_t>(blockIdx.y) * A.n_rows + r) * A.dim_padded + c] = all;
        } else {
            GradT* const g = static_cast<GradT*>(A.grad) + r * A.grad_stride + c;
            all *= A.scale;
            *g = rounded<GradT>(A.accumulate ? all + static_cast<float>(*g) : all);
        }
    }
}

// The chunks' sums of a row, in order: sixteen slots of every sixteenth chunk each, then the slots.
template <typename GradT> __global__ __launch_bounds__(THREADS) void few_join_kernel(GradArgs A) {
    constexpr int LANES = 16, SLOTS = THREADS / LANES;
    __shared__ f32x4 sums[SLOTS][LANES];
    const uint32_t lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int64_t col = (static_cast<int64_t>(blockIdx.x) * LANES + lane) * 4;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (col < A.dim)
#pragma unroll 8
        for (uint32_t c = slot; c < A.chunks; c += SLOTS)
            sum += *reinterpret_cast<const f32x4*>(A.partial + (static_cast<int64_t>(c) * A.n_rows + blockIdx.y) * A.dim_padded + col);
    sums[slot][lane] = sum;
    __syncthreads();
    if (slot != 0 || col >= A.dim) return;
    for (int w = 1; w < SLOTS; ++w) sum += sums[w][lane];
    GradT* const g = static_cast<GradT*>(A.grad) + blockIdx.y * A.grad_stride + col;
    const int n = static_cast<int>(min(A.dim - col, int64_t(4)));
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = sum[i] * A.scale;
        if (A.accumulate && i < n) x[i] += static_cast<float>(g[i]);
    }
    store_some(g, x, n);
}

// ---- host side ----

int passes_of(int64_t n_rows) {          // of eight bits, for the numbers 0 .. n_rows
    int passes = 1;
    while (passes < 4 && (static_cast<uint64_t>(n_rows) >> (8 * passes)) != 0) ++passes;
    return passes;
}

struct GradPlan {
    bool direct, few, ranked;          // the forms that need no order; how the others order
    uint32_t chunk, chunks, blocks, items;
    int64_t dim_padded;
    int64_t order, row, partial, joins, other_order, other_row, counts, bytes;     // places in the workspace
};

// What is in the workspace, and where: every part begins on 256 bytes.
GradPlan plan_of(int64_t tokens, int64_t n_rows, int64_t dim) {
    GradPlan p{};
    p.direct = tokens == 0 || is_direct(tokens, n_rows, dim);
    p.few = !p.direct && n_rows <= FEW_ROWS;
    p.ranked = tokens <= RANKED_TOKENS;
    if (p.direct) return p;                                  // no workspace
    // Chunks of 16 to 64 tokens: longer ones leave less to join, shorter ones more lanes that sum, of which a chip full is wanted.
    const int64_t lanes = tokens * ceil_div(std::max<int64_t>(dim, 1), VEC);
    p.chunk = lanes / 64 >= 131072 ? 64 : lanes / 32 >= 65536 ? 32 : 16;
    p.chunks = static_cast<uint32_t>(ceil_div(tokens, p.chunk));
    p.dim_padded = ceil_div(dim, VEC) * VEC;
    // radix sort: at most 256 workgroups, since each adds up the counts of all
    const int64_t items = std::max<int64_t>(1024, ceil_div(ceil_div(tokens, 256), THREADS) * THREADS);
    p.items = static_cast<uint32_t>(items);
    p.blocks = static_cast<uint32_t>(ceil_div(tokens, items));
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += ceil_div(bytes, 256) * 256;
        return here;
    };
    if (p.few) {
        // At least 128 tokens a chunk, all of them on their way at once, and no more than 2048 workgroups.
        const int64_t slices = ceil_div(std::max<int64_t>(dim, 1), FEW_LANES * VEC), most = std::max<int64_t>(2048 / slices, 1);
        p.chunk = static_cast<uint32_t>(std::max<int64_t>(ceil_div(ceil_div(tokens, most), FEW_TOKENS * FEW_AHEAD), 1) * (FEW_TOKENS * FEW_AHEAD));
        p.chunks = static_cast<uint32_t>(ceil_div(tokens, p.chunk));
        if (p.chunks > 1) p.partial = take(static_cast<int64_t>(p.chunks) * n_rows * p.dim_padded * 4);
        p.bytes = at;
        return p;
    }
    p.order = take(tokens * 4);
    p.row = take(tokens * 4);
    p.partial = take(2 * static_cast<int64_t>(p.chunks) * p.dim_padded * 4);
    p.joins = take((1 + static_cast<int64_t>(p.chunks)) * 8);
    if (!p.ranked) {
        p.other_order = take(tokens * 4);
        p.other_row = take(tokens * 4);
        p.counts = take(static_cast<int64_t>(p.blocks) * DIGITS * 4);
    }
    p.bytes = at;
    return p;
}

bool grad_sizes_ok(int64_t n_tokens, int64_t n_rows, int64_t dim) {
    return n_tokens >= 0 && n_tokens <= MOST_TOKENS && n_rows >= 0 && n_rows < 0x7fffffff && dim >= 0 && dim <= MOST_DIM;
}

}  // namespace

int ops::note(hipError_t e) {
    if (e == hipSuccess) return MGWFBP_OK;
    g_last_hip_error = static_cast<int>(e);
    return MGWFBP_EHIP;
}

extern "C" {

int mgwfbp_layers_last_hip_error(void) { return g_last_hip_error; }

int mgwfbp_embed(const mgwfbp_table* tables, int32_t n_tables, int32_t table_dtype, int64_t n_tokens, int64_t dim,
                 void* d_out, int64_t out_stride, int32_t out_dtype, void* hip_stream) {
    if (tables == nullptr || n_tables < 1 || n_tables > MGWFBP_MAX_TABLES) return MGWFBP_EINVAL;
    if (!is_dtype(table_dtype) || !is_dtype(out_dtype)) return MGWFBP_EINVAL;
    if (n_tokens < 0 || n_tokens > MOST_TOKENS || dim < 0 || dim > MOST_DIM) return MGWFBP_EINVAL;
    if (!is_matrix(n_tokens, dim, out_stride, dtype_bytes(out_dtype))) return MGWFBP_EINVAL;
    EmbedArgs a{};
    for (int32_t k = 0; k < n_tables; ++k) {
        const mgwfbp_table& t = tables[k];
        if (t.id_type != MGWFBP_I32 && t.id_type != MGWFBP_I64) return MGWFBP_EINVAL;
        if (!is_matrix(t.n_rows, dim, t.row_stride, dtype_bytes(table_dtype))) return MGWFBP_EINVAL;
        if (n_tokens > 0 && dim > 0) {
            if (t.d_ids == nullptr || !is_aligned(t.d_ids, t.id_type == MGWFBP_I64 ? 8 : 4)) return MGWFBP_EINVAL;
            if (t.n_rows > 0 && (t.d_rows == nullptr || !is_aligned(t.d_rows, dtype_bytes(table_dtype)))) return MGWFBP_EINVAL;
        }
        a.table[k] = {t.d_rows, t.d_ids, t.n_rows, t.row_stride, t.scale, t.id_type};
    }
    if (n_tokens == 0 || dim == 0) return MGWFBP_OK;
    if (d_out == nullptr || !is_aligned(d_out, dtype_bytes(out_dtype))) return MGWFBP_EINVAL;
    a.out = d_out;
    a.out_stride = out_stride;
    a.tokens = n_tokens;
    a.dim = dim;
    a.vecs = static_cast<uint32_t>(ceil_div(dim, VEC));
    // pages so long that their vectors number less than 2^31, and at most 65535 of them
    a.page = static_cast<uint32_t>(std::min<int64_t>(n_tokens, (int64_t(1) << 31) / a.vecs - 1));
    if (ceil_div(n_tokens, a.page) > 65535) return MGWFBP_EINVAL;
    const dim3 grid(static_cast<uint32_t>(ceil_div(static_cast<int64_t>(a.page) * a.vecs, THREADS)),
                    static_cast<uint32_t>(ceil_div(n_tokens, a.page)));
    return with_dtype(table_dtype, [&](auto* table_type) {
        return with_dtype(out_dtype, [&](auto* out_type) {
            typedef std::remove_pointer_t<decltype(table_type)> TabT;
            typedef std::remove_pointer_t<decltype(out_type)> OutT;
            void (*kernel)(EmbedArgs) = n_tables == 1 ? embed_kernel<TabT, OutT, 1> : n_tables == 2 ? embed_kernel<TabT, OutT, 2>
                                      : n_tables == 3 ? embed_kernel<TabT, OutT, 3> : embed_kernel<TabT, OutT, 4>;
            return launch(kernel, a, grid, dim3(THREADS), hip_stream);
        });
    });
}

int mgwfbp_embed_grad_workspace(int64_t n_tokens, int64_t n_rows, int64_t dim, uint64_t* bytes_out) {
    if (bytes_out == nullptr || !grad_sizes_ok(n_tokens, n_rows, dim)) return MGWFBP_EINVAL;
    *bytes_out = static_cast<uint64_t>(plan_of(n_tokens, n_rows, dim).bytes);
    return MGWFBP_OK;
}

int mgwfbp_embed_grad(const void* d_ids, int32_t id_type, int64_t n_tokens, const void* d_dy, int64_t dy_stride,
                      int32_t dy_dtype, float scale, int64_t padding_row, int32_t accumulate, void* d_grad, int64_t n_rows,
                      int64_t dim, int64_t grad_stride, int32_t grad_dtype, void* d_workspace, uint64_t workspace_bytes,
                      void* hip_stream) {
    if (!grad_sizes_ok(n_tokens, n_rows, dim) || !is_dtype(dy_dtype) || !is_dtype(grad_dtype)) return MGWFBP_EINVAL;
    if (id_type != MGWFBP_I32 && id_type != MGWFBP_I64) return MGWFBP_EINVAL;
    if (!is_matrix(n_tokens, dim, dy_stride, dtype_bytes(dy_dtype))) return MGWFBP_EINVAL;
    if (!is_matrix(n_rows, dim, grad_stride, dtype_bytes(grad_dtype))) return MGWFBP_EINVAL;
    if (n_rows == 0 || dim == 0) return MGWFBP_OK;
    if (d_grad == nullptr || !is_aligned(d_grad, dtype_bytes(grad_dtype))) return MGWFBP_EINVAL;
    const GradPlan p = plan_of(n_tokens, n_rows, dim);
    if (n_tokens > 0) {
        if (d_ids == nullptr || !is_aligned(d_ids, id_type == MGWFBP_I64 ? 8 : 4)) return MGWFBP_EINVAL;
        if (d_dy == nullptr || !is_aligned(d_dy, dtype_bytes(dy_dtype))) return MGWFBP_EINVAL;
        if (p.bytes > 0 && (d_workspace == nullptr || !is_aligned(d_workspace, 256) || workspace_bytes < static_cast<uint64_t>(p.bytes)))
            return MGWFBP_EINVAL;
    } else if (accumulate) {
        return MGWFBP_OK;
    }
    GradArgs a{};
    unsigned char* const ws = static_cast<unsigned char*>(d_workspace);
    a.ids = d_ids;
    a.id_type = id_type;
    a.dy = d_dy;
    a.dy_stride = dy_stride;
    a.grad = d_grad;
    a.grad_stride = n_rows == 1 ? dim : grad_stride;
    a.n_rows = n_rows;
    a.dim = dim;
    a.padding_row = padding_row;
    a.tokens = n_tokens;
    a.dim_padded = p.dim_padded;
    a.scale = scale;
    a.accumulate = accumulate != 0;
    a.chunk = p.chunk;
    a.chunks = p.chunks;
    a.items = p.items;
    a.vecs = static_cast<uint32_t>(ceil_div(dim, VEC));
    a.page = static_cast<uint32_t>(std::min<int64_t>(std::max<uint32_t>(p.chunks, 1), (int64_t(1) << 30) / a.vecs));
    if (n_tokens > 0) {
        a.order = reinterpret_cast<uint32_t*>(ws + p.order);
        a.row = reinterpret_cast<int32_t*>(ws + p.row);
        a.partial = reinterpret_cast<float*>(ws + p.partial);
        a.joins = reinterpret_cast<u32x2*>(ws + p.joins);
    }
    if (p.direct && n_tokens > 0) {
        // Rows of a workgroup: about 32 KiB of the gradient, but no fewer than its wavefronts, and so few that the chip is full.
        const int64_t slices = ceil_div(dim, 64 * VEC), share = std::max<int64_t>(DIRECT_WAVES, 32768 / (std::min<int64_t>(dim, 64 * VEC) * dtype_bytes(grad_dtype)));
        a.clear_rows = static_cast<uint32_t>(std::max<int64_t>(DIRECT_WAVES, std::min(share, ceil_div(n_rows * slices, 1024))));
        const dim3 direct_grid(static_cast<uint32_t>(ceil_div(n_rows, a.clear_rows)), static_cast<uint32_t>(slices));
        return with_dtype(dy_dtype, [&](auto* dy_type) {
            return with_dtype(grad_dtype, [&](auto* grad_type) {
                return launch(direct_kernel<std::remove_pointer_t<decltype(dy_type)>, std::remove_pointer_t<decltype(grad_type)>>, a, direct_grid, dim3(THREADS),
                              hip_stream);
            });
        });
    }
    if (p.few) {
        const dim3 few_grid(static_cast<uint32_t>(ceil_div(dim, FEW_LANES * VEC)), p.chunks);
        const int status = with_dtype(dy_dtype, [&](auto* dy_type) {
            return with_dtype(grad_dtype, [&](auto* grad_type) {
                typedef std::remove_pointer_t<decltype(dy_type)> DyT;
                typedef std::remove_pointer_t<decltype(grad_type)> GradT;
                return launch(n_rows <= 2 ? few_rows_kernel<DyT, GradT, 2> : few_rows_kernel<DyT, GradT, FEW_ROWS>, a, few_grid, dim3(THREADS), hip_stream);
            });
        });
        if (status != MGWFBP_OK || p.chunks < 2) return status;
        const dim3 join_grid(static_cast<uint32_t>(ceil_div(dim, 64)), static_cast<uint32_t>(n_rows));
        return with_dtype(grad_dtype, [&](auto* grad_type) {
            return launch(few_join_kernel<std::remove_pointer_t<decltype(grad_type)>>, a, join_grid, dim3(THREADS), hip_stream);
        });
    }
    // A workgroup clears about 32 KiB, at most one row a thread.
    a.clear_rows = static_cast<uint32_t>(std::min<int64_t>(THREADS, std::max<int64_t>(1, 32768 / (dim * dtype_bytes(grad_dtype)))));
    int rc = MGWFBP_OK;
    if (n_tokens > 0 && p.ranked) {
        void (*narrow)(GradArgs) = id_type == MGWFBP_I64 ? rank_kernel<uint32_t, int64_t> : rank_kernel<uint32_t, int32_t>;
        void (*wide)(GradArgs) = id_type == MGWFBP_I64 ? rank_kernel<uint64_t, int64_t> : rank_kernel<uint64_t, int32_t>;
        rc = launch(n_rows <= NARROW_ROWS ? narrow : wide, a, dim3(static_cast<uint32_t>(ceil_div(n_tokens, RANK_EACH))), dim3(THREADS), hip_stream);
        if (rc != MGWFBP_OK) return rc;
    } else if (n_tokens > 0) {
        uint32_t* const order[2] = {a.order, reinterpret_cast<uint32_t*>(ws + p.other_order)};
        int32_t* const row[2] = {a.row, reinterpret_cast<int32_t*>(ws + p.other_row)};
        a.counts = reinterpret_cast<uint32_t*>(ws + p.counts);
        const int passes = passes_of(n_rows);
        for (int pass = 0; pass < passes; ++pass) {             // the last one ends in order and row
            const int to = (passes - 1 - pass) % 2;
            a.order = order[to];
            a.row = row[to];
            a.other_order = order[1 - to];
            a.other_row = row[1 - to];
            a.shift = 8 * pass;
            a.from_ids = pass == 0;
            rc = launch(digit_kernel, a, dim3(p.blocks), dim3(THREADS), hip_stream);
            if (rc == MGWFBP_OK) rc = launch(move_kernel, a, dim3(p.blocks), dim3(THREADS), hip_stream);
            if (rc != MGWFBP_OK) return rc;
        }
    }
    const uint32_t clearing = accumulate ? 0 : static_cast<uint32_t>(ceil_div(n_rows, a.clear_rows));
    a.sum_blocks = n_tokens > 0 ? static_cast<uint32_t>(ceil_div(static_cast<int64_t>(a.page) * a.vecs, THREADS)) : 0;
    const dim3 grid(a.sum_blocks + clearing, std::max<uint32_t>(static_cast<uint32_t>(ceil_div(p.chunks, a.page)), 1));
    rc = with_dtype(dy_dtype, [&](auto* dy_type) {
        return with_dtype(grad_dtype, [&](auto* grad_type) {
            typedef std::remove_pointer_t<decltype(dy_type)> DyT;
            typedef std::remove_pointer_t<decltype(grad_type)> GradT;
            return launch(accumulate ? sum_kernel<DyT, GradT, true> : sum_kernel<DyT, GradT, false>, a, grid, dim3(THREADS), hip_stream);
        });
    });
    if (rc != MGWFBP_OK || p.chunks < 2) return rc;
    // 64 columns a workgroup: a compute unit takes in about 25 GB/s, so a long row wants many of them.
    a.join_width = 1;
    while (a.join_width < 16 && a.join_width * 4 < dim) a.join_width *= 2;
    const int64_t join_slices = ceil_div(dim, 4 * static_cast<int64_t>(a.join_width));
    const dim3 join_grid(std::min<uint32_t>(p.chunks - 1, static_cast<uint32_t>(std::max<int64_t>(1024 / join_slices, 1))), static_cast<uint32_t>(join_slices));
    return with_dtype(grad_dtype, [&](auto* grad_type) {
        return launch(join_kernel<std::remove_pointer_t<decltype(grad_type)>>, a, join_grid, dim3(THREADS), hip_stream);
    });
}

}  // extern "C"
