// Weight and bias gradient of a linear layer from its output's gradient and its input's 8-bit checkpoint.
//
//   mgwfbp_act_linear_grad   dw[o,c] = sum over groups g of scale[g,c] * (sum over the group's tokens of dy[t,o] * q[t,c])
//                            db[o] = sum over tokens of dy[t,o]
//
// The inner sums run on the matrix cores.  q is a whole number of at most 7 bits and a sign, exact in bfloat16 and
// binary16, so the products are exact and a group's sum has the roundings of a binary32 sum alone; the scale is applied to
// the sum of 128 tokens, in binary32.  A binary32 dy is cut into three bfloat16 parts of 8 bits each, which together are dy,
// and takes three products.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "act_layout.h"
#include "device_types.h"
#include "mgwfbp_layers.h"

namespace {

using namespace ops;

constexpr int GROUP = MGWFBP_ACT_GROUP;
constexpr int MAX_SPLITS = 64;
constexpr int BIAS_SHARES = 8;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct LinearArgs {
    const void* dy;
    const int8_t* q;
    const float* scale;
    void* dw;
    void* db;
    float* partial;                    // [splits][outputs][channels_padded], and the bias parts behind it
    float* bias_partial;               // [splits * bias_shares][outputs]
    int64_t dy_stride, ld, dw_stride, channels_padded;
    int64_t q_columns;                 // of q: own_columns(channels)
    int32_t tokens, channels, outputs;
    uint32_t tiles_c, tiles, splits, groups, groups_per_split, bias_shares, bias_blocks;
    int32_t accumulate;
};

// What the matrix cores multiply for a type of dy.
template <typename T> struct Mma {
    typedef __bf16 elem;
    typedef bf16x8 frag;
    static __device__ __forceinline__ f32x16 mul(frag a, frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<_Float16> {
    typedef _Float16 elem;
    typedef f16x8 frag;
    static __device__ __forceinline__ f32x16 mul(frag a, frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// LDS: tiles of STEP rows (tokens) by COLS columns of 2 bytes.  A fragment of the matrix instruction has eight tokens of one
// column in a lane, so it is read transposed (ds_read_b64_tr_b16: sixteen lanes read four rows of 16 columns and get four
// tokens of a column each).  Rows begin on the same bank, so the 32-byte pieces of a row are exchanged by a pattern of the
// row's two lowest bits: 0, 2, 5, 7 puts the pieces of four rows on different banks, and those of the next sixteen lanes, which
// read the neighbouring 16 columns, on others again (rows of 64 columns begin on two banks in turn: 0, 0, 2, 2).
template <int COLS> __device__ __forceinline__ uint32_t lds_at(uint32_t row, uint32_t col) {
    const uint32_t r = row & 3, pattern = COLS == 64 ? r & 2 : 2 * r + (r >> 1);
    return row * (COLS * 2) + ((col / 16 ^ pattern) * 32) + (col % 16) * 2;
}

template <int COLS, typename Frag> __device__ __forceinline__ Frag read_fragment(const char* tile, uint32_t at) {
    typedef __attribute__((address_space(3))) s16x4* lds;
    union { s16x4 half[2]; Frag whole; } u;
    u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(tile + at));
    u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(tile + at + 4 * (COLS * 2)));
    return u.whole;
}

// The parts of dy that are multiplied, highest first: dy itself where it has 16 bits.
template <typename T> struct Parts { static constexpr int n = 1; };
template <> struct Parts<float> { static constexpr int n = 3; };

template <typename T> __device__ __forceinline__ void split(const Raw8<T>& x, typename Mma<T>::frag (&part)[Parts<T>::n]) {
    if constexpr (sizeof(T) == 2) {
        part[0] = x.v;
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            float rest = get(x, i);
            const bool infinite = (__builtin_bit_cast(uint32_t, rest) & 0x7fffffffu) == 0x7f800000u;
#pragma unroll
            for (int p = 0; p < 3; ++p) {                     // the upper 16 bits, cut: what is left is exact
                const float head = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, rest) & 0xffff0000u);
                part[p][i] = static_cast<__bf16>(head);
                rest = infinite ? 0.f : rest - head;
            }
        }
    }
}

// A workgroup's tile of dw and how it is taken: WAVES_O x WAVES_C wavefronts of FRAGS 32 outputs by 64 channels each, STEP tokens
// at a time through one of BUFFERS buffers in LDS.
template <typename DyT, int FRAGS_, int WAVES_O_, int WAVES_C_, int STEP_, int BUFFERS_> struct Shape {
    static constexpr int FRAGS = FRAGS_, WAVES_O = WAVES_O_, WAVES_C = WAVES_C_, STEP = STEP_, BUFFERS = BUFFERS_;
    static constexpr int AHEAD = BUFFERS - 1;                                // steps between LDS and the matrix cores
    static constexpr int THREADS = WAVES_O * WAVES_C * 64;
    static constexpr int TILE_O = WAVES_O * FRAGS * 32, TILE_C = WAVES_C * 64;
    static constexpr int PARTS = Parts<DyT>::n;
    static constexpr int DY_BYTES = STEP * TILE_O * 2, X_BYTES = STEP * TILE_C * 2;
    static constexpr int BUFFER = PARTS * DY_BYTES + X_BYTES;
    static constexpr int DY_VECS = STEP * TILE_O / VEC / THREADS;            // vectors that a thread brings
    static constexpr int DY_ROWS = THREADS / (TILE_O / VEC);                 // rows that all threads bring at once
    static constexpr int XW = STEP * TILE_C / 16 >= THREADS ? 16 : 8;         // channels of q that a thread brings at once
    static constexpr int X_VECS = STEP * TILE_C / XW / THREADS;
    static constexpr int X_ROWS = THREADS / (TILE_C / XW);
    typedef uint32_t X __attribute__((ext_vector_type(XW / 4)));
    static constexpr int STEPS = GROUP / STEP;
    static constexpr int LDS = BUFFERS * BUFFER > TILE_O * TILE_C * 4 ? BUFFERS * BUFFER : TILE_O * TILE_C * 4;     // buffers, then the tile
};

template <typename DyT, typename S> struct Staged { Raw8<DyT> dy[S::DY_VECS]; typename S::X q[S::X_VECS]; };

// The pieces of a step on the way to LDS: a vector of dy, or of q.
template <typename DyT, typename S> __device__ __forceinline__ void put_dy(const Staged<DyT, S>& from, char* buffer, int j, uint32_t row, uint32_t col) {
    typename Mma<DyT>::frag part[S::PARTS];
    split<DyT>(from.dy[j], part);
#pragma unroll
    for (int p = 0; p < S::PARTS; ++p)
        *reinterpret_cast<typename Mma<DyT>::frag*>(buffer + p * S::DY_BYTES + lds_at<S::TILE_O>(row + S::DY_ROWS * j, col)) = part[p];
}
template <typename DyT, typename S> __device__ __forceinline__ void put_q(const Staged<DyT, S>& from, char* buffer, int j, uint32_t row, uint32_t col) {
#pragma unroll
    for (int h = 0; h < S::XW / VEC; ++h) {
        typename Mma<DyT>::frag x;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            x[i] = static_cast<typename Mma<DyT>::elem>(static_cast<float>(static_cast<int32_t>(from.q[j][2 * h + i / 4]) << (24 - 8 * (i % 4)) >> 24));
        *reinterpret_cast<typename Mma<DyT>::frag*>(buffer + S::PARTS * S::DY_BYTES + lds_at<S::TILE_C>(row + S::X_ROWS * j, col + h * VEC)) = x;
    }
}
template <typename DyT, typename S>
__device__ __forceinline__ void put_step(const Staged<DyT, S>& from, char* buffer, uint32_t dy_row, uint32_t dy_col, uint32_t q_row, uint32_t q_col) {
#pragma unroll
    for (int j = 0; j < S::DY_VECS; ++j) put_dy<DyT, S>(from, buffer, j, dy_row, dy_col);
#pragma unroll
    for (int j = 0; j < S::X_VECS; ++j) put_q<DyT, S>(from, buffer, j, q_row, q_col);
}

// The threads' sums of a tile's outputs, added in the order of their rows: to db, or as a part of the bias.
template <typename GradT, typename S>
__device__ __forceinline__ void write_bias(const LinearArgs& A, float* sums, const float (&bias)[VEC], int32_t o0, uint32_t row, uint32_t col, void* db,
                                           uint32_t part) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < VEC; ++i) sums[row * S::TILE_O + col + i] = bias[i];
    __syncthreads();
    const int32_t o = o0 + threadIdx.x;
    if (threadIdx.x >= S::TILE_O || o >= A.outputs) return;
    float all = 0.f;
    for (int w = 0; w < S::DY_ROWS; ++w) all += sums[w * S::TILE_O + threadIdx.x];
    if (db == nullptr) {
        A.bias_partial[static_cast<int64_t>(part) * A.outputs + o] = all;
    } else {
        GradT* const b = static_cast<GradT*>(db) + o;
        *b = rounded<GradT>(all + (A.accumulate ? static_cast<float>(*b) : 0.f));
    }
}

// A workgroup's tile to memory: `rows` rows of `cols` elements, `stride` apart, are there.  It goes through LDS, so that it is
// written in pieces of 16 bytes a lane.  Element e of a lane is in row 8 (e / 4) + 4 (lane / 32) + e % 4 and column lane % 32;
// the halves of a wavefront would meet on the same banks, so rows with bit 2 have neighbouring pieces of 32 columns exchanged.
template <typename S, bool STREAM, typename T>
__device__ __forceinline__ void write_tile(float* tile, const f32x16 (&value)[S::FRAGS][2], uint32_t wave_o, uint32_t wave_c, uint32_t lane, T* out,
                                           int64_t stride, int32_t rows, int32_t cols, bool accumulate) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::FRAGS; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t row = wave_o + i * 32 + e / 4 * 8 + lane / 32 * 4 + e % 4, col = wave_c + j * 32 + lane % 32;
                tile[row * S::TILE_C + (col ^ (row & 4) * 8)] = value[i][j][e];
            }
    __syncthreads();
    constexpr int W = 16 / sizeof(T), ROW_VECS = S::TILE_C / W;
    const uint32_t col = threadIdx.x % ROW_VECS * W;
    const int n = cols - static_cast<int32_t>(col);
    if (n <= 0) return;
    T* w = out + threadIdx.x / ROW_VECS * stride + col;
#pragma unroll 4
    for (int32_t row = threadIdx.x / ROW_VECS; row < min(rows, S::TILE_O); row += S::THREADS / ROW_VECS) {
        float x[W];
#pragma unroll
        for (int i = 0; i < W; i += 4) {
            const f32x4 four = *reinterpret_cast<const f32x4*>(tile + row * S::TILE_C + ((col + i) ^ (row & 4) * 8));
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i + e] = four[e];
        }
        if (accumulate)
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (i < n) x[i] += static_cast<float>(w[i]);
        store_some<STREAM>(w, x, n);
        w += S::THREADS / ROW_VECS * stride;
    }
}

// Tokens move from memory to registers, from there (binary32 cut into its parts, q widened) to LDS, and from LDS to the
// matrix cores.  Two steps are on their way in registers and AHEAD in the other buffers while a step is multiplied; one
// barrier a step.  With three buffers a step's first fragments are read before the barrier that ends the step before, so that
// the matrix cores go on right behind it.  RAGGED: the outputs are no multiple of eight, and the vector that holds the last ones is read element
// by element (or there are no channels).  Other vectors behind the last output or channel are read from the last ones that exist: what they make
// belongs to no element of dw.
//
// 1024 channels, 4096 outputs, 32775 binary16 tokens: 334 us with the join, 820 TFLOP/s; 4096 bfloat16 tokens 51 us, 43 of them
// here and 7 for the join.  Nothing is busy all the time: by the counters of the long one the matrix cores are for 39 % of a compute unit's
// cycles and LDS for as many; a wavefront spends 30 % of its life waiting for memory, LDS or a barrier and
// 40 % for its turn to issue.  The clock is 2.0 GHz, held down by power: with zeros for every element the same call takes three
// quarters of the time.  Three buffers of 64 tokens, and writes between the products, come from there; a higher priority of some wavefronts,
// loads between the products, and tiles in panels for each die are level or worse, and the scales moved between the next
// group's products do not fit into the registers.
template <typename DyT, typename GradT, typename S, bool RAGGED>
__global__ __launch_bounds__(S::THREADS, 2) void linear_kernel(LinearArgs A) {
    typedef typename Mma<DyT>::frag Frag;
    __shared__ __align__(256) char lds[S::LDS];

    // Consecutive workgroups go to the eight dies in turn; each die gets consecutive tiles, so that the tiles that share dy or q
    // share its L2.
    const uint32_t per_die = gridDim.x / 8;
    const uint32_t id = blockIdx.x < per_die * 8 ? blockIdx.x % 8 * per_die + blockIdx.x / 8 : blockIdx.x;
    const uint32_t split_no = id / A.tiles, tile = id - split_no * A.tiles;
    const uint32_t tile_o = tile / A.tiles_c, tile_c = tile - tile_o * A.tiles_c;
    const int32_t o0 = tile_o * S::TILE_O, c0 = tile_c * S::TILE_C;
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t wave_o = wave / S::WAVES_C * (S::FRAGS * 32), wave_c = wave % S::WAVES_C * 64;
    const int32_t t_first = split_no * A.groups_per_split * GROUP;
    const int32_t t_end = min(A.tokens, static_cast<int32_t>((split_no + 1) * A.groups_per_split * GROUP));

    const uint32_t dy_col = threadIdx.x % (S::TILE_O / VEC) * VEC, dy_row = threadIdx.x / (S::TILE_O / VEC);
    const uint32_t q_col = threadIdx.x % (S::TILE_C / S::XW) * S::XW, q_row = threadIdx.x / (S::TILE_C / S::XW);
    const int32_t o_in = o0 + static_cast<int32_t>(dy_col);
    const int dy_n = RAGGED ? max(0, min(A.outputs - o_in, VEC)) : VEC;
    const DyT* const dy_at = static_cast<const DyT*>(A.dy) + (RAGGED ? o_in : min(o_in, A.outputs - VEC));
    const int8_t* const q_at = A.q + piece_at(c0 + q_col, A.q_columns, S::XW);

    const DyT* dy_next = dy_at + (t_first + static_cast<int64_t>(dy_row)) * A.dy_stride;      // the rows that are fetched next
    const int8_t* q_next = q_at + (t_first + static_cast<int64_t>(q_row)) * A.ld;
    int32_t t_next = t_first;

    // The next STEP rows; rows behind the last token are zeros.
    auto fetch = [&](Staged<DyT, S>& to, auto steady) {
        if (decltype(steady)::value || t_next + S::STEP <= A.tokens) {
#pragma unroll
            for (int j = 0; j < S::DY_VECS; ++j) to.dy[j] = load8(dy_next + j * (S::DY_ROWS * A.dy_stride), dy_n);
#pragma unroll
            for (int j = 0; j < S::X_VECS; ++j)
                if (!RAGGED || A.ld > 0) to.q[j] = *reinterpret_cast<const typename S::X*>(q_next + j * (S::X_ROWS * A.ld));
        } else {
            const int32_t dy_rows = A.tokens - t_next - static_cast<int32_t>(dy_row), q_rows = A.tokens - t_next - static_cast<int32_t>(q_row);
#pragma unroll
            for (int j = 0; j < S::DY_VECS; ++j) to.dy[j] = load8(dy_next + j * (S::DY_ROWS * A.dy_stride), S::DY_ROWS * j < dy_rows ? dy_n : 0);
#pragma unroll
            for (int j = 0; j < S::X_VECS; ++j) {
                to.q[j] = typename S::X(0);
                if ((!RAGGED || A.ld > 0) && S::X_ROWS * j < q_rows) to.q[j] = *reinterpret_cast<const typename S::X*>(q_next + j * (S::X_ROWS * A.ld));
            }
        }
        t_next += S::STEP;
        dy_next += S::STEP * A.dy_stride;
        q_next += S::STEP * A.ld;
    };
    constexpr int TURNS = S::STEP / 16;
    auto put_some = [&](const Staged<DyT, S>& from, char* buffer, int turn) {          // a step in TURNS parts
#pragma unroll
        for (int j = 0; j < S::DY_VECS; ++j)
            if (j * TURNS / S::DY_VECS == turn) put_dy<DyT, S>(from, buffer, j, dy_row, dy_col);
#pragma unroll
        for (int j = 0; j < S::X_VECS; ++j)
            if (j * TURNS / S::X_VECS == turn) put_q<DyT, S>(from, buffer, j, q_row, q_col);
    };
    float bias[VEC] = {};
    const uint32_t share = A.db != nullptr && tile_c < A.bias_shares ? tile_c : ~0u;       // the steps whose bias this workgroup adds
    uint32_t step = 0;
    auto add_bias = [&](const Staged<DyT, S>& from) {
        if (step == share)
#pragma unroll
            for (int j = 0; j < S::DY_VECS; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) bias[i] += get(from.dy[j], i);
        step = step + 1 == A.bias_shares ? 0 : step + 1;
    };

    // where a lane reads: rows 8 (lane / 32) + (lane % 16) / 4, columns 16 (lane / 16 % 2) + 4 (lane % 4) of a 32-column piece
    const uint32_t r = lane / 32 * 8 + lane % 16 / 4, cc = lane / 16 % 2 * 16 + lane % 4 * 4;
    uint32_t at_o[S::FRAGS], at_c[2];
#pragma unroll
    for (int f = 0; f < S::FRAGS; ++f) at_o[f] = lds_at<S::TILE_O>(r, wave_o + f * 32 + cc);
#pragma unroll
    for (int f = 0; f < 2; ++f) at_c[f] = lds_at<S::TILE_C>(r, wave_c + f * 32 + cc) + S::PARTS * S::DY_BYTES;
    f32x16 sum[S::FRAGS][2];
    // One step, in UNITS turns of a few products; the fragments of a turn are read during the one before.  Between them, a later
    // step is put into its buffer.  (The turns are kept apart: moved into each other they take more registers than there
    // are.)
    constexpr int UNITS = TURNS * S::PARTS;
    Frag x[2][2], y[2][S::FRAGS];
    auto read = [&](uint32_t buffer, int u) {
        const int k = u / S::PARTS, p = S::PARTS - 1 - u % S::PARTS;
        if (u % S::PARTS == 0)
#pragma unroll
            for (int f = 0; f < 2; ++f) x[k % 2][f] = read_fragment<S::TILE_C, Frag>(lds + buffer, at_c[f] + k * 16 * (S::TILE_C * 2));
#pragma unroll
        for (int f = 0; f < S::FRAGS; ++f)
            y[u % 2][f] = read_fragment<S::TILE_O, Frag>(lds + buffer, at_o[f] + p * S::DY_BYTES + k * 16 * (S::TILE_O * 2));
    };
    auto multiply = [&](uint32_t buffer, uint32_t after, bool first, auto&& between) {
        if constexpr (S::AHEAD == 1) read(buffer, 0);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            if (u + 1 < UNITS) read(buffer, u + 1);
            else if constexpr (S::AHEAD > 1) read(after, 0);
            if (u % S::PARTS == 0) between(u / S::PARTS);
#pragma unroll
            for (int i = 0; i < S::FRAGS; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) sum[i][j] = Mma<DyT>::mul(y[u % 2][i], x[u / S::PARTS % 2][j], first && u == 0 ? f32x16{} : sum[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    static_assert(S::AHEAD == 1 || (UNITS % 2 == 0 && TURNS % 2 == 0), "a step's first fragments go where its first turn looks for them");

    f32x16 total[S::FRAGS][2] = {};
    Staged<DyT, S> staged[2];
    uint32_t buffer = 0;                                      // that of the present step
    auto behind = [&](int n) {                                // that of the n-th step after it
        const uint32_t at = buffer + n * S::BUFFER;
        return at < S::BUFFERS * S::BUFFER ? at : at - S::BUFFERS * S::BUFFER;
    };
    const int32_t steps = (t_end - t_first + S::STEP - 1) / S::STEP;
    if (steps > 0) {
#pragma unroll
        for (int n = 0; n < S::AHEAD + 2; ++n) {
            if (n >= 2 && n - 2 < steps) {
                add_bias(staged[n % 2]);
                put_step<DyT, S>(staged[n % 2], lds + (n - 2) * S::BUFFER, dy_row, dy_col, q_row, q_col);
            }
            if (n < steps) fetch(staged[n % 2], std::false_type());
        }
        __syncthreads();
        if constexpr (S::AHEAD > 1) read(0, 0);
    }
    auto group = [&](int32_t at, auto steady) {               // the steps from `at`, a group's first
        float scale[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const int32_t c = c0 + wave_c + f * 32 + lane % 32;
            scale[f] = c < A.channels ? A.scale[(t_first / GROUP + at / S::STEPS) * A.ld + c] : 0.f;
        }
#pragma unroll
        for (int s = 0; s < S::STEPS; ++s) {
            Staged<DyT, S>& later = staged[(s + S::AHEAD) % 2];
            const uint32_t to = behind(S::AHEAD), after = behind(1);
            if constexpr (decltype(steady)::value) {
                add_bias(later);
                multiply(buffer, after, s == 0, [&](int k) { put_some(later, lds + to, k); });
                fetch(later, steady);
                __syncthreads();
            } else if (at + s < steps) {
                if (at + s + S::AHEAD < steps) {
                    add_bias(later);
                    put_step<DyT, S>(later, lds + to, dy_row, dy_col, q_row, q_col);
                }
                if (at + s + S::AHEAD + 2 < steps) fetch(later, steady);
                multiply(buffer, after, s == 0, [](int) {});             // behind the last step: fragments that nothing uses
                __syncthreads();
            }
            buffer = after;
        }
#pragma unroll
        for (int i = 0; i < S::FRAGS; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) total[i][j][e] = __builtin_fmaf(scale[j], sum[i][j][e], total[i][j][e]);
    };
    int32_t at = 0;
    // as long as every step of a group has AHEAD + 2 whole ones behind it
    for (; (at + S::STEPS + S::AHEAD + 2) * S::STEP <= t_end - t_first; at += S::STEPS) group(at, std::true_type());
    for (; at < steps; at += S::STEPS) group(at, std::false_type());

    if (share != ~0u)
        write_bias<GradT, S>(A, reinterpret_cast<float*>(lds), bias, o0, dy_row, dy_col, A.splits * A.bias_shares > 1 ? nullptr : A.db,
                             split_no * A.bias_shares + share);
    float* const whole = reinterpret_cast<float*>(lds);
    if (A.splits > 1)
        write_tile<S, false>(whole, total, wave_o, wave_c, lane, A.partial + (static_cast<int64_t>(split_no) * A.outputs + o0) * A.channels_padded + c0,
                             A.channels_padded, A.outputs - o0, static_cast<int32_t>(A.channels_padded) - c0, false);
    else
        write_tile<S, false>(whole, total, wave_o, wave_c, lane, static_cast<GradT*>(A.dw) + o0 * A.dw_stride + c0, A.dw_stride, A.outputs - o0,
                             A.channels - c0, A.accumulate);
}

// Few tokens, one group of them: what counts is dw, which is written once, so the tiles are small and many workgroups share a
// compute unit: while some write their tiles, others read and multiply theirs.  A scale belongs to one sum; there is nothing to
// join.  32 tokens, 25088 channels, 4096 outputs, binary32: 71 us, 412 MB at 5.8 TB/s, nearly all of it the write of dw (a bare fill
// writes 6.8).
template <typename DyT> using Short = Shape<DyT, 1, 2, 2, 32, 1>;
// A dw larger than the 256 MB memory-side cache is written past it.  32 tokens, 25088 channels, binary32, with a reader behind (a
// maximum over dw): 392 MB 183 us streamed and 209 kept, 196 MB 99 and 91, 98 MB 57 and 47; the kernel alone is 1 to 7 %
// faster streamed at every size.
constexpr int64_t STREAM_BYTES = 256 << 20;
constexpr int SHORT_TILE_O = 64, SHORT_PER_CU = 4;

template <typename DyT, typename GradT, bool RAGGED, bool STREAM>
__global__ __launch_bounds__(Short<DyT>::THREADS, SHORT_PER_CU) void linear_short_kernel(LinearArgs A) {
    typedef Short<DyT> S;
    typedef typename Mma<DyT>::frag Frag;
    __shared__ __align__(256) char lds[S::LDS];
    const uint32_t tile_o = blockIdx.x / A.tiles_c, tile_c = blockIdx.x - tile_o * A.tiles_c;
    const int32_t o0 = tile_o * S::TILE_O, c0 = tile_c * S::TILE_C;
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t wave_o = wave / S::WAVES_C * (S::FRAGS * 32), wave_c = wave % S::WAVES_C * 64;
    const uint32_t dy_col = threadIdx.x % (S::TILE_O / VEC) * VEC, dy_row = threadIdx.x / (S::TILE_O / VEC);
    const uint32_t q_col = threadIdx.x % (S::TILE_C / S::XW) * S::XW, q_row = threadIdx.x / (S::TILE_C / S::XW);
    const int32_t o_in = o0 + static_cast<int32_t>(dy_col);
    const int dy_n = RAGGED ? max(0, min(A.outputs - o_in, VEC)) : VEC;
    const DyT* const dy_at = static_cast<const DyT*>(A.dy) + (RAGGED ? o_in : min(o_in, A.outputs - VEC));
    const int8_t* const q_at = A.q + piece_at(c0 + q_col, A.q_columns, S::XW);
    const uint32_t r = lane / 32 * 8 + lane % 16 / 4, cc = lane / 16 % 2 * 16 + lane % 4 * 4;
    float scale[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        const int32_t c = c0 + wave_c + f * 32 + lane % 32;
        scale[f] = A.tokens > 0 && c < A.channels ? A.scale[c] : 0.f;      // without tokens there is no scale
    }
    float bias[VEC] = {};
    f32x16 sum[S::FRAGS][2] = {};
    for (int32_t t0 = 0; t0 < A.tokens; t0 += S::STEP) {
        Staged<DyT, S> staged;
#pragma unroll
        for (int j = 0; j < S::DY_VECS; ++j) {
            const int32_t t = t0 + dy_row + S::DY_ROWS * j;
            staged.dy[j] = load8(dy_at + t * A.dy_stride, t < A.tokens ? dy_n : 0);
        }
#pragma unroll
        for (int j = 0; j < S::X_VECS; ++j) {
            const int32_t t = t0 + q_row + S::X_ROWS * j;
            staged.q[j] = typename S::X(0);
            if (t < A.tokens && (!RAGGED || A.ld > 0)) staged.q[j] = *reinterpret_cast<const typename S::X*>(q_at + t * A.ld);
        }
        if (t0 > 0) __syncthreads();
        put_step<DyT, S>(staged, lds, dy_row, dy_col, q_row, q_col);
        if (A.db != nullptr && tile_c == 0)
#pragma unroll
            for (int j = 0; j < S::DY_VECS; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) bias[i] += get(staged.dy[j], i);
        __syncthreads();
        const int turns = min(S::STEP, A.tokens - t0 + 15) / 16;
#pragma unroll
        for (int k = 0; k < S::STEP / 16; ++k) {
            if (k >= turns) break;
            Frag x[2];
#pragma unroll
            for (int f = 0; f < 2; ++f)
                x[f] = read_fragment<S::TILE_C, Frag>(lds + S::PARTS * S::DY_BYTES, lds_at<S::TILE_C>(r, wave_c + f * 32 + cc) + k * 16 * (S::TILE_C * 2));
#pragma unroll
            for (int p = S::PARTS - 1; p >= 0; --p)
#pragma unroll
                for (int i = 0; i < S::FRAGS; ++i) {
                    const Frag y = read_fragment<S::TILE_O, Frag>(lds + p * S::DY_BYTES, lds_at<S::TILE_O>(r, wave_o + i * 32 + cc) + k * 16 * (S::TILE_O * 2));
#pragma unroll
                    for (int j = 0; j < 2; ++j) sum[i][j] = Mma<DyT>::mul(y, x[j], sum[i][j]);
                }
        }
    }
    if (A.db != nullptr && tile_c == 0) write_bias<GradT, S>(A, reinterpret_cast<float*>(lds), bias, o0, dy_row, dy_col, A.db, 0);
#pragma unroll
    for (int i = 0; i < S::FRAGS; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[i][j][e] *= scale[j];
    write_tile<S, STREAM>(reinterpret_cast<float*>(lds), sum, wave_o, wave_c, lane, static_cast<GradT*>(A.dw) + o0 * A.dw_stride + c0, A.dw_stride,
                          A.outputs - o0, A.channels - c0, A.accumulate);
}

constexpr int JOIN_THREADS = 256;

// The splits' sums, in order: a thread takes four channels of an output.  The first bias_blocks workgroups join the bias.  Two splits of
// 4096 outputs and 1024 channels, 42 MB: 7 us, half of it the launch and the first wait for memory.
template <typename GradT> __global__ __launch_bounds__(JOIN_THREADS) void linear_join_kernel(LinearArgs A) {
    if (blockIdx.x < A.bias_blocks) {
        const int32_t o = blockIdx.x * JOIN_THREADS + threadIdx.x;
        if (o >= A.outputs) return;
        float sum = 0.f;
#pragma unroll 8
        for (uint32_t s = 0; s < A.splits * A.bias_shares; ++s) sum += A.bias_partial[static_cast<int64_t>(s) * A.outputs + o];
        GradT* const b = static_cast<GradT*>(A.db) + o;
        *b = rounded<GradT>(sum + (A.accumulate ? static_cast<float>(*b) : 0.f));
        return;
    }
    const uint32_t at = (blockIdx.x - A.bias_blocks) * JOIN_THREADS + threadIdx.x;
    const uint32_t vecs = static_cast<uint32_t>(A.channels_padded / 4);
    const uint32_t o = at / vecs, c = (at - o * vecs) * 4;
    if (o >= static_cast<uint32_t>(A.outputs)) return;
    const float* p = A.partial + static_cast<int64_t>(o) * A.channels_padded + c;
    const int64_t next = A.outputs * A.channels_padded;
    f32x4 all = *reinterpret_cast<const f32x4*>(p);
#pragma unroll 4
    for (uint32_t s = 1; s < A.splits; ++s) all += *reinterpret_cast<const f32x4*>(p += next);
    GradT* const w = static_cast<GradT*>(A.dw) + static_cast<int64_t>(o) * A.dw_stride + c;
    float sum[4] = {all[0], all[1], all[2], all[3]};
    if (A.accumulate)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < static_cast<uint32_t>(A.channels)) sum[i] += static_cast<float>(w[i]);
    store_some(w, sum, A.channels - static_cast<int32_t>(c));
}

// The tiles: 256 outputs by 128 channels, 64 tokens a step, 144 KiB of LDS.  Where dy takes three parts, 128 outputs by 256 channels,
// 32 tokens and 128 KiB: q's bytes are the cheaper ones there (1024 channels, 4096 outputs, 32768 tokens 753 us, the other
// way round 830; level in 16 bits).
template <typename DyT> using Wide = Shape<DyT, 2, sizeof(DyT) == 4 ? 2 : 4, sizeof(DyT) == 4 ? 4 : 2, sizeof(DyT) == 4 ? 32 : 64, sizeof(DyT) == 4 ? 2 : 3>;
// Square ones: 128 outputs by 128 channels, half as many registers for sums.
template <typename DyT> using Square = Shape<DyT, 1, 4, 2, sizeof(DyT) == 4 ? 32 : 64, sizeof(DyT) == 4 ? 2 : 3>;
enum { SHORT, SQUARE, WIDE, WIDE_PARTS };
constexpr int TILE_O[] = {SHORT_TILE_O, 128, 256, 128}, TILE_C[] = {128, 128, 128, 256};
static_assert(Wide<float>::TILE_O == TILE_O[WIDE_PARTS] && Wide<__bf16>::TILE_O == TILE_O[WIDE] && Square<float>::TILE_O == TILE_O[SQUARE], "tiles");

struct LinearPlan {
    int form;
    uint32_t tiles_o, tiles_c, groups, splits, groups_per_split, bias_shares;
    int64_t channels_padded, bias_at, bytes;
};

// Which tiles.  Wide ones read least (binary16, 4096 channels and outputs, 8192 tokens: 333 us, square 423).  But where they are
// at most half as many as the compute units they are split over the tokens and joined, and with few tokens that costs more than it
// gives: 1024 channels, 4096 outputs, 1024 tokens 31 us, square 17; 4096 tokens 55 and 54; 1024 outputs and 16384 tokens
// 55 and 60; binary32 with 256 tokens, 1024 channels and outputs 18 and 13.
constexpr int64_t SQUARE_GROUPS = 16;

LinearPlan plan_of(int64_t tokens, int64_t channels, int64_t outputs, bool parts) {
    LinearPlan p{};
    p.groups = static_cast<uint32_t>(ceil_div(tokens, GROUP));
    const int wide = parts ? WIDE_PARTS : WIDE;
    p.form = p.groups <= 1 ? SHORT : p.groups <= SQUARE_GROUPS && ceil_div(outputs, TILE_O[wide]) * ceil_div(channels, TILE_C[wide]) < 256 ? SQUARE : wide;
    p.tiles_c = static_cast<uint32_t>(std::max<int64_t>(ceil_div(channels, TILE_C[p.form]), 1));       // the bias is made with some tile
    p.tiles_o = static_cast<uint32_t>(ceil_div(outputs, TILE_O[p.form]));
    const int64_t tiles = static_cast<int64_t>(p.tiles_o) * p.tiles_c;
    // As many workgroups as there are compute units, 256, at most, and two groups at the least for each of them.  In whole numbers: 129 to 255
    // tiles are not split, and with more than 256 the last round of workgroups is as long as a full one.  bfloat16, 4096 tokens (32768):
    // 1024 channels to 4096 outputs, 256 workgroups, 630 TFLOP/s (810); 1280 to 5120, 200 of them, 670 (700); 1536 to 6144, 288, 550 (550);
    // 2048 to 8192, 512, 860 (840).
    int64_t splits = std::min<int64_t>({256 / std::max<int64_t>(tiles, 1), std::max<uint32_t>(p.groups / 2, 1), MAX_SPLITS});
    splits = std::max<int64_t>(splits, 1);
    p.groups_per_split = static_cast<uint32_t>(ceil_div(std::max<uint32_t>(p.groups, 1), splits));
    p.splits = static_cast<uint32_t>(ceil_div(std::max<uint32_t>(p.groups, 1), p.groups_per_split));
    p.bias_shares = p.splits > 1 ? std::min<uint32_t>(p.tiles_c, BIAS_SHARES) : 1;
    p.channels_padded = ceil_div(channels, 4) * 4;
    const int64_t sums = p.splits > 1 ? p.splits * outputs * p.channels_padded * 4 : 0;
    p.bias_at = ceil_div(sums, 256) * 256;
    p.bytes = p.splits > 1 ? p.bias_at + static_cast<int64_t>(p.splits) * p.bias_shares * outputs * 4 : 0;
    return p;
}

bool sizes_ok(int64_t tokens, int64_t channels, int64_t outputs) {
    return tokens >= 0 && tokens <= (int64_t(1) << 23) && channels >= 0 && channels <= (int64_t(1) << 23) && outputs >= 0 &&
           outputs <= (int64_t(1) << 23) && ceil_div(channels, 128) * ceil_div(outputs, 128) <= (int64_t(1) << 22);
}

}  // namespace

extern "C" {

int mgwfbp_act_linear_grad_workspace(int64_t n_tokens, int64_t n_channels, int64_t n_outputs, uint64_t* bytes_out) {
    if (bytes_out == nullptr || !sizes_ok(n_tokens, n_channels, n_outputs)) return MGWFBP_EINVAL;
    *bytes_out = static_cast<uint64_t>(std::max(plan_of(n_tokens, n_channels, n_outputs, false).bytes, plan_of(n_tokens, n_channels, n_outputs, true).bytes));
    return MGWFBP_OK;
}

int mgwfbp_act_linear_grad(const int8_t* d_q, const float* d_scale, int64_t ld, int64_t n_tokens, int64_t n_channels,
                           const void* d_dy, int64_t dy_stride, int32_t dy_dtype, int64_t n_outputs, int32_t accumulate,
                           void* d_dw, int64_t dw_stride, void* d_db, int32_t grad_dtype, void* d_workspace,
                           uint64_t workspace_bytes, void* hip_stream) {
    if (!sizes_ok(n_tokens, n_channels, n_outputs) || !is_dtype(dy_dtype) || !is_dtype(grad_dtype)) return MGWFBP_EINVAL;
    if (!is_matrix(n_tokens, n_outputs, dy_stride, dtype_bytes(dy_dtype)) ||
        !is_matrix(n_outputs, n_channels, dw_stride, dtype_bytes(grad_dtype)))
        return MGWFBP_EINVAL;
    if (n_outputs == 0 || (n_channels == 0 && d_db == nullptr)) return MGWFBP_OK;
    if (n_channels > 0) {
        if (d_dw == nullptr || !is_aligned(d_dw, dtype_bytes(grad_dtype))) return MGWFBP_EINVAL;
        if (n_tokens > 0 && (d_q == nullptr || d_scale == nullptr || !is_aligned(d_q, 16) || !is_aligned(d_scale, 16) ||
                             ld < n_channels || ld % 16 != 0 || !is_matrix(n_tokens, n_channels, ld, 4)))
            return MGWFBP_EINVAL;
    }
    if (d_db != nullptr && !is_aligned(d_db, dtype_bytes(grad_dtype))) return MGWFBP_EINVAL;
    if (n_tokens > 0 && (d_dy == nullptr || !is_aligned(d_dy, dtype_bytes(dy_dtype)))) return MGWFBP_EINVAL;
    const LinearPlan p = plan_of(n_tokens, n_channels, n_outputs, dy_dtype == MGWFBP_F32);
    if (p.bytes > 0 && (d_workspace == nullptr || !is_aligned(d_workspace, 256) || workspace_bytes < static_cast<uint64_t>(p.bytes)))
        return MGWFBP_EINVAL;
    LinearArgs a{};
    a.dy = d_dy;
    a.q = d_q;
    a.scale = d_scale;
    a.dw = d_dw;
    a.db = d_db;
    a.partial = static_cast<float*>(d_workspace);
    a.bias_partial = reinterpret_cast<float*>(static_cast<unsigned char*>(d_workspace) + p.bias_at);
    a.dy_stride = dy_stride;
    a.ld = ld;
    a.q_columns = own_columns(n_channels);
    a.dw_stride = dw_stride;
    a.tokens = static_cast<int32_t>(n_tokens);
    a.channels = static_cast<int32_t>(n_channels);
    a.outputs = static_cast<int32_t>(n_outputs);
    a.channels_padded = p.channels_padded;
    a.tiles_c = p.tiles_c;
    a.tiles = p.tiles_o * p.tiles_c;
    a.splits = p.splits;
    a.groups = p.groups;
    a.groups_per_split = p.groups_per_split;
    a.bias_shares = p.bias_shares;
    a.accumulate = accumulate != 0;
    if (n_channels == 0) a.ld = 0;                       // no q: the bias alone
    // Split launches have at most 256 tiles, so that the join's threads number less than 2^22.
    a.bias_blocks = d_db != nullptr ? static_cast<uint32_t>(ceil_div(n_outputs, JOIN_THREADS)) : 0;
    const dim3 join_grid(a.bias_blocks + static_cast<uint32_t>(p.splits > 1 ? ceil_div(n_outputs * (p.channels_padded / 4), JOIN_THREADS) : 0));
    return with_dtype(dy_dtype, [&](auto* dy_type) {
        return with_dtype(grad_dtype, [&](auto* grad_type) {
            typedef std::remove_pointer_t<decltype(dy_type)> DyT;
            typedef std::remove_pointer_t<decltype(grad_type)> GradT;
            const bool ragged = n_outputs % VEC != 0 || a.ld == 0;
            const bool stream = n_outputs * n_channels * static_cast<int64_t>(sizeof(GradT)) >= STREAM_BYTES;
            void (*few)(LinearArgs) = ragged ? (stream ? linear_short_kernel<DyT, GradT, true, true> : linear_short_kernel<DyT, GradT, true, false>)
                                             : (stream ? linear_short_kernel<DyT, GradT, false, true> : linear_short_kernel<DyT, GradT, false, false>);
            void (*square)(LinearArgs) = ragged ? linear_kernel<DyT, GradT, Square<DyT>, true> : linear_kernel<DyT, GradT, Square<DyT>, false>;
            void (*wide)(LinearArgs) = ragged ? linear_kernel<DyT, GradT, Wide<DyT>, true> : linear_kernel<DyT, GradT, Wide<DyT>, false>;
            const int rc = launch(p.form == SHORT ? few : p.form == SQUARE ? square : wide, a, dim3(a.tiles * a.splits),
                                  dim3(p.form == SHORT ? Short<DyT>::THREADS : p.form == SQUARE ? Square<DyT>::THREADS : Wide<DyT>::THREADS), hip_stream);
            if (rc != MGWFBP_OK || a.splits == 1) return rc;
            return launch(linear_join_kernel<GradT>, a, join_grid, dim3(JOIN_THREADS), hip_stream);
        });
    });
}

}  // extern "C"
