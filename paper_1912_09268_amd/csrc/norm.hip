// Root-mean-square norm with the residual's addition, its 8-bit checkpoint, and the way back from that.
//
//   mgwfbp_norm            h = x + residual, rounded to the stream's type;  rstd[t] = 1 / sqrt(mean of h[t,:]^2 + eps)
//                          n = h * rstd;  y = n * weight;  n in 8 bits as act8.hip does, and the steps of y beside those of n
//   mgwfbp_norm_backward   n^ = q * scale;  g = weight * dy;  dh = dresidual + rstd * (g - n^ * mean of g n^);  dw = sum over t of dy n^
//
// What is kept is n, not h and not y: one memory of 8 bits serves the norm's way back, which needs n, and the weight gradient of the
// linear layer behind it, which needs y.  Steps belong to channels, and so does the weight, so y is held by n's codes with the steps
// scale * weight.
//
// The mean square is summed in binary64 and rstd rounded to binary32 once.  So n, a binary32 product, and with it every code and
// step, is the same whatever the order of the sum; in binary32 the last bit of rstd would go by it, and a code next to a border by
// that.  It also leaves no square that overflows.  A multiplication in binary64 for each element is nothing beside its memory.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "act_code.h"
#include "act_layout.h"
#include "device_types.h"
#include "mgwfbp_layers.h"
#include "spans.h"
#include "teams.h"

namespace {

using namespace ops;

constexpr int GROUP = MGWFBP_ACT_GROUP;

// Eight weights from col on, of which n are there; all 1 where there is no weight.
__device__ __forceinline__ void load_weight(const void* w, int32_t type, int64_t col, int n, float (&out)[VEC]) {
    if (w == nullptr) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) out[i] = 1.f;
    } else if (type == MGWFBP_F32) {
        const Raw8<float> r = load8(static_cast<const float*>(w) + col, n);
#pragma unroll
        for (int i = 0; i < VEC; ++i) out[i] = get(r, i);
    } else if (type == MGWFBP_BF16) {
        const Raw8<__bf16> r = load8(static_cast<const __bf16*>(w) + col, n);
#pragma unroll
        for (int i = 0; i < VEC; ++i) out[i] = get(r, i);
    } else {
        const Raw8<_Float16> r = load8(static_cast<const _Float16*>(w) + col, n);
#pragma unroll
        for (int i = 0; i < VEC; ++i) out[i] = get(r, i);
    }
}

__device__ __forceinline__ int columns_at(int64_t channels, int64_t col) {
    return static_cast<int>(max(static_cast<int64_t>(0), min(channels - col, static_cast<int64_t>(VEC))));
}

// ---------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------

struct NormArgs {
    const void* x;
    const void* residual;
    const void* weight;
    void* h;
    void* y;
    float* rstd;
    int64_t x_stride, residual_stride, h_stride, y_stride;
    int64_t tokens, channels;
    double eps;
    int32_t weight_type;
};

// A team of TEAM lanes has a row, V vectors of eight columns a lane: the row stays in registers between the sum and the product.
// Bound by memory and, in short calls, by the launch and two waits: 4096 tokens of 1024 bfloat16 channels with residual 8.0 us, 34 MB at
// 4.2 TB/s; 32775 tokens of 4096 binary16 channels on a binary32 stream, with the codes, 400 us, 2.3 GB at 5.6 TB/s.  (Two rows a team at a time, which
// halves the readings of the weight, are level to 5 % slower.)
template <typename T, typename S, int TEAM, int V> __global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void norm_kernel(NormArgs A) {
    constexpr int THREADS = TEAM < 256 ? 256 : TEAM;
    const uint32_t lane = threadIdx.x % TEAM;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * (THREADS / TEAM) + threadIdx.x / TEAM;
    const bool here = t < A.tokens;                          // teams of a workgroup go on together: they share its barriers
    const int64_t row = here ? t : 0;
    Raw8<T> x[V];
    Raw8<S> res[V];
    float h[V][VEC], w[V][VEC];
    int n[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int64_t col = (static_cast<int64_t>(v) * TEAM + lane) * VEC;
        n[v] = here ? columns_at(A.channels, col) : 0;
        x[v] = load8(static_cast<const T*>(A.x) + row * A.x_stride + col, n[v]);
        if (A.residual != nullptr) res[v] = load8(static_cast<const S*>(A.residual) + row * A.residual_stride + col, n[v]);
        load_weight(A.weight, A.weight_type, col, n[v], w[v]);
    }
    double squares = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            h[v][i] = get(x[v], i);
            if (A.residual != nullptr) h[v][i] = static_cast<float>(rounded<S>(h[v][i] + get(res[v], i)));
            squares = __builtin_fma(static_cast<double>(h[v][i]), static_cast<double>(h[v][i]), squares);
        }
        if (A.residual != nullptr) store8(static_cast<S*>(A.h) + row * A.h_stride + (static_cast<int64_t>(v) * TEAM + lane) * VEC, h[v], n[v]);
    }
    if constexpr (TEAM <= 64) {
        squares = lanes_sum<TEAM>(squares);
    } else {
        __shared__ double room[TEAM / 64];
        squares = workgroup_sum<TEAM>(squares, room);
    }
    const float rstd = static_cast<float>(1.0 / sqrt(squares / static_cast<double>(A.channels) + A.eps));
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float y[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) y[i] = h[v][i] * rstd * w[v][i];
        store8(static_cast<T*>(A.y) + row * A.y_stride + (static_cast<int64_t>(v) * TEAM + lane) * VEC, y, n[v]);
    }
    if (A.rstd != nullptr && here && lane == 0) A.rstd[t] = rstd;
}

// Rows that do not fit a workgroup's registers: h is made, summed and, where there is a residual, written, and taken up again.
template <typename T, typename S> __global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs A) {
    constexpr int THREADS = 1024;
    const int64_t t = blockIdx.x, step = THREADS * VEC, first = static_cast<int64_t>(threadIdx.x) * VEC;
    const T* const x = static_cast<const T*>(A.x) + t * A.x_stride;
    const S* const residual = static_cast<const S*>(A.residual) + t * A.residual_stride;
    S* const h = static_cast<S*>(A.h) + t * A.h_stride;
    T* const y = static_cast<T*>(A.y) + t * A.y_stride;
    double squares = 0.0;
    for (int64_t col = first; col < A.channels; col += step) {
        const int n = columns_at(A.channels, col);
        const Raw8<T> a = load8(x + col, n);
        float sum[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] = get(a, i);
        if (A.residual != nullptr) {
            const Raw8<S> b = load8(residual + col, n);
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] = static_cast<float>(rounded<S>(sum[i] + get(b, i)));
            store8(h + col, sum, n);
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) squares = __builtin_fma(static_cast<double>(sum[i]), static_cast<double>(sum[i]), squares);
    }
    __shared__ double room[THREADS / 64];
    squares = workgroup_sum<THREADS>(squares, room);
    const float rstd = static_cast<float>(1.0 / sqrt(squares / static_cast<double>(A.channels) + A.eps));
    for (int64_t col = first; col < A.channels; col += step) {
        const int n = columns_at(A.channels, col);
        float w[VEC], out[VEC];
        load_weight(A.weight, A.weight_type, col, n, w);
        if (A.residual != nullptr) {                         // what this very lane has written
            const Raw8<S> b = load8(const_cast<const S*>(h) + col, n);
#pragma unroll
            for (int i = 0; i < VEC; ++i) out[i] = get(b, i) * rstd * w[i];
        } else {
            const Raw8<T> a = load8(x + col, n);
#pragma unroll
            for (int i = 0; i < VEC; ++i) out[i] = get(a, i) * rstd * w[i];
        }
        store8(y + col, out, n);
    }
    if (A.rstd != nullptr && threadIdx.x == 0) A.rstd[t] = rstd;
}

struct CodeArgs {
    const void* h;
    const float* rstd;
    const void* weight;
    int8_t* q;
    float* scale;
    float* linear_scale;
    int64_t h_stride, ld, tokens, channels;
    uint32_t col_blocks;
    int32_t weight_type;
};

constexpr int CODE_THREADS = 256;

// n = h * rstd in 8 bits: a workgroup has 8 LANES channels of a group of tokens in registers while it looks for the largest magnitude.
// h has just been written or read and mostly comes from the caches, the last groups first.  Its magnitudes are known behind the whole group alone, so the norm,
// which has whole rows, cannot make them: 4096 tokens of 1024 bfloat16 channels 5.0 us, 13 MB, a launch and two waits.
template <typename S, int LANES> __global__ __launch_bounds__(CODE_THREADS) void code_kernel(CodeArgs A) {
    constexpr int BLOCK_COLS = LANES * VEC, ROWS = CODE_THREADS / LANES, STEPS = GROUP / ROWS;
    const uint32_t from_end = blockIdx.x / A.col_blocks, cb = blockIdx.x - from_end * A.col_blocks, g = gridDim.x / A.col_blocks - 1 - from_end;
    const uint32_t lane = threadIdx.x % LANES, row = threadIdx.x / LANES;
    const int64_t col = static_cast<int64_t>(cb) * BLOCK_COLS + lane * VEC;
    const int n = columns_at(A.channels, col);
    const int64_t t0 = static_cast<int64_t>(g) * GROUP + row;
    const S* const from = static_cast<const S*>(A.h) + t0 * A.h_stride + col;
    Raw8<S> h[STEPS];
    float rstd[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const bool here = t0 + s * ROWS < A.tokens;
        h[s] = load8(from + s * (ROWS * A.h_stride), here ? n : 0);
        rstd[s] = here ? A.rstd[t0 + s * ROWS] : 0.f;
    }
    float w[VEC];
    load_weight(A.weight, A.weight_type, col, n, w);
    uint32_t most[VEC] = {};                                 // bit patterns without sign: infinities and NaN are above all finite ones
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int i = 0; i < VEC; ++i) most[i] = max(most[i], __builtin_bit_cast(uint32_t, get(h[s], i) * rstd[s]) & 0x7fffffffu);
    __shared__ uint32_t of_wave[CODE_THREADS / 64][BLOCK_COLS];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
#pragma unroll
        for (int d = LANES; d < 64; d *= 2) most[i] = max(most[i], static_cast<uint32_t>(__shfl_xor(static_cast<int>(most[i]), d)));
        if (threadIdx.x % 64 < LANES) of_wave[threadIdx.x / 64][lane * VEC + i] = most[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < VEC; ++i)
#pragma unroll
        for (int v = 0; v < CODE_THREADS / 64; ++v) most[i] = max(most[i], of_wave[v][lane * VEC + i]);
    if (col >= own_columns(A.channels)) return;
    float scale[VEC], inv[VEC], linear[VEC];
    u32x2 keep = {0, 0};                                     // a group that is not finite has codes of 0
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const bool finite = most[i] < 0x7f800000u;
        scale[i] = max(__builtin_bit_cast(float, finite ? most[i] : 0u), 0x1p-100f) * (1.f / 127.f);
        inv[i] = 1.f / scale[i];
        keep[i / 4] |= finite ? 0xffu << (8 * (i % 4)) : 0u;
        scale[i] = i >= n ? 0.f : finite ? scale[i] : __builtin_nanf("");
        linear[i] = i >= n ? 0.f : scale[i] * w[i];
    }
    if (row == 0) {
        store8(A.scale + g * A.ld + col, scale);
        store8(A.linear_scale + g * A.ld + col, linear);
    }
    int8_t* const q = A.q + t0 * A.ld + col;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        if (t0 + s * ROWS >= A.tokens) break;
        float r[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) r[i] = get(h[s], i) * rstd[s] * inv[i];
        *reinterpret_cast<u32x2*>(q + s * (ROWS * A.ld)) = u32x2{four_codes(r[0], r[1], r[2], r[3]), four_codes(r[4], r[5], r[6], r[7])} & keep;
    }
}

// ---------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------

struct BackArgs {
    const int8_t* q;
    const float* scale;
    const float* rstd;
    const void* weight;
    const void* dy;
    const void* dres;
    void* dh;
    void* dx;
    float* partial;                      // [workgroups][padded]: sums of dw; null where there is no dw
    float* mean;                         // [tokens] of rows too long for a team
    int64_t ld, dy_stride, dres_stride, dh_stride, dx_stride, padded;
    int64_t tokens, channels;
    int64_t rows;                        // of a team, or of a workgroup's tile of a long row
    float over_channels;
    int32_t weight_type;
};

template <typename T, typename S> __device__ __forceinline__ void finish(const BackArgs& A, int64_t t, int64_t col, int n, const float (&grad)[VEC], const Raw8<S>& dres) {
    float dh[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) dh[i] = A.dres != nullptr ? get(dres, i) + grad[i] : grad[i];
    store8(static_cast<S*>(A.dh) + t * A.dh_stride + col, dh, n);
    if (A.dx != nullptr) store8(static_cast<T*>(A.dx) + t * A.dx_stride + col, dh, n);
}

// A team of TEAM lanes goes through `rows` consecutive rows, V vectors of eight columns a lane, the next row on its way while one is
// worked on; the lanes' columns stay the same, so their share of dw stays in registers.  Bound by memory: 32775 tokens of 4096 binary16 channels on
// a binary32 stream 291 us, 1.5 GB at 5.1 TB/s, four wavefronts a SIMD that wait for 60 % of their time; 4096 tokens of 1024 bfloat16 channels 12 us, of which joining dw is a launch of 4.
// Small teams share a workgroup, so that there are few sums of dw to join.
constexpr int back_threads(int team, int vecs) { return team >= 256 ? team : vecs == 1 ? 1024 : 512; }

template <typename T, typename S, int TEAM, int V> __global__ __launch_bounds__(back_threads(TEAM, V)) void back_kernel(BackArgs A) {
    constexpr int THREADS = back_threads(TEAM, V), TEAMS = THREADS / TEAM;
    const uint32_t lane = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    const int64_t begin = (static_cast<int64_t>(blockIdx.x) * TEAMS + team) * A.rows;
    const int64_t end = min(begin + A.rows, A.tokens);
    int64_t col[V];
    int n[V];
    float w[V][VEC], sum[V][VEC] = {};
#pragma unroll
    for (int v = 0; v < V; ++v) {
        col[v] = (static_cast<int64_t>(v) * TEAM + lane) * VEC;
        n[v] = columns_at(A.channels, col[v]);
        load_weight(A.weight, A.weight_type, col[v], n[v], w[v]);
    }
    struct Row {
        u32x2 q[V];
        Raw8<T> dy[V];
        Raw8<S> dres[V];
        float rstd;
    };
    auto load = [&](int64_t t) {
        Row r;
        r.rstd = t < end ? A.rstd[t] : 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int m = t < end ? n[v] : 0;
            r.q[v] = u32x2{0, 0};
            if (m > 0) r.q[v] = *reinterpret_cast<const u32x2*>(A.q + t * A.ld + col[v]);
            r.dy[v] = load8(static_cast<const T*>(A.dy) + t * A.dy_stride + col[v], m);
            if (A.dres != nullptr) r.dres[v] = load8(static_cast<const S*>(A.dres) + t * A.dres_stride + col[v], m);
        }
        return r;
    };
    constexpr int ROOM = TEAM > 64 ? 2 * (TEAM / 64) : 1;    // two rows' sums, so that one barrier a row is enough
    __shared__ float room[ROOM];
    Raw8<float> scale[V];
    int64_t group = -1;
    Row next = load(begin);
    for (int64_t t = begin; t < end; ++t) {                  // a workgroup of one team shares barriers: all its lanes have the same rows
        const Row now = next;
        next = load(t + 1);
        if (t / GROUP != group) {
            group = t / GROUP;
#pragma unroll
            for (int v = 0; v < V; ++v) scale[v] = load8(A.scale + group * A.ld + col[v], n[v]);
        }
        float dot = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float normed = code_of(now.q[v], i) * get(scale[v], i), dy = get(now.dy[v], i);
                sum[v][i] = __builtin_fmaf(dy, normed, sum[v][i]);
                dot = __builtin_fmaf(dy * w[v][i], normed, dot);
            }
        if constexpr (TEAM <= 64) dot = lanes_sum<TEAM>(dot);
        else dot = workgroup_sum<TEAM>(dot, room + (t % 2) * (TEAM / 64));
        const float mean = dot * A.over_channels;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (n[v] <= 0) continue;
            float grad[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) grad[i] = now.rstd * (get(now.dy[v], i) * w[v][i] - code_of(now.q[v], i) * get(scale[v], i) * mean);
            finish<T, S>(A, t, col[v], n[v], grad, now.dres[v]);
        }
    }
    if (A.partial == nullptr) return;
    if constexpr (TEAMS == 1) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (col[v] < A.padded) store8(A.partial + blockIdx.x * A.padded + col[v], sum[v]);
    } else {
        __shared__ float shares[TEAMS][TEAM * V * VEC];
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i) shares[team][(v * TEAM + lane) * VEC + i] = sum[v][i];
        __syncthreads();
        for (int c = threadIdx.x; c < TEAM * V * VEC && c < A.padded; c += THREADS) {
            float s = shares[0][c];
#pragma unroll
            for (int k = 1; k < TEAMS; ++k) s += shares[k][c];
            A.partial[blockIdx.x * A.padded + c] = s;
        }
    }
}

// Rows too long for a team: the mean first ...
template <typename T> __global__ __launch_bounds__(1024) void back_mean_kernel(BackArgs A) {
    constexpr int THREADS = 1024;
    const int64_t t = blockIdx.x;
    float dot = 0.f;
    for (int64_t col = static_cast<int64_t>(threadIdx.x) * VEC; col < A.channels; col += THREADS * VEC) {
        const int n = columns_at(A.channels, col);
        const u32x2 q = *reinterpret_cast<const u32x2*>(A.q + t * A.ld + col);
        const Raw8<float> scale = load8(A.scale + t / GROUP * A.ld + col, n);
        const Raw8<T> dy = load8(static_cast<const T*>(A.dy) + t * A.dy_stride + col, n);
        float w[VEC];
        load_weight(A.weight, A.weight_type, col, n, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < n) dot = __builtin_fmaf(get(dy, i) * w[i], code_of(q, i) * get(scale, i), dot);
    }
    __shared__ float room[THREADS / 64];
    dot = workgroup_sum<THREADS>(dot, room);
    if (threadIdx.x == 0) A.mean[t] = dot * A.over_channels;
}

// ... and then tiles of 2048 columns and `rows` rows.
constexpr int TILE = 256;
template <typename T, typename S> __global__ __launch_bounds__(TILE) void back_tile_kernel(BackArgs A) {
    const int64_t col = (static_cast<int64_t>(blockIdx.x) * TILE + threadIdx.x) * VEC;
    const int n = columns_at(A.channels, col);
    if (n == 0) return;
    const int64_t begin = static_cast<int64_t>(blockIdx.y) * A.rows, end = min(begin + A.rows, A.tokens);
    float w[VEC], sum[VEC] = {};
    load_weight(A.weight, A.weight_type, col, n, w);
    for (int64_t t = begin; t < end; ++t) {
        const u32x2 q = *reinterpret_cast<const u32x2*>(A.q + t * A.ld + col);
        const Raw8<float> scale = load8(A.scale + t / GROUP * A.ld + col, n);
        const Raw8<T> dy = load8(static_cast<const T*>(A.dy) + t * A.dy_stride + col, n);
        Raw8<S> dres;
        if (A.dres != nullptr) dres = load8(static_cast<const S*>(A.dres) + t * A.dres_stride + col, n);
        float grad[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float normed = code_of(q, i) * (i < n ? get(scale, i) : 0.f);
            sum[i] = __builtin_fmaf(get(dy, i), normed, sum[i]);
            grad[i] = A.rstd[t] * (get(dy, i) * w[i] - normed * A.mean[t]);
        }
        finish<T, S>(A, t, col, n, grad, dres);
    }
    if (A.partial != nullptr) store8(A.partial + blockIdx.y * A.padded + col, sum);
}

struct JoinArgs {
    const float* partial;
    void* dw;
    int64_t padded, channels;
    int32_t parts, accumulate, grad_type;
};

constexpr int JOIN_COLS = 32, JOIN_ROWS = 32;

// dw from the workgroups' sums, in order.
__global__ __launch_bounds__(JOIN_COLS * JOIN_ROWS) void join_kernel(JoinArgs A) {
    const int lane = threadIdx.x % JOIN_COLS, row = threadIdx.x / JOIN_COLS;
    const int64_t col = static_cast<int64_t>(blockIdx.x) * JOIN_COLS + lane;
    float sum = 0.f;
    if (col < A.channels) {
#pragma unroll 8
        for (int p = row; p < A.parts; p += JOIN_ROWS) sum += A.partial[p * A.padded + col];
    }
    __shared__ float sums[JOIN_ROWS][JOIN_COLS + 1];
    sums[row][lane] = sum;
    __syncthreads();
    if (row != 0 || col >= A.channels) return;
#pragma unroll
    for (int r = 1; r < JOIN_ROWS; ++r) sum += sums[r][lane];
    if (A.grad_type == MGWFBP_F32) {
        float* const to = static_cast<float*>(A.dw) + col;
        *to = A.accumulate ? *to + sum : sum;
    } else if (A.grad_type == MGWFBP_BF16) {
        __bf16* const to = static_cast<__bf16*>(A.dw) + col;
        *to = rounded<__bf16>(A.accumulate ? static_cast<float>(*to) + sum : sum);
    } else {
        _Float16* const to = static_cast<_Float16*>(A.dw) + col;
        *to = rounded<_Float16>(A.accumulate ? static_cast<float>(*to) + sum : sum);
    }
}

// ---- host side -------------------------------------------------------------------------------

constexpr int64_t MOST_TOKENS = int64_t(1) << 26, MOST_CHANNELS = int64_t(1) << 23, TEAM_CHANNELS = 16384, BACK_TEAM_CHANNELS = 8192;

// Pieces of 128 channels and 128 tokens below which a workgroup takes half of one: 1003 tokens of 1001 binary32 channels 5.9 and 4.8 us.  Norm and codes of 1024 bfloat16
// channels, whole pieces and halves: 1024 tokens (64 pieces) 8.0 and 7.5 us, 2048 (128) 8.9 and 8.5, 4096 (256) 11.4 both, as are 192 to 512 pieces of other shapes within 1 %;
// 8192 tokens of 2048 (1024) 25.9 and 26.7 (binary32 44.6 and 43.6).  Beyond, whole lines of q are better: 32775 tokens of 4096 channels, binary16 on a binary32 stream, 400 and 424.
constexpr int64_t NARROW_BELOW = 256;

// Calls f with the team and the vectors of a lane for rows of `channels` columns, up to BACK_TEAM_CHANNELS.  Us forward and back, bfloat16, the other shape
// behind the one taken: 65536 tokens of 128 channels 16 x 1 12 and 14, 64 x 1 27 and 30; 32768 of 512 64 x 1 25 and 30, 16 x 4 25 and 53; 32768 of 1024
// 64 x 2 46 and 53, 256 x 1 58 and 86; 8192 of 2048 256 x 1 25 and 31, 64 x 4 26 and 53; 32775 of 4096, binary16 on a binary32 stream, 512 x 1 280 and 291,
// 256 x 2 293 and 296; 4096 of 6000 512 x 2 41 and 59, 1024 x 1 45 and 57.
template <int T_, int V_> struct Shape { static constexpr int team = T_, vecs = V_; };
template <typename F> auto with_shape(int64_t channels, F&& f) {
    if (channels <= 128) return f(Shape<16, 1>());
    if (channels <= 512) return f(Shape<64, 1>());
    if (channels <= 1024) return f(Shape<64, 2>());
    if (channels <= 2048) return f(Shape<256, 1>());
    if (channels <= 4096) return f(Shape<512, 1>());
    return f(Shape<512, 2>());
}

// How the way back is cut: workgroups, rows of a team (or of a tile).
struct Cut {
    int64_t workgroups, rows, padded;
    bool wide;
};
Cut cut_of(int64_t tokens, int64_t channels) {
    Cut c{};
    c.padded = ceil_div(channels, VEC) * VEC;
    c.wide = channels > BACK_TEAM_CHANNELS;
    if (c.wide) {
        c.rows = std::max<int64_t>(16, ceil_div(tokens, std::max<int64_t>(1, 1024 / ceil_div(channels, TILE * VEC))));
        c.rows = std::max(c.rows, ceil_div(tokens, 65535));
        c.workgroups = ceil_div(tokens, c.rows);
        return c;
    }
    const int64_t teams = with_shape(channels, [](auto s) { return static_cast<int64_t>(back_threads(decltype(s)::team, decltype(s)::vecs) / decltype(s)::team); });
    c.rows = ceil_div(tokens, (teams > 1 ? 256 : 512) * teams);
    c.workgroups = ceil_div(tokens, c.rows * teams);
    return c;
}

// The types of a branch and of the stream it is added to: the same, or a binary32 stream.
template <typename F> int with_types(int32_t dtype, int32_t stream, F&& f) {
    return with_dtype(dtype, [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        if (stream == dtype) return f(static_cast<T*>(nullptr), static_cast<T*>(nullptr));
        return stream == MGWFBP_F32 ? f(static_cast<T*>(nullptr), static_cast<float*>(nullptr)) : static_cast<int>(MGWFBP_EINVAL);
    });
}

bool sizes_ok(int64_t tokens, int64_t channels) { return tokens >= 0 && tokens <= MOST_TOKENS && channels >= 0 && channels <= MOST_CHANNELS; }
bool types_ok(int32_t dtype, int32_t stream) { return is_dtype(dtype) && (stream == dtype || stream == MGWFBP_F32); }
bool kept_ok(const int8_t* q, const float* scale, const float* rstd, int64_t tokens, int64_t channels, int64_t ld) {
    return q != nullptr && scale != nullptr && rstd != nullptr && is_aligned(q, 16) && is_aligned(scale, 16) && is_aligned(rstd, 4) && ld >= channels &&
           ld % 16 == 0 && is_matrix(tokens, channels, ld, 4);
}
bool side_ok(const void* p, int64_t tokens, int64_t channels, int64_t stride, int32_t dtype) {
    return p != nullptr && is_aligned(p, dtype_bytes(dtype)) && is_matrix(tokens, channels, stride, dtype_bytes(dtype));
}
int64_t weight_bytes(const void* w, int32_t type) { return w == nullptr ? 0 : dtype_bytes(type); }
bool weight_ok(const void* w, int32_t type) { return w == nullptr || (is_dtype(type) && is_aligned(w, dtype_bytes(type))); }

}  // namespace

extern "C" {

int mgwfbp_norm(const void* d_x, int64_t x_stride, int32_t dtype, const void* d_residual, int64_t residual_stride, int32_t stream_dtype,
                int64_t n_tokens, int64_t n_channels, const void* d_weight, int32_t weight_dtype, double eps, void* d_h, int64_t h_stride,
                void* d_y, int64_t y_stride, float* d_rstd, int8_t* d_q, float* d_scale, float* d_linear_scale, int64_t ld, void* hip_stream) {
    if (!types_ok(dtype, stream_dtype) || !sizes_ok(n_tokens, n_channels) || !weight_ok(d_weight, weight_dtype)) return MGWFBP_EINVAL;
    if (!(eps >= 0x1p-100) || !(eps <= 0x1p100)) return MGWFBP_EINVAL;
    if (n_tokens == 0 || n_channels == 0) return MGWFBP_OK;
    if ((d_residual == nullptr) != (d_h == nullptr) || (d_residual == nullptr && stream_dtype != dtype)) return MGWFBP_EINVAL;
    const bool keep = d_q != nullptr;
    if (keep != (d_rstd != nullptr) || keep != (d_scale != nullptr) || keep != (d_linear_scale != nullptr)) return MGWFBP_EINVAL;
    if (!side_ok(d_x, n_tokens, n_channels, x_stride, dtype) || !side_ok(d_y, n_tokens, n_channels, y_stride, dtype)) return MGWFBP_EINVAL;
    if (d_residual != nullptr && (!side_ok(d_residual, n_tokens, n_channels, residual_stride, stream_dtype) ||
                                  !side_ok(d_h, n_tokens, n_channels, h_stride, stream_dtype)))
        return MGWFBP_EINVAL;
    if (keep && (!kept_ok(d_q, d_scale, d_rstd, n_tokens, n_channels, ld) || !is_aligned(d_linear_scale, 16))) return MGWFBP_EINVAL;
    const int64_t bytes = dtype_bytes(dtype), stream_bytes = dtype_bytes(stream_dtype), own = own_columns(n_channels), groups = ceil_div(n_tokens, GROUP);
    const uint32_t H = 1, Y = 2, made_of_x = d_residual == nullptr && keep;             // the codes are made of h, behind y
    if (tangled({matrix_span(d_h, n_tokens, n_channels, h_stride, stream_bytes), matrix_span(d_y, n_tokens, n_channels, y_stride, bytes), vector_span(d_rstd, n_tokens, 4),
                 matrix_span(d_q, n_tokens, own, ld, 1), matrix_span(d_scale, groups, own, ld, 4), matrix_span(d_linear_scale, groups, own, ld, 4)},
                {{matrix_span(d_x, n_tokens, n_channels, x_stride, bytes), made_of_x ? 0 : H | Y},
                 {matrix_span(d_residual, n_tokens, n_channels, residual_stride, stream_bytes), H | Y},
                 {vector_span(d_weight, n_channels, weight_bytes(d_weight, weight_dtype)), 0}}))
        return MGWFBP_EINVAL;
    CodeArgs c{};
    const bool narrow = ceil_div(n_channels, 128) * ceil_div(n_tokens, GROUP) < NARROW_BELOW;
    c.col_blocks = static_cast<uint32_t>(ceil_div(n_channels, narrow ? 64 : 128));
    const int64_t code_blocks = c.col_blocks * ceil_div(n_tokens, GROUP);
    if (keep && code_blocks >= (int64_t(1) << 24)) return MGWFBP_EINVAL;
    NormArgs a{};
    a.x = d_x;
    a.residual = d_residual;
    a.weight = d_weight;
    a.h = d_h;
    a.y = d_y;
    a.rstd = d_rstd;
    a.x_stride = x_stride;
    a.residual_stride = residual_stride;
    a.h_stride = h_stride;
    a.y_stride = y_stride;
    a.tokens = n_tokens;
    a.channels = n_channels;
    a.eps = eps;
    a.weight_type = weight_dtype;
    const int status = with_types(dtype, stream_dtype, [&](auto* type, auto* stream_type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        typedef std::remove_pointer_t<decltype(stream_type)> S;
        if (n_channels > TEAM_CHANNELS) return launch(norm_long_kernel<T, S>, a, dim3(static_cast<uint32_t>(n_tokens)), dim3(1024), hip_stream);
        if (n_channels > BACK_TEAM_CHANNELS) return launch(norm_kernel<T, S, 1024, 2>, a, dim3(static_cast<uint32_t>(n_tokens)), dim3(1024), hip_stream);
        return with_shape(n_channels, [&](auto s) {
            constexpr int TEAM = decltype(s)::team, THREADS = TEAM < 256 ? 256 : TEAM;
            void (*kernel)(NormArgs) = norm_kernel<T, S, TEAM, decltype(s)::vecs>;
            return launch(kernel, a, dim3(static_cast<uint32_t>(ceil_div(n_tokens, THREADS / TEAM))), dim3(THREADS), hip_stream);
        });
    });
    if (status != MGWFBP_OK || !keep) return status;
    c.h = d_residual != nullptr ? d_h : d_x;
    c.rstd = d_rstd;
    c.weight = d_weight;
    c.q = d_q;
    c.scale = d_scale;
    c.linear_scale = d_linear_scale;
    c.h_stride = d_residual != nullptr ? h_stride : x_stride;
    c.ld = ld;
    c.tokens = n_tokens;
    c.channels = n_channels;
    c.weight_type = weight_dtype;
    return with_dtype(stream_dtype, [&](auto* type) {
        typedef std::remove_pointer_t<decltype(type)> S;
        return launch(narrow ? code_kernel<S, 8> : code_kernel<S, 16>, c, dim3(static_cast<uint32_t>(code_blocks)), dim3(CODE_THREADS), hip_stream);
    });
}

int mgwfbp_norm_backward_workspace(int64_t n_tokens, int64_t n_channels, uint64_t* bytes_out) {
    if (!sizes_ok(n_tokens, n_channels) || bytes_out == nullptr) return MGWFBP_EINVAL;
    *bytes_out = 0;
    if (n_tokens == 0 || n_channels == 0) return MGWFBP_OK;
    const Cut c = cut_of(n_tokens, n_channels);
    *bytes_out = static_cast<uint64_t>(c.workgroups * c.padded + (c.wide ? n_tokens : 0)) * 4;
    return MGWFBP_OK;
}

int mgwfbp_norm_backward(const int8_t* d_q, const float* d_scale, int64_t ld, const float* d_rstd, int64_t n_tokens, int64_t n_channels,
                         const void* d_weight, int32_t weight_dtype, const void* d_dy, int64_t dy_stride, int32_t dtype, const void* d_dresidual,
                         int64_t dresidual_stride, void* d_dh, int64_t dh_stride, int32_t stream_dtype, void* d_dx, int64_t dx_stride, int32_t accumulate,
                         void* d_dw, int32_t grad_dtype, void* d_workspace, uint64_t workspace_bytes, void* hip_stream) {
    if (!types_ok(dtype, stream_dtype) || !sizes_ok(n_tokens, n_channels) || !weight_ok(d_weight, weight_dtype)) return MGWFBP_EINVAL;
    if (d_dw != nullptr && (!is_dtype(grad_dtype) || !is_aligned(d_dw, dtype_bytes(grad_dtype)))) return MGWFBP_EINVAL;
    if (n_channels == 0) return MGWFBP_OK;
    JoinArgs j{};
    j.dw = d_dw;
    j.channels = n_channels;
    j.accumulate = accumulate != 0;
    j.grad_type = grad_dtype;
    const dim3 join_grid(static_cast<uint32_t>(ceil_div(n_channels, JOIN_COLS)));
    if (n_tokens == 0) return d_dw == nullptr || accumulate ? static_cast<int>(MGWFBP_OK) : launch(join_kernel, j, join_grid, dim3(JOIN_COLS * JOIN_ROWS), hip_stream);
    if (!kept_ok(d_q, d_scale, d_rstd, n_tokens, n_channels, ld) || !side_ok(d_dy, n_tokens, n_channels, dy_stride, dtype) ||
        !side_ok(d_dh, n_tokens, n_channels, dh_stride, stream_dtype) ||
        (d_dresidual != nullptr && !side_ok(d_dresidual, n_tokens, n_channels, dresidual_stride, stream_dtype)) ||
        (d_dx != nullptr && !side_ok(d_dx, n_tokens, n_channels, dx_stride, dtype)))
        return MGWFBP_EINVAL;
    const Cut cut = cut_of(n_tokens, n_channels);
    uint64_t needed = 0;
    if (d_dw != nullptr || cut.wide) {
        mgwfbp_norm_backward_workspace(n_tokens, n_channels, &needed);
        if (d_workspace == nullptr || !is_aligned(d_workspace, 256) || workspace_bytes < needed) return MGWFBP_EINVAL;
    }
    const int64_t bytes = dtype_bytes(dtype), stream_bytes = dtype_bytes(stream_dtype), own = own_columns(n_channels);
    const uint32_t DH = 1, DX = 2;
    if (tangled({matrix_span(d_dh, n_tokens, n_channels, dh_stride, stream_bytes), matrix_span(d_dx, n_tokens, n_channels, dx_stride, bytes),
                 vector_span(d_dw, n_channels, weight_bytes(d_dw, grad_dtype)), vector_span(d_workspace, static_cast<int64_t>(needed), 1)},
                {{matrix_span(d_dy, n_tokens, n_channels, dy_stride, bytes), DH | DX},
                 {matrix_span(d_dresidual, n_tokens, n_channels, dresidual_stride, stream_bytes), DH | DX},
                 {matrix_span(d_q, n_tokens, own, ld, 1), 0},
                 {matrix_span(d_scale, ceil_div(n_tokens, GROUP), own, ld, 4), 0},
                 {vector_span(d_rstd, n_tokens, 4), 0},
                 {vector_span(d_weight, n_channels, weight_bytes(d_weight, weight_dtype)), 0}}))
        return MGWFBP_EINVAL;
    BackArgs a{};
    a.q = d_q;
    a.scale = d_scale;
    a.rstd = d_rstd;
    a.weight = d_weight;
    a.dy = d_dy;
    a.dres = d_dresidual;
    a.dh = d_dh;
    a.dx = d_dx;
    a.partial = d_dw == nullptr ? nullptr : static_cast<float*>(d_workspace);
    a.mean = cut.wide ? static_cast<float*>(d_workspace) + cut.workgroups * cut.padded : nullptr;
    a.ld = ld;
    a.dy_stride = dy_stride;
    a.dres_stride = dresidual_stride;
    a.dh_stride = dh_stride;
    a.dx_stride = dx_stride;
    a.padded = cut.padded;
    a.tokens = n_tokens;
    a.channels = n_channels;
    a.rows = cut.rows;
    a.over_channels = 1.f / static_cast<float>(n_channels);
    a.weight_type = weight_dtype;
    const int status = with_types(dtype, stream_dtype, [&](auto* type, auto* stream_type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        typedef std::remove_pointer_t<decltype(stream_type)> S;
        if (cut.wide) {
            const int s = launch(back_mean_kernel<T>, a, dim3(static_cast<uint32_t>(n_tokens)), dim3(1024), hip_stream);
            if (s != MGWFBP_OK) return s;
            return launch(back_tile_kernel<T, S>, a, dim3(static_cast<uint32_t>(ceil_div(n_channels, TILE * VEC)), static_cast<uint32_t>(cut.workgroups)), dim3(TILE),
                          hip_stream);
        }
        return with_shape(n_channels, [&](auto s) {
            constexpr int TEAM = decltype(s)::team, V = decltype(s)::vecs, THREADS = back_threads(TEAM, V);
            void (*kernel)(BackArgs) = back_kernel<T, S, TEAM, V>;
            return launch(kernel, a, dim3(static_cast<uint32_t>(cut.workgroups)), dim3(THREADS), hip_stream);
        });
    });
    if (status != MGWFBP_OK || d_dw == nullptr) return status;
    j.partial = a.partial;
    j.padded = cut.padded;
    j.parts = static_cast<int32_t>(cut.workgroups);
    return launch(join_kernel, j, join_grid, dim3(JOIN_COLS * JOIN_ROWS), hip_stream);
}

}  // extern "C"
