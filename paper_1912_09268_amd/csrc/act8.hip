// Activation checkpoints in 8 bits: making them, and the way back through an activation function.
//
//   mgwfbp_act_store      scale[g,c] = max(max over the group's tokens of |x[t,c]|, 2^-100) / 127
//                         q[t,c] = x[t,c] / scale[g,c] rounded to the nearest whole number, ties to even;  y = f(x)
//   mgwfbp_act_backward   x^ = q * scale;  dx = dy * f'(x^);  y = f(x^)
//
// A group is MGWFBP_ACT_GROUP consecutive tokens of one channel.  The largest magnitudes of activations sit in single
// channels, so a scale of its own for each channel loses less than one for each token; and mgwfbp_act_linear_grad sums over
// tokens, so that a group's scale comes out of the sum.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "act_code.h"
#include "act_kinds.h"
#include "act_layout.h"
#include "device_types.h"
#include "mgwfbp_layers.h"

namespace {

using namespace ops;

constexpr int THREADS = 256;
constexpr int GROUP = MGWFBP_ACT_GROUP;

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------------------------
// store
// ---------------------------------------------------------------------------------------------

struct StoreArgs {
    const void* x;
    void* y;
    int8_t* q;
    float* scale;
    int64_t x_stride, y_stride, ld;      // ld: of q and of scale
    int64_t tokens, channels;
    uint32_t col_blocks;
};

constexpr int LANES = 16;                                    // lanes side by side: 128 channels, whole lines of q and of 16-bit x
constexpr int BLOCK_COLS = LANES * VEC;
constexpr int ROWS = THREADS / LANES;                        // rows of a step
constexpr int STEPS = GROUP / ROWS;

// Magnitudes of eight elements as bit patterns without sign, in which infinities and NaN are above all finite ones; 16-bit types
// are kept in pairs.
template <typename T> struct Magnitudes {
    static constexpr int N = VEC * sizeof(T) / 4;
    uint32_t m[N] = {};
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        if constexpr (sizeof(T) == 4) return max(a, b);
        else return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
    }
    __device__ __forceinline__ void take(const Raw8<T>& x) {
        typedef uint32_t words __attribute__((ext_vector_type(N)));
        const words w = __builtin_bit_cast(words, x);
#pragma unroll
        for (int i = 0; i < N; ++i) m[i] = larger(m[i], w[i] & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu));
    }
    __device__ __forceinline__ void take(int i, uint32_t other) { m[i] = larger(m[i], other); }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, m[i]);
        else return static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(m[i / 2] >> (16 * (i % 2)))));
    }
};

// A workgroup takes 128 channels of a group: the whole of it stays in registers between the search for the largest magnitude
// and the rounding, so x is read once.  y does not wait for that: it is made and written as rows arrive.  4096 tokens of 4096
// bfloat16 channels with GELU: 21 us, 84 MB at 4.0 TB/s, and 15 without the function's arithmetic, which is what is left above the
// rate of a copy (an instruction an element is 0.4 us).  (Fewer wavefronts side by side than the registers allow are level.)
template <typename T, int KIND, bool Y> __global__ __launch_bounds__(THREADS) void store_kernel(StoreArgs A) {
    const uint32_t g = blockIdx.x / A.col_blocks, cb = blockIdx.x - g * A.col_blocks;
    const uint32_t lane = threadIdx.x % LANES, row = threadIdx.x / LANES;
    const int64_t col = static_cast<int64_t>(cb) * BLOCK_COLS + lane * VEC;
    const int n = static_cast<int>(max(static_cast<int64_t>(0), min(A.channels - col, static_cast<int64_t>(VEC))));
    const int64_t t0 = static_cast<int64_t>(g) * GROUP + row;
    const T* const from = static_cast<const T*>(A.x) + t0 * A.x_stride + col;
    T* const to = static_cast<T*>(A.y) + t0 * A.y_stride + col;
    Raw8<T> x[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) x[s] = load8(from + s * (ROWS * A.x_stride), t0 + s * ROWS < A.tokens ? n : 0);
    Magnitudes<T> most;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        most.take(x[s]);
        if constexpr (Y)
            if (t0 + s * ROWS < A.tokens && n > 0) {
                float out[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    float slope;
                    activate<KIND>(get(x[s], i), out[i], slope);
                }
                store8(to + s * (ROWS * A.y_stride), out, n);
            }
    }
    constexpr int N = Magnitudes<T>::N;
    __shared__ uint32_t of_wave[THREADS / 64][LANES * N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        most.take(i, __shfl_xor(most.m[i], 16));
        most.take(i, __shfl_xor(most.m[i], 32));
        if (threadIdx.x % 64 < LANES) of_wave[threadIdx.x / 64][lane * N + i] = most.m[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) most.take(i, of_wave[w][lane * N + i]);
    if (col >= own_columns(A.channels)) return;
    float scale[VEC], inv[VEC];
    u32x2 keep = {0, 0};                                     // a group that is not finite has codes of 0
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        // The bound keeps scale and its inverse normal numbers.
        const float largest = most.get(i);
        const bool finite = __builtin_bit_cast(uint32_t, largest) < 0x7f800000u;
        scale[i] = max(largest, 0x1p-100f) * (1.f / 127.f);
        inv[i] = 1.f / scale[i];
        keep[i / 4] |= finite ? 0xffu << (8 * (i % 4)) : 0u;
        scale[i] = i >= n ? 0.f : finite ? scale[i] : __builtin_nanf("");
    }
    if (row == 0) store8(A.scale + g * A.ld + col, scale);
    int8_t* const q = A.q + t0 * A.ld + col;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        if (t0 + s * ROWS >= A.tokens) break;
        float r[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) r[i] = get(x[s], i) * inv[i];
        *reinterpret_cast<u32x2*>(q + s * (ROWS * A.ld)) = u32x2{four_codes(r[0], r[1], r[2], r[3]), four_codes(r[4], r[5], r[6], r[7])} & keep;
    }
}

// ---------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------

struct BackwardArgs {
    const int8_t* q;
    const float* scale;
    const void* dy;
    void* dx;
    void* y;
    int64_t ld, dy_stride, dx_stride, y_stride;
    int64_t tokens, channels;
    uint32_t vecs, page;                 // vectors of a row; blocks of rows per blockIdx.y
};

constexpr int BACK_ROWS = 8;             // rows of a lane, all of one group: they share its scales

// One lane for eight channels of eight tokens, four of them on their way at a time; nothing is shared between lanes.  Bound by
// memory: 65536 tokens of 4096 binary16 channels with tanh GELU, gradient and value, 337 us, 1.9 GB at 5.6 TB/s; 4096 bfloat16 tokens
// with GELU, gradient alone, 18 us, 84 MB at 4.6 TB/s.  f' is computed and not stored: that would be as many bytes as dy.
template <typename T, int KIND, bool SLOPE, bool VALUE> __global__ __launch_bounds__(THREADS) void backward_kernel(BackwardArgs A) {
    const uint32_t at = blockIdx.x * THREADS + threadIdx.x;
    const uint32_t in_page = at / A.vecs, v = at - in_page * A.vecs;
    const int64_t t0 = (static_cast<int64_t>(blockIdx.y) * A.page + in_page) * BACK_ROWS;
    if (in_page >= A.page || t0 >= A.tokens) return;
    const int64_t col = static_cast<int64_t>(v) * VEC;
    const int n = static_cast<int>(min(A.channels - col, static_cast<int64_t>(VEC)));
    const Raw8<float> scale = load8(A.scale + t0 / GROUP * A.ld + col);
#pragma unroll
    for (int r0 = 0; r0 < BACK_ROWS; r0 += 4) {
        u32x2 q[4];
        Raw8<T> dy[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t t = min(t0 + r0 + r, A.tokens - 1);
            q[r] = *reinterpret_cast<const u32x2*>(A.q + t * A.ld + col);
            if constexpr (SLOPE) dy[r] = load8(static_cast<const T*>(A.dy) + t * A.dy_stride + col, n);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t t = t0 + r0 + r;
            if (t >= A.tokens) return;
            float dx[VEC], y[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float slope;
                activate<KIND>(code_of(q[r], i) * get(scale, i), y[i], slope);
                if constexpr (SLOPE) dx[i] = get(dy[r], i) * slope;
            }
            if constexpr (SLOPE) store8(static_cast<T*>(A.dx) + t * A.dx_stride + col, dx, n);
            if constexpr (VALUE) store8(static_cast<T*>(A.y) + t * A.y_stride + col, y, n);
        }
    }
}

bool is_kind(int32_t k) { return k >= MGWFBP_IDENTITY && k <= MGWFBP_SILU; }

bool act_ok(int64_t tokens, int64_t channels, const void* q, const void* scale, int64_t ld) {
    if (tokens < 0 || tokens > (int64_t(1) << 26) || channels < 0 || channels > (int64_t(1) << 23)) return false;
    if (tokens == 0 || channels == 0) return true;
    return q != nullptr && scale != nullptr && is_aligned(q, 16) && is_aligned(scale, 16) && ld >= channels && ld % 16 == 0 &&
           is_matrix(tokens, channels, ld, 4);
}

bool side_ok(const void* p, int64_t tokens, int64_t channels, int64_t stride, int32_t dtype) {
    return p == nullptr || (is_aligned(p, dtype_bytes(dtype)) && is_matrix(tokens, channels, stride, dtype_bytes(dtype)));
}

}  // namespace

extern "C" {

int mgwfbp_act_dims(int64_t n_tokens, int64_t n_channels, int64_t* ld_out, int64_t* n_groups_out) {
    if (n_tokens < 0 || n_tokens > (int64_t(1) << 26) || n_channels < 0 || n_channels > (int64_t(1) << 23)) return MGWFBP_EINVAL;
    if (ld_out != nullptr) *ld_out = own_columns(n_channels);
    if (n_groups_out != nullptr) *n_groups_out = ops::ceil_div(n_tokens, GROUP);
    return MGWFBP_OK;
}

int mgwfbp_act_store(const void* d_x, int64_t x_stride, int32_t dtype, int64_t n_tokens, int64_t n_channels, int32_t kind,
                     int8_t* d_q, float* d_scale, int64_t ld, void* d_y, int64_t y_stride, void* hip_stream) {
    if (!is_dtype(dtype) || !is_kind(kind) || !act_ok(n_tokens, n_channels, d_q, d_scale, ld)) return MGWFBP_EINVAL;
    if (n_tokens == 0 || n_channels == 0) return MGWFBP_OK;
    if (d_x == nullptr || !side_ok(d_x, n_tokens, n_channels, x_stride, dtype) || !side_ok(d_y, n_tokens, n_channels, y_stride, dtype))
        return MGWFBP_EINVAL;
    StoreArgs a{};
    a.x = d_x;
    a.y = d_y;
    a.q = d_q;
    a.scale = d_scale;
    a.x_stride = x_stride;
    a.y_stride = y_stride;
    a.ld = ld;
    a.tokens = n_tokens;
    a.channels = n_channels;
    a.col_blocks = static_cast<uint32_t>(ceil_div(n_channels, BLOCK_COLS));
    const int64_t blocks = a.col_blocks * ceil_div(n_tokens, GROUP);
    if (blocks >= (int64_t(1) << 24)) return MGWFBP_EINVAL;
    return with_dtype(dtype, [&](auto* type) {
        return with_kind(kind, [&](auto k) {
            typedef std::remove_pointer_t<decltype(type)> T;
            void (*kernel)(StoreArgs) = d_y == nullptr ? store_kernel<T, MGWFBP_IDENTITY, false> : store_kernel<T, decltype(k)::value, true>;
            return launch(kernel, a, dim3(static_cast<uint32_t>(blocks)), dim3(THREADS), hip_stream);
        });
    });
}

int mgwfbp_act_backward(const int8_t* d_q, const float* d_scale, int64_t ld, int64_t n_tokens, int64_t n_channels, int32_t kind,
                        const void* d_dy, int64_t dy_stride, void* d_dx, int64_t dx_stride, void* d_y, int64_t y_stride,
                        int32_t dtype, void* hip_stream) {
    if (!is_dtype(dtype) || !is_kind(kind) || !act_ok(n_tokens, n_channels, d_q, d_scale, ld)) return MGWFBP_EINVAL;
    if ((d_dx == nullptr) != (d_dy == nullptr)) return MGWFBP_EINVAL;
    if (n_tokens == 0 || n_channels == 0) return MGWFBP_OK;
    if (d_dx == nullptr && d_y == nullptr) return MGWFBP_EINVAL;
    if (!side_ok(d_dy, n_tokens, n_channels, dy_stride, dtype) || !side_ok(d_dx, n_tokens, n_channels, dx_stride, dtype) ||
        !side_ok(d_y, n_tokens, n_channels, y_stride, dtype))
        return MGWFBP_EINVAL;
    BackwardArgs a{};
    a.q = d_q;
    a.scale = d_scale;
    a.dy = d_dy;
    a.dx = d_dx;
    a.y = d_y;
    a.ld = ld;
    a.dy_stride = dy_stride;
    a.dx_stride = dx_stride;
    a.y_stride = y_stride;
    a.tokens = n_tokens;
    a.channels = n_channels;
    a.vecs = static_cast<uint32_t>(ceil_div(n_channels, VEC));
    const int64_t row_blocks = ceil_div(n_tokens, BACK_ROWS);
    a.page = static_cast<uint32_t>(std::min<int64_t>(row_blocks, (int64_t(1) << 31) / a.vecs - 1));
    if (ceil_div(row_blocks, a.page) > 65535) return MGWFBP_EINVAL;
    const dim3 grid(static_cast<uint32_t>(ceil_div(static_cast<int64_t>(a.page) * a.vecs, THREADS)),
                    static_cast<uint32_t>(ceil_div(row_blocks, a.page)));
    return with_dtype(dtype, [&](auto* type) {
        return with_kind(kind, [&](auto k) {
            typedef std::remove_pointer_t<decltype(type)> T;
            constexpr int K = decltype(k)::value;
            void (*kernel)(BackwardArgs) = d_dx == nullptr ? backward_kernel<T, K, false, true>
                                         : d_y == nullptr ? backward_kernel<T, K, true, false> : backward_kernel<T, K, true, true>;
            return launch(kernel, a, grid, dim3(THREADS), hip_stream);
        });
    });
}

}  // extern "C"
