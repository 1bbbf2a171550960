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

#include "device_types.h"
#include "mgwfbp_layers.h"

namespace {

using namespace ops;

constexpr int GROUP = MGWFBP_ACT_GROUP;
constexpr int THREADS = 256;
constexpr int TILE_O = 128, TILE_C = 128, STEP = 64;          // outputs, channels and tokens that a workgroup takes at a time
constexpr int MAX_SPLITS = 64;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct LinearArgs {
    const void* dy;
    const int8_t* q;
    const float* scale;
    void* dw;
    void* db;
    float* partial;                    // [splits][outputs][channels_padded], and the bias parts behind it
    float* bias_partial;               // [bias_parts][outputs]
    int64_t dy_stride, ld, dw_stride;
    int64_t tokens, channels, outputs, channels_padded;
    uint32_t tiles_c, tiles, splits, groups, groups_per_split, bias_parts;
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

// LDS: tiles of STEP rows (tokens) by 128 columns of 2 bytes.  A fragment of the matrix instruction has eight tokens of one
// column in a lane, so it is read transposed (ds_read_b64_tr_b16: sixteen lanes read four rows of 16 columns and get four
// tokens of a column each).  The four rows begin on the same bank, so the 64-byte pieces of a row are exchanged by the
// row's two lowest bits.
constexpr int ROW_BYTES = 256;
__device__ __forceinline__ uint32_t lds_at(uint32_t row, uint32_t col) {
    return row * ROW_BYTES + ((col / 32 ^ (row & 3)) * 64) + (col % 32) * 2;
}

template <typename Frag> __device__ __forceinline__ Frag read_fragment(const char* tile, uint32_t at) {
    typedef __attribute__((address_space(3))) s16x4* lds;
    union { s16x4 half[2]; Frag whole; } u;
    u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(tile + at));
    u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(tile + at + 4 * ROW_BYTES));
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

template <typename DyT, typename GradT>
__global__ __launch_bounds__(THREADS) void linear_kernel(LinearArgs A) {
    typedef typename Mma<DyT>::elem E;
    typedef typename Mma<DyT>::frag Frag;
    constexpr int PARTS = Parts<DyT>::n;
    constexpr int TILE_BYTES = STEP * ROW_BYTES;
    __shared__ __align__(256) char lds[(PARTS + 1) * TILE_BYTES];
    char* const lds_x = lds + PARTS * TILE_BYTES;

    const uint32_t split_no = blockIdx.x / A.tiles, tile = blockIdx.x - split_no * A.tiles;
    const uint32_t tile_o = tile / A.tiles_c, tile_c = tile - tile_o * A.tiles_c;
    const int64_t o0 = static_cast<int64_t>(tile_o) * TILE_O, c0 = static_cast<int64_t>(tile_c) * TILE_C;
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t wave_o = wave / 2 * 64, wave_c = wave % 2 * 64;

    // what a thread brings: of dy four vectors of 8 columns, of q two of 16
    const uint32_t dy_col = threadIdx.x % 16 * 8, dy_row = threadIdx.x / 16;       // rows dy_row + 16 j
    const uint32_t q_col = threadIdx.x % 8 * 16, q_row = threadIdx.x / 8;          // rows q_row + 32 j
    const int dy_n = static_cast<int>(max(int64_t(0), min(A.outputs - o0 - dy_col, int64_t(VEC))));
    const bool q_here = c0 + q_col < A.ld;
    Raw8<DyT> dy[4];
    u32x4 q[2];
    auto fetch = [&](int64_t t0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t t = t0 + dy_row + 16 * j;
            dy[j] = load8(static_cast<const DyT*>(A.dy) + t * A.dy_stride + o0 + dy_col, t < A.tokens ? dy_n : 0);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t t = t0 + q_row + 32 * j;
            q[j] = u32x4{0, 0, 0, 0};
            if (q_here && t < A.tokens) q[j] = *reinterpret_cast<const u32x4*>(A.q + t * A.ld + c0 + q_col);
        }
    };
    auto put = [&] {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            Frag part[PARTS];
            split<DyT>(dy[j], part);
#pragma unroll
            for (int p = 0; p < PARTS; ++p) *reinterpret_cast<Frag*>(lds + p * TILE_BYTES + lds_at(dy_row + 16 * j, dy_col)) = part[p];
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                Frag x;
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    x[i] = static_cast<E>(static_cast<float>(static_cast<int32_t>(q[j][2 * h + i / 4]) << (24 - 8 * (i % 4)) >> 24));
                *reinterpret_cast<Frag*>(lds_x + lds_at(q_row + 32 * j, q_col + 8 * h)) = x;
            }
    };

    // where a lane reads: rows 8 (lane / 32) + (lane % 16) / 4, columns 16 (lane / 16 % 2) + 4 (lane % 4) of a 32-column piece
    const uint32_t r = lane / 32 * 8 + lane % 16 / 4, cc = lane / 16 % 2 * 16 + lane % 4 * 4;
    uint32_t at_o[2], at_c[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        at_o[f] = lds_at(r, wave_o + f * 32 + cc);
        at_c[f] = lds_at(r, wave_c + f * 32 + cc);
    }

    f32x16 total[2][2] = {};
    const uint32_t g_first = split_no * A.groups_per_split, g_end = min(g_first + A.groups_per_split, A.groups);
    if (g_first < g_end) fetch(static_cast<int64_t>(g_first) * GROUP);
    for (uint32_t g = g_first; g < g_end; ++g) {
        float scale[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const int64_t c = c0 + wave_c + f * 32 + lane % 32;
            scale[f] = c < A.channels ? A.scale[g * A.ld + c] : 0.f;
        }
        f32x16 sum[2][2] = {};
        for (int s = 0; s < GROUP / STEP; ++s) {
            const int64_t t0 = static_cast<int64_t>(g) * GROUP + s * STEP;
            if (t0 >= A.tokens) break;
            __syncthreads();
            put();
            __syncthreads();
            if (t0 + STEP < A.tokens && (s + 1 < GROUP / STEP || g + 1 < g_end)) fetch(t0 + STEP);
            const int turns = static_cast<int>(min(int64_t(STEP / 16), (A.tokens - t0 + 15) / 16));
#pragma unroll
            for (int k = 0; k < STEP / 16; ++k) {
                if (k >= turns) break;
                Frag x[2];
#pragma unroll
                for (int f = 0; f < 2; ++f) x[f] = read_fragment<Frag>(lds_x, at_c[f] + k * 16 * ROW_BYTES);
#pragma unroll
                for (int p = PARTS - 1; p >= 0; --p) {
                    Frag y[2];
#pragma unroll
                    for (int f = 0; f < 2; ++f) y[f] = read_fragment<Frag>(lds + p * TILE_BYTES, at_o[f] + k * 16 * ROW_BYTES);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 2; ++j) sum[i][j] = Mma<DyT>::mul(y[i], x[j], sum[i][j]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) total[i][j][e] = __builtin_fmaf(scale[j], sum[i][j][e], total[i][j][e]);
    }

    // element e of a lane: row 8 (e / 4) + 4 (lane / 32) + e % 4, column lane % 32
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t c = c0 + wave_c + j * 32 + lane % 32;
            if (c >= A.channels) continue;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int64_t o = o0 + wave_o + i * 32 + e / 4 * 8 + lane / 32 * 4 + e % 4;
                if (o >= A.outputs) continue;
                if (A.splits > 1) {
                    A.partial[(static_cast<int64_t>(split_no) * A.outputs + o) * A.channels_padded + c] = total[i][j][e];
                } else {
                    GradT* const w = static_cast<GradT*>(A.dw) + o * A.dw_stride + c;
                    const float had = A.accumulate ? static_cast<float>(*w) : 0.f;
                    *w = rounded<GradT>(total[i][j][e] + had);
                }
            }
        }
}

// The splits' sums, in order.
template <typename GradT> __global__ __launch_bounds__(THREADS) void linear_join_kernel(LinearArgs A) {
    const int64_t c = (static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x) * 4;
    if (c >= A.channels) return;
    for (int64_t o = blockIdx.y; o < A.outputs; o += gridDim.y) {
        f32x4 sum = *reinterpret_cast<const f32x4*>(A.partial + o * A.channels_padded + c);
#pragma unroll 4
        for (uint32_t s = 1; s < A.splits; ++s)
            sum += *reinterpret_cast<const f32x4*>(A.partial + (static_cast<int64_t>(s) * A.outputs + o) * A.channels_padded + c);
        GradT* const w = static_cast<GradT*>(A.dw) + o * A.dw_stride + c;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < A.channels) w[i] = rounded<GradT>(sum[i] + (A.accumulate ? static_cast<float>(w[i]) : 0.f));
    }
}

constexpr int BIAS_TOKENS = 256;       // tokens of a part

// Column sums of dy: 128 columns of 256 tokens by a workgroup.
template <typename DyT> __global__ __launch_bounds__(THREADS) void bias_kernel(LinearArgs A) {
    const uint32_t lane = threadIdx.x % 16, row = threadIdx.x / 16;
    const int64_t o = (static_cast<int64_t>(blockIdx.x) * 16 + lane) * VEC;
    const int n = static_cast<int>(max(int64_t(0), min(A.outputs - o, int64_t(VEC))));
    float sum[VEC] = {};
#pragma unroll 8
    for (int s = 0; s < BIAS_TOKENS / 16; ++s) {
        const int64_t t = static_cast<int64_t>(blockIdx.y) * BIAS_TOKENS + s * 16 + row;
        const Raw8<DyT> x = load8(static_cast<const DyT*>(A.dy) + t * A.dy_stride + o, t < A.tokens ? n : 0);
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] += get(x, i);
    }
    __shared__ float sums[16][16 * VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) sums[row][lane * VEC + i] = sum[i];
    __syncthreads();
    const int64_t out = static_cast<int64_t>(blockIdx.x) * 16 * VEC + threadIdx.x;
    if (threadIdx.x < 16 * VEC && out < A.outputs) {
        float all = 0.f;
        for (int w = 0; w < 16; ++w) all += sums[w][threadIdx.x];
        A.bias_partial[static_cast<int64_t>(blockIdx.y) * A.outputs + out] = all;
    }
}

template <typename GradT> __global__ __launch_bounds__(THREADS) void bias_join_kernel(LinearArgs A) {
    const int64_t o = static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x;
    if (o >= A.outputs) return;
    float sum = 0.f;
#pragma unroll 8
    for (uint32_t s = 0; s < A.bias_parts; ++s) sum += A.bias_partial[static_cast<int64_t>(s) * A.outputs + o];
    GradT* const b = static_cast<GradT*>(A.db) + o;
    *b = rounded<GradT>(sum + (A.accumulate ? static_cast<float>(*b) : 0.f));
}

struct LinearPlan {
    uint32_t tiles_o, tiles_c, groups, splits, groups_per_split, bias_parts;
    int64_t channels_padded, bias_at, bytes;
};

LinearPlan plan_of(int64_t tokens, int64_t channels, int64_t outputs) {
    LinearPlan p{};
    p.tiles_o = static_cast<uint32_t>(ceil_div(outputs, TILE_O));
    p.tiles_c = static_cast<uint32_t>(ceil_div(channels, TILE_C));
    p.groups = static_cast<uint32_t>(ceil_div(tokens, GROUP));
    const int64_t tiles = static_cast<int64_t>(p.tiles_o) * p.tiles_c;
    // enough workgroups for two on each of the 256 compute units, and two groups at the least for each of them
    int64_t splits = std::min<int64_t>({512 / std::max<int64_t>(tiles, 1), std::max<uint32_t>(p.groups / 2, 1), MAX_SPLITS});
    splits = std::max<int64_t>(splits, 1);
    p.groups_per_split = static_cast<uint32_t>(ceil_div(std::max<uint32_t>(p.groups, 1), splits));
    p.splits = static_cast<uint32_t>(ceil_div(std::max<uint32_t>(p.groups, 1), p.groups_per_split));
    p.channels_padded = ceil_div(channels, 4) * 4;
    p.bias_parts = static_cast<uint32_t>(ceil_div(std::max<int64_t>(tokens, 1), BIAS_TOKENS));
    const int64_t sums = p.splits > 1 ? p.splits * outputs * p.channels_padded * 4 : 0;
    p.bias_at = ceil_div(sums, 256) * 256;
    p.bytes = p.bias_at + p.bias_parts * outputs * 4;
    return p;
}

bool sizes_ok(int64_t tokens, int64_t channels, int64_t outputs) {
    return tokens >= 0 && tokens <= (int64_t(1) << 23) && channels >= 0 && channels <= (int64_t(1) << 23) && outputs >= 0 &&
           outputs <= (int64_t(1) << 23) && ceil_div(channels, TILE_C) * ceil_div(outputs, TILE_O) <= (int64_t(1) << 23);
}

}  // namespace

extern "C" {

int mgwfbp_act_linear_grad_workspace(int64_t n_tokens, int64_t n_channels, int64_t n_outputs, uint64_t* bytes_out) {
    if (bytes_out == nullptr || !sizes_ok(n_tokens, n_channels, n_outputs)) return MGWFBP_EINVAL;
    *bytes_out = static_cast<uint64_t>(plan_of(n_tokens, n_channels, n_outputs).bytes);
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
    const LinearPlan p = plan_of(n_tokens, n_channels, n_outputs);
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
    a.dw_stride = dw_stride;
    a.tokens = n_tokens;
    a.channels = n_channels;
    a.outputs = n_outputs;
    a.channels_padded = p.channels_padded;
    a.tiles_c = p.tiles_c;
    a.tiles = p.tiles_o * p.tiles_c;
    a.splits = p.splits;
    a.groups = p.groups;
    a.groups_per_split = p.groups_per_split;
    a.bias_parts = p.bias_parts;
    a.accumulate = accumulate != 0;
    return with_dtype(dy_dtype, [&](auto* dy_type) {
        return with_dtype(grad_dtype, [&](auto* grad_type) {
            typedef std::remove_pointer_t<decltype(dy_type)> DyT;
            typedef std::remove_pointer_t<decltype(grad_type)> GradT;
            int rc = MGWFBP_OK;
            if (n_channels > 0) rc = launch(linear_kernel<DyT, GradT>, a, dim3(a.tiles * a.splits), dim3(THREADS), hip_stream);
            if (rc == MGWFBP_OK && n_channels > 0 && a.splits > 1)
                rc = launch(linear_join_kernel<GradT>, a,
                            dim3(static_cast<uint32_t>(ceil_div(n_channels, 4 * THREADS)), static_cast<uint32_t>(std::min<int64_t>(n_outputs, 65535))),
                            dim3(THREADS), hip_stream);
            if (rc == MGWFBP_OK && d_db != nullptr)
                rc = launch(bias_kernel<DyT>, a, dim3(static_cast<uint32_t>(ceil_div(n_outputs, 16 * VEC)), a.bias_parts), dim3(THREADS), hip_stream);
            if (rc == MGWFBP_OK && d_db != nullptr)
                rc = launch(bias_join_kernel<GradT>, a, dim3(static_cast<uint32_t>(ceil_div(n_outputs, THREADS))), dim3(THREADS), hip_stream);
            return rc;
        });
    });
}

}  // extern "C"
