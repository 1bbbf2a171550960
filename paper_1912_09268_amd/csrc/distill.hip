// Loss of a language model's last layer, forward and backward in one pass: cross entropy with a label, and the divergence from a
// teacher that is known by its top logits.
//
//   p_j = exp(s_j / tau) / sum over the teacher's entries of a row;  q = softmax(z);  r = softmax(z / tau)
//   loss = w * (lw * (-log q[label]) + tw * tau^2 * sum over j of p_j (log p_j - log r[id_j]))
//   dz   = w * (lw * (q - [label]) + tw * tau * (r - sum over j of p_j [id_j]))
//
// A workgroup has a row.  It holds it as it is in memory between the largest value, the sums and the gradient, so z is read once
// and dz written once; rows that do not fit are read twice, with the largest value and the sums found together.  The few places
// with a label or an entry of the teacher are written once more behind the others: their z are taken up first (dz may lie over z),
// and an entry's place gets what all entries of that place have, so the same index twice in a row counts twice.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "device_types.h"
#include "mgwfbp_layers.h"

namespace {

using namespace ops;

constexpr float LOG2_E = 1.44269504088896341f;
constexpr int MOST_TOP = MGWFBP_MAX_TOP;

struct DistillArgs {
    const void* z;
    void* dz;
    const void* labels;
    const void* ids;
    const void* teacher;
    const float* row_weight;
    float* loss;
    int64_t z_stride, dz_stride, ids_stride, teacher_stride;
    int64_t tokens, vocabulary;
    float label_weight, teacher_weight, tau, over_tau;
    int32_t top, label_type, id_type, teacher_type;
};

__device__ __forceinline__ float number_at(const void* p, int32_t type, int64_t i) {
    if (type == MGWFBP_F32) return static_cast<const float*>(p)[i];
    if (type == MGWFBP_BF16) return static_cast<float>(static_cast<const __bf16*>(p)[i]);
    return static_cast<float>(static_cast<const _Float16*>(p)[i]);
}
// An index, -1 if it is none of the vocabulary's.
__device__ __forceinline__ int32_t id_at(const void* p, int32_t type, int64_t i, int64_t vocabulary) {
    const int64_t id = type == MGWFBP_I64 ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
    return id >= 0 && id < vocabulary ? static_cast<int32_t>(id) : -1;
}

template <int THREADS> __device__ __forceinline__ float workgroup_max(float x, float* room) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x = __builtin_fmaxf(x, __shfl_xor(x, d));
    if constexpr (THREADS == 64) return x;
    if (threadIdx.x % 64 == 0) room[threadIdx.x / 64] = x;
    __syncthreads();
    x = room[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) x = __builtin_fmaxf(x, room[w]);
    return x;
}
template <int THREADS, int N> __device__ __forceinline__ void workgroup_sums(float (&x)[N], float (*room)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int d = 32; d > 0; d /= 2) x[i] += __shfl_xor(x[i], d);
    if constexpr (THREADS == 64) return;
    if (threadIdx.x % 64 == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) room[threadIdx.x / 64][i] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = room[0][i];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) x[i] += room[w][i];
    }
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log_of(float x) { return __builtin_logf(x); }

// V vectors of eight elements a lane hold a row; V = 0: they do not.
template <typename T, int THREADS, int V> __global__ __launch_bounds__(THREADS) void distill_kernel(DistillArgs A) {
    __shared__ int32_t at_id[MOST_TOP + 1];                  // the teacher's entries and, behind them, the label
    __shared__ float at_z[MOST_TOP + 1], at_p[MOST_TOP + 1];
    __shared__ float room_max[2][THREADS / 64], room_sum[THREADS / 64][4];
    const int64_t t = blockIdx.x;
    const T* const z = static_cast<const T*>(A.z) + t * A.z_stride;
    T* const dz = static_cast<T*>(A.dz) + t * A.dz_stride;
    const int64_t first = static_cast<int64_t>(threadIdx.x) * VEC;
    constexpr int64_t STEP = THREADS * VEC;
    auto left = [&](int64_t col) { return static_cast<int>(max(static_cast<int64_t>(0), min(A.vocabulary - col, static_cast<int64_t>(VEC)))); };

    const float weight = A.row_weight == nullptr ? 1.f : A.row_weight[t];
    const int32_t label = A.labels == nullptr || A.label_weight == 0.f ? -1 : id_at(A.labels, A.label_type, t, A.vocabulary);
    const int top = A.teacher_weight == 0.f || weight == 0.f ? 0 : A.top;
    Raw8<T> x[V > 0 ? V : 1];
    if constexpr (V > 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = load8(z + first + v * STEP, weight != 0.f ? left(first + v * STEP) : 0);
    }
    // the teacher's entries: an index outside and a logit of -inf are no entry
    float best = -__builtin_inff();
    for (int j = threadIdx.x; j < top; j += THREADS) {
        int32_t id = id_at(A.ids, A.id_type, t * A.ids_stride + j, A.vocabulary);
        const float s = number_at(A.teacher, A.teacher_type, t * A.teacher_stride + j);
        if (s == -__builtin_inff()) id = -1;
        at_id[j] = id;
        at_p[j] = s;
        at_z[j] = id >= 0 ? static_cast<float>(z[id]) : 0.f;
        if (id >= 0) best = __builtin_fmaxf(best, s);       // a NaN is no maximum, but the sums have it
    }
    if (threadIdx.x == 0) {
        at_id[top] = label;
        at_z[top] = label >= 0 ? static_cast<float>(z[label]) : 0.f;
        at_p[top] = 0.f;
    }
    bool some = false;
    for (int j = threadIdx.x; j < top; j += THREADS) some |= at_id[j] >= 0;
    const bool taught = __syncthreads_or(some);
    if (weight == 0.f || (label < 0 && !taught)) {           // nothing is asked of this row
        if (threadIdx.x == 0) A.loss[t] = 0.f;
        if (A.dz != nullptr) {
            const float zero[VEC] = {};
            for (int64_t col = first; col < A.vocabulary; col += STEP) store8(dz + col, zero, left(col));
        }
        return;
    }
    best = workgroup_max<THREADS>(best, room_max[0]);

    // One softmax or two: where tau is 1 or only one part is asked for, one of them, with both weights.
    const bool both = label >= 0 && taught && A.tau != 1.f;
    const float c = label >= 0 || A.tau == 1.f ? LOG2_E : LOG2_E * A.over_tau, ct = LOG2_E * A.over_tau;
    float most = -__builtin_inff();
    float sums[4] = {};                                      // of exp z, exp z / tau, the teacher's exp, and its terms
    auto add = [&](const Raw8<T>& r, int n, float from) {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < n) {
                const float d = get(r, i) - from;
                sums[0] += exp2_of(d * c);
                if (both) sums[1] += exp2_of(d * ct);
            }
    };
    if constexpr (V > 0) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i < left(first + v * STEP)) most = __builtin_fmaxf(most, get(x[v], i));
        most = workgroup_max<THREADS>(most, room_max[1]);
#pragma unroll
        for (int v = 0; v < V; ++v) add(x[v], left(first + v * STEP), most);
    } else {
        for (int64_t col = first; col < A.vocabulary; col += STEP) {
            const int n = left(col);
            const Raw8<T> r = load8(z + col, n);
            float higher = most;
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i < n) higher = __builtin_fmaxf(higher, get(r, i));
            const float from = higher == -__builtin_inff() ? 0.f : higher;       // nothing but -inf so far: they add 0
            if (higher != most) {
                sums[0] *= exp2_of((most - from) * c);
                sums[1] *= exp2_of((most - from) * ct);
                most = higher;
            }
            add(r, n, from);
        }
        const float mine = most;
        most = workgroup_max<THREADS>(most, room_max[1]);
        if (mine != most) {
            const float d = mine - most;
            sums[0] *= exp2_of(d * c);
            sums[1] *= exp2_of(d * ct);
        }
    }
    for (int j = threadIdx.x; j < top; j += THREADS) {       // a lane's own entries
        if (at_id[j] < 0) {
            at_p[j] = 0.f;
            continue;
        }
        const float d = (at_p[j] - best) * A.over_tau, e = exp2_of(d * LOG2_E);
        at_p[j] = e;
        sums[2] += e;
        if (!(e == 0.f)) sums[3] += e * (d - (at_z[j] - most) * A.over_tau);
    }
    workgroup_sums<THREADS>(sums, room_sum);
    if (!both) sums[1] = sums[0];
    if (threadIdx.x == 0) {
        float loss = 0.f;
        if (label >= 0) loss = A.label_weight * (log_of(sums[0]) - (at_z[top] - most));
        if (taught) loss += A.teacher_weight * A.tau * A.tau * (sums[3] / sums[2] - log_of(sums[2]) + log_of(sums[1]));
        A.loss[t] = weight * loss;
    }
    if (A.dz == nullptr) return;
    const float by_label = label >= 0 ? weight * A.label_weight : 0.f, by_teacher = taught ? weight * A.teacher_weight * A.tau : 0.f;
    const float f = (both ? by_label : by_label + by_teacher) / sums[0], ft = both ? by_teacher / sums[1] : 0.f;
    auto slope = [&](float value) {
        const float d = value - most;
        float g = exp2_of(d * c) * f;
        if (both) g = __builtin_fmaf(exp2_of(d * ct), ft, g);
        return g;
    };
    auto put = [&](const Raw8<T>& r, int64_t col) {
        float g[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) g[i] = slope(get(r, i));
        store8(dz + col, g, left(col));
    };
    if constexpr (V > 0) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (first + v * STEP < A.vocabulary) put(x[v], first + v * STEP);
    } else {
        for (int64_t col = first; col < A.vocabulary; col += STEP) put(load8(z + col, left(col)), col);
    }
    __syncthreads();                                         // the places of entries are written again
    const float per_entry = by_teacher / sums[2];
    for (int j = threadIdx.x; j <= top; j += THREADS) {
        const int32_t id = at_id[j];
        if (id < 0) continue;
        float p = 0.f;
        for (int i = 0; i < top; ++i) p += at_id[i] == id ? at_p[i] : 0.f;
        float g = slope(at_z[j]);
        if (taught) g -= per_entry * p;
        if (id == label) g -= by_label;
        dz[id] = rounded<T>(g);
    }
}

bool side_ok(const void* p, int64_t rows, int64_t width, int64_t stride, int64_t bytes) { return p != nullptr && is_aligned(p, bytes) && is_matrix(rows, width, stride, bytes); }
bool ids_ok(int32_t type) { return type == MGWFBP_I32 || type == MGWFBP_I64; }

template <int T_, int V_> struct Shape { static constexpr int threads = T_, vecs = V_; };
template <typename T, typename F> int with_shape(int64_t vocabulary, F&& f) {
    constexpr bool WIDE = sizeof(T) == 4;
    if (vocabulary <= 512) return f(Shape<64, 1>());
    if (vocabulary <= 2048) return f(Shape<256, 1>());
    if (vocabulary <= 8192) return f(Shape<256, 4>());
    if (vocabulary <= 16384) return f(Shape<512, 4>());
    if (vocabulary <= 32768) return f(Shape<1024, 4>());
    if (vocabulary <= 65536) return f(Shape<1024, 8>());
    if constexpr (!WIDE)
        if (vocabulary <= 131072) return f(Shape<1024, 16>());
    return f(Shape<1024, 0>());
}

}  // namespace

extern "C" {

int mgwfbp_distill(const void* d_z, int64_t z_stride, int32_t dtype, int64_t n_tokens, int64_t n_vocabulary, const void* d_labels, int32_t label_type,
                   const void* d_ids, int64_t ids_stride, int32_t id_type, const void* d_teacher, int64_t teacher_stride, int32_t teacher_dtype, int32_t n_top,
                   float temperature, float label_weight, float teacher_weight, const float* d_row_weight, float* d_loss, void* d_dz, int64_t dz_stride,
                   void* hip_stream) {
    if (!is_dtype(dtype) || n_tokens < 0 || n_tokens > (int64_t(1) << 26) || n_vocabulary < 1 || n_vocabulary > (int64_t(1) << 23)) return MGWFBP_EINVAL;
    if (n_top < 0 || n_top > MOST_TOP || !(temperature >= 0x1p-20f && temperature <= 0x1p20f) || !std::isfinite(label_weight) || !std::isfinite(teacher_weight))
        return MGWFBP_EINVAL;
    if (n_top > 0 && (!ids_ok(id_type) || !is_dtype(teacher_dtype))) return MGWFBP_EINVAL;
    if (d_labels != nullptr && (!ids_ok(label_type) || !is_aligned(d_labels, label_type == MGWFBP_I64 ? 8 : 4))) return MGWFBP_EINVAL;
    if (n_tokens == 0) return MGWFBP_OK;
    const int64_t bytes = dtype_bytes(dtype);
    if (!side_ok(d_z, n_tokens, n_vocabulary, z_stride, bytes) || (d_dz != nullptr && !side_ok(d_dz, n_tokens, n_vocabulary, dz_stride, bytes)) ||
        d_loss == nullptr || !is_aligned(d_loss, 4) || !is_aligned(d_row_weight, 4))
        return MGWFBP_EINVAL;
    if (n_top > 0 && (!side_ok(d_ids, n_tokens, n_top, ids_stride, id_type == MGWFBP_I64 ? 8 : 4) ||
                      !side_ok(d_teacher, n_tokens, n_top, teacher_stride, dtype_bytes(teacher_dtype))))
        return MGWFBP_EINVAL;
    DistillArgs a{};
    a.z = d_z;
    a.dz = d_dz;
    a.labels = d_labels;
    a.ids = d_ids;
    a.teacher = d_teacher;
    a.row_weight = d_row_weight;
    a.loss = d_loss;
    a.z_stride = z_stride;
    a.dz_stride = dz_stride;
    a.ids_stride = ids_stride;
    a.teacher_stride = teacher_stride;
    a.tokens = n_tokens;
    a.vocabulary = n_vocabulary;
    a.label_weight = label_weight;
    a.teacher_weight = teacher_weight;
    a.tau = temperature;
    a.over_tau = 1.f / temperature;
    a.top = n_top;
    a.label_type = label_type;
    a.id_type = id_type;
    a.teacher_type = teacher_dtype;
    return with_dtype(dtype, [&](auto* type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        return with_shape<T>(n_vocabulary, [&](auto s) {
            constexpr int THREADS = decltype(s)::threads;
            void (*kernel)(DistillArgs) = distill_kernel<T, THREADS, decltype(s)::vecs>;
            return launch(kernel, a, dim3(static_cast<uint32_t>(n_tokens)), dim3(THREADS), hip_stream);
        });
    });
}

}  // extern "C"
