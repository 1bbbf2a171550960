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
#include "spans.h"
#include "teams.h"

namespace {

using namespace ops;

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

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
    float* stats;                        // [tokens][parts][3]: of a row's part, its largest value and its sums of exp z and exp z / tau
    float* kept_z;                       // [tokens][kept_stride]: z of the teacher's entries and of the label
    int64_t z_stride, dz_stride, ids_stride, teacher_stride, kept_stride, parts;
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

// Over the lanes of a workgroup, in every lane: the largest of each of N numbers, or the sum.  `room` is used once.
template <int THREADS, int N, typename F> __device__ __forceinline__ void workgroup_all(float (&x)[N], float (*room)[N], F&& join) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = lanes_all<64>(x[i], join);
    if constexpr (THREADS > 64) {
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) room[threadIdx.x / 64][i] = x[i];
        __syncthreads();
        // sixteen lanes take a wavefront's each
        constexpr int WAVES = THREADS / 64;
        const int w = threadIdx.x % WAVES;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = lanes_all<WAVES>(room[w][i], join);
        }
    }
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log_of(float x) { return __builtin_logf(x); }

// The label's place behind the teacher's entries: the next multiple of four.
__host__ __device__ constexpr int label_place(int top) { return (top + 3) / 4 * 4; }

// The teacher's entries of a row and its label in LDS, as much as there are.  Entry j belongs to lane j % THREADS from beginning to end.
template <int THREADS> struct Entries {
    int32_t* id;                                             // -1: none
    float* p;                                                // the teacher's logit, and exp of it later
    float* z;
    uint8_t* again;                                          // another entry has the same index
    static __host__ __device__ constexpr int bytes(int top) { return (label_place(top) + 4) * (3 * 4 + 1); }
    __device__ __forceinline__ explicit Entries(int top) {
        extern __shared__ __attribute__((aligned(16))) int32_t memory[];
        const int room = label_place(top) + 4;               // so that all begin on 16 bytes
        id = memory;
        p = reinterpret_cast<float*>(memory + room);
        z = p + room;
        again = reinterpret_cast<uint8_t*>(z + room);
    }
    // One lane: the places between the entries and the label, and the label.
    __device__ __forceinline__ void close(int top, int32_t label) {
        const int end = label_place(top);
        for (int j = top; j < end; ++j) id[j] = -1;
        id[end] = label;
        p[end] = 0.f;
    }
    // After a barrier: whether an entry's index is another one's, too.  Nearly none is.  A workgroup of one wavefront has had none yet (its reductions
    // need no LDS), and what other lanes have put into LDS is seen behind one only.
    __device__ __forceinline__ void find_again(int top) {
        if constexpr (THREADS == 64) __syncthreads();
        const int end = label_place(top);
        for (int j = threadIdx.x; j <= end; j += THREADS) {
            const int32_t mine = id[j];
            int same = j == end;
            if (mine >= 0) {
#pragma unroll 4
                for (int i = 0; i < end; i += 4) {
                    const i32x4 four = *reinterpret_cast<const i32x4*>(id + i);
                    same += (four[0] == mine) + (four[1] == mine) + (four[2] == mine) + (four[3] == mine);
                }
            }
            again[j] = same > 1;
        }
    }
    // What all entries of one's index have together, in their order.
    __device__ __forceinline__ float together(int j, int top) const {
        if (!again[j]) return p[j];
        const int32_t mine = id[j];
        float sum = 0.f;
        for (int i = 0; i < top; i += 4) {
            const i32x4 four = *reinterpret_cast<const i32x4*>(id + i);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (four[k] == mine) sum += p[i + k];
        }
        return sum;
    }
};

// What is asked of a row, and its softmaxes: one or two of them; where tau is 1 or only one part is asked for, one, with both weights.
struct Asked {
    float weight, c, ct;
    int32_t label;
    bool taught, both;
    __device__ __forceinline__ void settle(const DistillArgs& A, bool taught_) {
        taught = taught_;
        both = label >= 0 && taught && A.tau != 1.f;
        c = label >= 0 || A.tau == 1.f ? LOG2_E : LOG2_E * A.over_tau;
        ct = LOG2_E * A.over_tau;
    }
};

// sums: of exp z, exp z / tau, the teacher's exp and its terms -> the loss
__device__ __forceinline__ float loss_of(const DistillArgs& A, const Asked& row, const float (&sums)[4], float below) {
    float loss = 0.f;
    if (row.label >= 0) loss = A.label_weight * (log_of(sums[0]) + below);
    if (row.taught) loss += A.teacher_weight * A.tau * A.tau * (sums[3] / sums[2] - log_of(sums[2]) + log_of(sums[1]));
    return row.weight * loss;
}

// The gradient of a logit, but for the label and the teacher's entries.
struct Slope {
    float high, c, ct, f, ft, by_label, per_entry;
    bool both;
    __device__ __forceinline__ Slope(const DistillArgs& A, const Asked& row, const float (&sums)[4], float high_) : high(high_), c(row.c), ct(row.ct), both(row.both) {
        by_label = row.label >= 0 ? row.weight * A.label_weight : 0.f;
        const float by_teacher = row.taught ? row.weight * A.teacher_weight * A.tau : 0.f;
        f = (both ? by_label : by_label + by_teacher) / sums[0];
        ft = both ? by_teacher / sums[1] : 0.f;
        per_entry = row.taught ? by_teacher / sums[2] : 0.f;
    }
    __device__ __forceinline__ float operator()(float value) const {
        const float d = value - high;
        const float g = exp2_of(d * c) * f;
        return both ? __builtin_fmaf(exp2_of(d * ct), ft, g) : g;
    }
    template <typename T> __device__ __forceinline__ void of(const Raw8<T>& r, float (&g)[VEC]) const {
        if (both) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float d = get(r, i) - high;
                g[i] = __builtin_fmaf(exp2_of(d * ct), ft, exp2_of(d * c) * f);
            }
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) g[i] = exp2_of((get(r, i) - high) * c) * f;
        }
    }
};

// exp of the teacher's entries and their terms, a lane's own ones.
template <int THREADS> __device__ __forceinline__ void teach(const DistillArgs& A, Entries<THREADS>& at, int top, float best, float high, float& sum, float& terms) {
    for (int j = threadIdx.x; j < top; j += THREADS) {
        if (at.id[j] < 0) {
            at.p[j] = 0.f;
            continue;
        }
        const float d = (at.p[j] - best) * A.over_tau, e = exp2_of(d * LOG2_E);
        at.p[j] = e;
        sum += e;
        if (!(e == 0.f)) terms += e * (d - (at.z[j] - high) * A.over_tau);
    }
}

// The elements i, from <= i < VEC, of eight.
template <typename T> __device__ __forceinline__ void add(const Raw8<T>& r, int from, float high, const Asked& row, float (&sums)[4]) {
    if (row.both) {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i >= from) {
                const float d = get(r, i) - high;
                sums[0] += exp2_of(d * row.c);
                sums[1] += exp2_of(d * row.ct);
            }
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i >= from) sums[0] += exp2_of((get(r, i) - high) * row.c);
    }
}

constexpr int AHEAD = 4;                 // vectors of a lane on their way where a row does not stay in registers

// V vectors of eight elements a lane hold a row of eight elements or more; V = 0: they do not.  Bound by memory, and by the exponentials where there are two
// softmaxes: 4096 rows of 30522 bfloat16 logits, 500 MB, with labels alone 94 us, 5.3 TB/s, with labels and 64 entries at another temperature 104; 129 rows of 100003
// binary32 logits, too long for registers, 31 us, 3.3 TB/s (4.9 counting both readings), as long as the last of them.
//
// The last vector of a row that is no multiple of eight begins before its place, so that it ends with the row; lanes behind it take it, too.
// What they have in common with the lane before is neither summed twice nor, being the same, wrong where it is written twice.
template <typename T, int THREADS, int V, int PER_SIMD> __global__ __launch_bounds__(THREADS, PER_SIMD) void distill_kernel(DistillArgs A) {
    __shared__ float room[THREADS / 64][3], room_sums[THREADS / 64][4];
    Entries<THREADS> at(A.top);
    const int64_t t = blockIdx.x;
    const T* const z = static_cast<const T*>(A.z) + t * A.z_stride;
    T* const dz = static_cast<T*>(A.dz) + t * A.dz_stride;
    const uint32_t vocabulary = static_cast<uint32_t>(A.vocabulary), first = threadIdx.x * VEC, last = vocabulary - VEC;
    constexpr uint32_t STEP = THREADS * VEC;
    constexpr int HELD = V > 0 ? V : AHEAD;

    Asked row;
    row.weight = A.row_weight == nullptr ? 1.f : A.row_weight[t];
    row.label = A.labels == nullptr || A.label_weight == 0.f ? -1 : id_at(A.labels, A.label_type, t, A.vocabulary);
    const int top = A.teacher_weight == 0.f || row.weight == 0.f ? 0 : A.top;
    // a lane's first entry is asked for before the row and its z behind it, so that neither waits
    const float LEAST = -__builtin_inff();
    const bool entry = static_cast<int>(threadIdx.x) < top;
    int32_t id = -1;
    float s = LEAST;
    if (entry) {
        id = id_at(A.ids, A.id_type, t * A.ids_stride + threadIdx.x, A.vocabulary);
        s = number_at(A.teacher, A.teacher_type, t * A.teacher_stride + threadIdx.x);
    }
    Raw8<T> x[HELD];
    if (row.weight != 0.f) {
#pragma unroll
        for (int v = 0; v < HELD; ++v) x[v] = load8(z + min(first + v * STEP, last));
    }
    float most[3] = {LEAST, LEAST, 0.f};                     // of the row, of the teacher's entries, and whether there are any
    auto enter = [&](int j, int32_t id, float s) {           // an index outside and a logit of -inf are no entry
        at.id[j] = id;
        at.p[j] = s;
        if (id >= 0) {
            most[1] = __builtin_fmaxf(most[1], s);           // a NaN is no maximum, but the sums have it
            most[2] = 1.f;
        }
    };
    if (s == LEAST) id = -1;
    float z_entry = 0.f;
    if (entry) {
        enter(threadIdx.x, id, s);
        if (id >= 0) z_entry = static_cast<float>(z[id]);
    }
    for (int j = threadIdx.x + THREADS; j < top; j += THREADS) {
        int32_t more = id_at(A.ids, A.id_type, t * A.ids_stride + j, A.vocabulary);
        const float logit = number_at(A.teacher, A.teacher_type, t * A.teacher_stride + j);
        if (logit == LEAST) more = -1;
        enter(j, more, logit);
        at.z[j] = more >= 0 ? static_cast<float>(z[more]) : 0.f;
    }
    float z_label = 0.f;
    const int place_of_label = label_place(top);
    const bool labelled = static_cast<int>(threadIdx.x) == place_of_label % THREADS;         // the lane of the label's place
    if (labelled) at.close(top, row.label);
    if (labelled && row.label >= 0) z_label = static_cast<float>(z[row.label]);
    if constexpr (V > 0) {
        if (row.weight != 0.f) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < VEC; ++i) most[0] = __builtin_fmaxf(most[0], get(x[v], i));
        }
    }
    workgroup_all<THREADS>(most, room, [](float a, float b) { return __builtin_fmaxf(a, b); });
    row.settle(A, most[2] != 0.f);
    if (row.weight == 0.f || (row.label < 0 && !row.taught)) {                  // nothing is asked of this row
        if (threadIdx.x == 0) A.loss[t] = 0.f;
        if (A.dz != nullptr) {
            const float zero[VEC] = {};
            for (uint32_t col = first; col < vocabulary; col += STEP) store8(dz + min(col, last), zero);
        }
        return;
    }
    if (entry) at.z[threadIdx.x] = z_entry;
    if (labelled) at.z[place_of_label] = z_label;
    at.find_again(top);
    float high = most[0], sums[4] = {};
    if constexpr (V > 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t col = first + v * STEP;
            if (col <= last) add(x[v], 0, high, row, sums);
            else if (col < vocabulary) add(x[v], static_cast<int>(col - last), high, row, sums);
        }
    } else {
        float mine = LEAST;
        for (uint32_t base = first; base < vocabulary; base += AHEAD * STEP) {
            Raw8<T> now[AHEAD];
#pragma unroll
            for (int v = 0; v < AHEAD; ++v) now[v] = x[v];
#pragma unroll
            for (int v = 0; v < AHEAD; ++v) x[v] = load8(z + min(base + (AHEAD + v) * STEP, last));
            float higher = mine;                             // a vector taken twice does no harm here
#pragma unroll
            for (int v = 0; v < AHEAD; ++v)
#pragma unroll
                for (int i = 0; i < VEC; ++i) higher = __builtin_fmaxf(higher, get(now[v], i));
            const float origin = higher == LEAST ? 0.f : higher;                 // nothing but -inf so far: they add 0
            if (higher != mine) {
                sums[0] *= exp2_of((mine - origin) * row.c);
                sums[1] *= exp2_of((mine - origin) * row.ct);
                mine = higher;
            }
#pragma unroll
            for (int v = 0; v < AHEAD; ++v) {
                const uint32_t col = base + v * STEP;
                if (col <= last) add(now[v], 0, origin, row, sums);
                else if (col < vocabulary) add(now[v], static_cast<int>(col - last), origin, row, sums);
            }
        }
        float all[1] = {mine};
        __shared__ float room_high[THREADS / 64][1];
        workgroup_all<THREADS>(all, room_high, [](float a, float b) { return __builtin_fmaxf(a, b); });
        high = all[0];
        if (mine != high) {
            sums[0] *= exp2_of((mine - high) * row.c);
            sums[1] *= exp2_of((mine - high) * row.ct);
        }
    }
    teach(A, at, top, most[1], high, sums[2], sums[3]);
    workgroup_all<THREADS>(sums, room_sums, [](float a, float b) { return a + b; });
    if (!row.both) sums[1] = sums[0];
    if (labelled) A.loss[t] = loss_of(A, row, sums, high - at.z[place_of_label]);
    if (A.dz == nullptr) return;
    const Slope slope(A, row, sums, high);
    float g[VEC];
    if constexpr (V > 0) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (first + v * STEP < vocabulary) {
                slope.of(x[v], g);
                store8(dz + min(first + v * STEP, last), g);
            }
    } else {
        // From behind: what was read last is nearest.  dz may be z: a lane's vectors are on their way before it writes those ahead of them, and
        // what two lanes have in common is written by the first of them alone.
        const uint32_t turns = (vocabulary + AHEAD * STEP - 1) / (AHEAD * STEP);
#pragma unroll
        for (int v = 0; v < AHEAD; ++v) x[v] = load8(z + min(first + ((turns - 1) * AHEAD + v) * STEP, last));
        for (uint32_t turn = turns; turn-- > 0;) {
            Raw8<T> now[AHEAD];
#pragma unroll
            for (int v = 0; v < AHEAD; ++v) now[v] = x[v];
            if (turn > 0) {
#pragma unroll
                for (int v = 0; v < AHEAD; ++v) x[v] = load8(z + min(first + ((turn - 1) * AHEAD + v) * STEP, last));
            }
#pragma unroll
            for (int v = 0; v < AHEAD; ++v) {
                const uint32_t col = first + (turn * AHEAD + v) * STEP;
                if (col >= vocabulary) continue;
                slope.of(now[v], g);
                if (col <= last) {
                    store8(dz + col, g);
                } else {
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        if (i >= static_cast<int>(col - last)) dz[last + i] = rounded<T>(g[i]);
                }
            }
        }
    }
    __syncthreads();                                         // the places of entries are written again
    for (int j = threadIdx.x; j <= place_of_label; j += THREADS) {
        const int32_t place = at.id[j];
        if (place >= 0) dz[place] = rounded<T>(slope(at.z[j]) - slope.per_entry * at.together(j, top) - (place == row.label ? slope.by_label : 0.f));
    }
}

// Few rows: each in parts of 256 lanes times V vectors.  First every part's largest value and sums, and the z of the row's entries, since dz may
// be z ...
constexpr int PART = 256;
template <typename T, int V> __global__ __launch_bounds__(PART) void part_kernel(DistillArgs A) {
    __shared__ float room[PART / 64][1], room_sums[PART / 64][2];
    const int64_t t = blockIdx.y;
    const T* const z = static_cast<const T*>(A.z) + t * A.z_stride;
    const uint32_t vocabulary = static_cast<uint32_t>(A.vocabulary), last = vocabulary - VEC, first = blockIdx.x * (PART * VEC * V) + threadIdx.x * VEC;
    Raw8<T> x[V];
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = load8(z + min(first + v * (PART * VEC), last));
    if (blockIdx.x == 0) {
        float* const kept = A.kept_z + t * A.kept_stride;
        for (int j = threadIdx.x; j < A.top; j += PART) {
            const int32_t id = id_at(A.ids, A.id_type, t * A.ids_stride + j, A.vocabulary);
            kept[j] = id >= 0 ? static_cast<float>(z[id]) : 0.f;
        }
        if (threadIdx.x == 0 && A.labels != nullptr) {
            const int32_t label = id_at(A.labels, A.label_type, t, A.vocabulary);
            kept[label_place(A.top)] = label >= 0 ? static_cast<float>(z[label]) : 0.f;
        }
    }
    float high[1] = {-__builtin_inff()}, sums[2] = {};
    // lanes behind the row take its last vector, which may be another part's, too: an origin that is larger than need be does no harm
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < VEC; ++i) high[0] = __builtin_fmaxf(high[0], get(x[v], i));
    workgroup_all<PART>(high, room, [](float a, float b) { return __builtin_fmaxf(a, b); });
    const float origin = high[0] == -__builtin_inff() ? 0.f : high[0], c = LOG2_E, ct = LOG2_E * A.over_tau;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const uint32_t col = first + v * (PART * VEC);
        const int from = col <= last ? 0 : col < vocabulary ? static_cast<int>(col - last) : VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i >= from) {
                const float d = get(x[v], i) - origin;
                sums[0] += exp2_of(d * c);
                if (A.tau != 1.f) sums[1] += exp2_of(d * ct);
            }
    }
    workgroup_all<PART>(sums, room_sums, [](float a, float b) { return a + b; });
    if (threadIdx.x == 0) {
        float* const to = A.stats + (t * gridDim.x + blockIdx.x) * 3;
        to[0] = high[0];
        to[1] = sums[0];
        to[2] = A.tau != 1.f ? sums[1] : sums[0];
    }
}

// ... then the row's, from all parts', and the gradient.
template <typename T, int V> __global__ __launch_bounds__(PART) void part_slope_kernel(DistillArgs A) {
    __shared__ float room[PART / 64][3], room_sums[PART / 64][4];
    Entries<PART> at(A.top);
    const int64_t t = blockIdx.y;
    const T* const z = static_cast<const T*>(A.z) + t * A.z_stride;
    T* const dz = static_cast<T*>(A.dz) + t * A.dz_stride;
    const uint32_t vocabulary = static_cast<uint32_t>(A.vocabulary), last = vocabulary - VEC, begin = blockIdx.x * (PART * VEC * V), first = begin + threadIdx.x * VEC;
    Asked row;
    row.weight = A.row_weight == nullptr ? 1.f : A.row_weight[t];
    row.label = A.labels == nullptr || A.label_weight == 0.f ? -1 : id_at(A.labels, A.label_type, t, A.vocabulary);
    const int top = A.teacher_weight == 0.f || row.weight == 0.f ? 0 : A.top, place_of_label = label_place(top);
    const float LEAST = -__builtin_inff();
    const float *const kept = A.kept_z + t * A.kept_stride, *const stats = A.stats + t * A.parts * 3;
    Raw8<T> x[V];
    if (A.dz != nullptr && row.weight != 0.f) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = load8(z + min(first + v * (PART * VEC), last));
    }
    float most[3] = {LEAST, LEAST, 0.f};
    for (int j = threadIdx.x; j < top; j += PART) {
        int32_t id = id_at(A.ids, A.id_type, t * A.ids_stride + j, A.vocabulary);
        const float s = number_at(A.teacher, A.teacher_type, t * A.teacher_stride + j);
        if (s == LEAST) id = -1;
        at.id[j] = id;
        at.p[j] = s;
        at.z[j] = kept[j];
        if (id >= 0) {
            most[1] = __builtin_fmaxf(most[1], s);
            most[2] = 1.f;
        }
    }
    if (static_cast<int>(threadIdx.x) == place_of_label % PART) {
        at.close(top, row.label);
        at.z[place_of_label] = row.label >= 0 ? kept[label_place(A.top)] : 0.f;
    }
    for (int p = threadIdx.x; p < A.parts; p += PART) most[0] = __builtin_fmaxf(most[0], stats[p * 3]);
    workgroup_all<PART>(most, room, [](float a, float b) { return __builtin_fmaxf(a, b); });
    row.settle(A, most[2] != 0.f);
    float g[VEC] = {};
    if (row.weight == 0.f || (row.label < 0 && !row.taught)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) A.loss[t] = 0.f;
        if (A.dz != nullptr) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (first + v * (PART * VEC) < vocabulary) store8(dz + min(first + v * (PART * VEC), last), g);
        }
        return;
    }
    at.find_again(top);
    const float high = most[0];
    float sums[4] = {};
    for (int p = threadIdx.x; p < A.parts; p += PART) {
        const float d = stats[p * 3] - high;
        if (row.label >= 0 || A.tau == 1.f) sums[0] += stats[p * 3 + 1] * exp2_of(d * LOG2_E);
        else sums[0] += stats[p * 3 + 2] * exp2_of(d * row.ct);
        sums[1] += stats[p * 3 + 2] * exp2_of(d * row.ct);
    }
    teach(A, at, top, most[1], high, sums[2], sums[3]);
    workgroup_all<PART>(sums, room_sums, [](float a, float b) { return a + b; });
    if (!row.both) sums[1] = sums[0];
    if (blockIdx.x == 0 && static_cast<int>(threadIdx.x) == place_of_label % PART) A.loss[t] = loss_of(A, row, sums, high - at.z[place_of_label]);
    if (A.dz == nullptr) return;
    const Slope slope(A, row, sums, high);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const uint32_t col = first + v * (PART * VEC);
        if (col >= vocabulary) continue;
        slope.of(x[v], g);
        if (col <= last) {
            store8(dz + col, g);
        } else {                                             // dz may be z, and what lies before is another part's
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i >= static_cast<int>(col - last)) dz[last + i] = rounded<T>(g[i]);
        }
    }
    __syncthreads();
    const uint32_t end = begin + PART * VEC * V;
    for (int j = threadIdx.x; j <= place_of_label; j += PART) {
        const int32_t place = at.id[j];
        if (place >= 0 && static_cast<uint32_t>(place) >= begin && static_cast<uint32_t>(place) < end)
            dz[place] = rounded<T>(slope(at.z[j]) - slope.per_entry * at.together(j, top) - (place == row.label ? slope.by_label : 0.f));
    }
}

// Vocabularies of fewer than eight logits: a lane for a row.
template <typename T> __global__ __launch_bounds__(64) void tiny_kernel(DistillArgs A) {
    const int64_t t = static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x;
    if (t >= A.tokens) return;
    const T* const z = static_cast<const T*>(A.z) + t * A.z_stride;
    T* const dz = static_cast<T*>(A.dz) + t * A.dz_stride;
    const int vocabulary = static_cast<int>(A.vocabulary);
    Asked row;
    row.weight = A.row_weight == nullptr ? 1.f : A.row_weight[t];
    row.label = A.labels == nullptr || A.label_weight == 0.f ? -1 : id_at(A.labels, A.label_type, t, A.vocabulary);
    const int top = A.teacher_weight == 0.f || row.weight == 0.f ? 0 : A.top;
    const float LEAST = -__builtin_inff();
    auto entry = [&](int j, float& s) {
        const int32_t id = id_at(A.ids, A.id_type, t * A.ids_stride + j, A.vocabulary);
        s = number_at(A.teacher, A.teacher_type, t * A.teacher_stride + j);
        return s == LEAST ? -1 : id;
    };
    float best = LEAST, high = LEAST, s, value[VEC] = {}, share[VEC] = {}, sums[4] = {}, g[VEC] = {};
    bool taught = false;
    for (int j = 0; j < top; ++j)
        if (entry(j, s) >= 0) {
            taught = true;
            best = __builtin_fmaxf(best, s);
        }
    row.settle(A, taught);
    const bool asked = row.weight != 0.f && (row.label >= 0 || taught);
    A.loss[t] = 0.f;
    if (asked) {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < vocabulary) {
                value[i] = static_cast<float>(z[i]);
                high = __builtin_fmaxf(high, value[i]);
            }
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < vocabulary) {
                sums[0] += exp2_of((value[i] - high) * row.c);
                sums[1] += exp2_of((value[i] - high) * row.ct);
            }
        for (int j = 0; j < top; ++j) {
            const int32_t id = entry(j, s);
            if (id < 0) continue;
            const float d = (s - best) * A.over_tau, e = exp2_of(d * LOG2_E);
            sums[2] += e;
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i == id) {
                    share[i] += e;
                    if (!(e == 0.f)) sums[3] += e * (d - (value[i] - high) * A.over_tau);
                }
        }
        if (!row.both) sums[1] = sums[0];
        float below = 0.f;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i == row.label) below = high - value[i];
        A.loss[t] = loss_of(A, row, sums, below);
        const Slope slope(A, row, sums, high);
#pragma unroll
        for (int i = 0; i < VEC; ++i) g[i] = slope(value[i]) - (taught ? slope.per_entry * share[i] : 0.f) - (i == row.label ? slope.by_label : 0.f);
    }
    if (A.dz != nullptr) store8(dz, g, vocabulary);
}

bool side_ok(const void* p, int64_t rows, int64_t width, int64_t stride, int64_t bytes) { return p != nullptr && is_aligned(p, bytes) && is_matrix(rows, width, stride, bytes); }
bool ids_ok(int32_t type) { return type == MGWFBP_I32 || type == MGWFBP_I64; }

// Lanes and vectors of a lane for a row, and wavefronts a SIMD.  Few lanes with many vectors have fewer barriers and joins, many lanes with few have
// registers for more rows at once.  Us, bfloat16, labels and 32 entries unless said otherwise, the other shape behind the one taken:
//   16384 rows of 512 logits            64 x 1    20    256 x 1     45
//   16384 rows of 2048 logits           64 x 4    38    256 x 1     56      labels alone 28, 38; 128 entries, 2000 rows: 26, 16
//   8192 rows of 8192 logits           256 x 4    59    1024 x 1    97
//   4096 rows of 16384 logits          512 x 4    60    1024 x 2    75
//   4096 rows of 30522 logits          512 x 8   106    1024 x 4   113      labels alone 106, 94, so theirs is the other; binary32 199, 194
//   2048 rows of 50001 logits         1024 x 8   105    re-read    157
//   1024 rows of 100003 logits        1024 x 16  132    re-read    137      (of 131072: 151, 145)
template <int T_, int V_, int P_> struct Shape { static constexpr int threads = T_, vecs = V_, per_simd = P_; };
template <typename T, typename F> int with_shape(int64_t vocabulary, int32_t top, bool both, F&& f) {
    constexpr bool WIDE = sizeof(T) == 4;
    if (vocabulary <= 512) return f(Shape<64, 1, 8>());
    if (vocabulary <= 2048 && top <= 64) return f(Shape<64, 4, WIDE ? 6 : 8>());
    if (vocabulary <= 2048) return f(Shape<256, 1, 8>());
    if (vocabulary <= 8192) return f(Shape<256, 4, WIDE ? 6 : 8>());
    if (vocabulary <= 16384) return f(Shape<512, 4, WIDE ? 6 : 8>());
    if constexpr (!WIDE)
        if (both && vocabulary <= 32768) return f(Shape<512, 8, 4>());
    if (vocabulary <= 32768) return f(Shape<1024, 4, WIDE ? 4 : 8>());
    if (vocabulary <= 65536) return f(Shape<1024, 8, WIDE ? 4 : 8>());
    if constexpr (!WIDE)
        if (vocabulary <= 131072) return f(Shape<1024, 16, 4>());
    return f(Shape<1024, 0, 4>());
}

// Rows are cut where there are few and they are long: whole and in parts, us, bfloat16 with labels and teacher: 1 row of 30522 logits 9.2 and 9.0, of
// 131072 24.8 and 9.0; 64 rows of 50001 16.6 and 13.0, of 131072 29.0 and 18.7; 129 rows of 50001 17.6 and 17.5, of 131072 32.2 and 28.6; binary32: 64 rows of
// 65536 18.2 and 17.2, of 100003 29.6 and 20.5, 129 of 131072 44.9 and 55.0.
constexpr int64_t MOST_FEW = 100, FEW_LOGITS = 32768;

// How few rows are cut into parts: how many, and of how many vectors a lane; 0 where rows are not cut.
struct Cut {
    int64_t parts, vecs;
};
Cut cut_of(int64_t tokens, int64_t vocabulary) {
    if (tokens > std::min(MOST_FEW, vocabulary / 1024) || vocabulary <= FEW_LOGITS) return {0, 0};
    Cut c{0, 1};
    while (c.vecs < 8 && tokens * ceil_div(vocabulary, PART * VEC * c.vecs) > 1024) c.vecs *= 2;
    c.parts = ceil_div(vocabulary, PART * VEC * c.vecs);
    return c;
}
uint64_t workspace_of(int64_t tokens, int64_t vocabulary, int32_t top) {
    const Cut c = cut_of(tokens, vocabulary);
    return c.parts == 0 ? 0 : static_cast<uint64_t>(tokens * (c.parts * 3 + label_place(top) + 1)) * 4;
}

}  // namespace

extern "C" {

int mgwfbp_distill_workspace(int64_t n_tokens, int64_t n_vocabulary, int32_t n_top, uint64_t* bytes_out) {
    if (n_tokens < 0 || n_tokens > (int64_t(1) << 26) || n_vocabulary < 1 || n_vocabulary > (int64_t(1) << 23) || n_top < 0 || n_top > MOST_TOP ||
        bytes_out == nullptr)
        return MGWFBP_EINVAL;
    *bytes_out = n_tokens == 0 ? 0 : workspace_of(n_tokens, n_vocabulary, n_top);
    return MGWFBP_OK;
}

int mgwfbp_distill(const void* d_z, int64_t z_stride, int32_t dtype, int64_t n_tokens, int64_t n_vocabulary, const void* d_labels, int32_t label_type,
                   const void* d_ids, int64_t ids_stride, int32_t id_type, const void* d_teacher, int64_t teacher_stride, int32_t teacher_dtype, int32_t n_top,
                   float temperature, float label_weight, float teacher_weight, const float* d_row_weight, float* d_loss, void* d_dz, int64_t dz_stride,
                   void* d_workspace, uint64_t workspace_bytes, void* hip_stream) {
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
    const uint64_t needed = workspace_of(n_tokens, n_vocabulary, n_top);
    const auto ids_bytes = [](int32_t type) { return type == MGWFBP_I64 ? 8 : 4; };
    const uint32_t DZ = 2;
    if (tangled({vector_span(d_loss, n_tokens, 4), matrix_span(d_dz, n_tokens, n_vocabulary, dz_stride, bytes), vector_span(d_workspace, static_cast<int64_t>(needed), 1)},
                {{matrix_span(d_z, n_tokens, n_vocabulary, z_stride, bytes), DZ},
                 {vector_span(d_labels, n_tokens, ids_bytes(label_type)), 0},
                 {matrix_span(d_ids, n_tokens, n_top, ids_stride, ids_bytes(id_type)), 0},
                 {matrix_span(d_teacher, n_tokens, n_top, teacher_stride, dtype_bytes(teacher_dtype)), 0},
                 {vector_span(d_row_weight, n_tokens, 4), 0}}))
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
    const Cut cut = cut_of(n_tokens, n_vocabulary);
    if (cut.parts > 0) {
        if (d_workspace == nullptr || !is_aligned(d_workspace, 256) || workspace_bytes < needed) return MGWFBP_EINVAL;
        a.stats = static_cast<float*>(d_workspace);
        a.parts = cut.parts;
        a.kept_z = a.stats + n_tokens * cut.parts * 3;
        a.kept_stride = label_place(n_top) + 1;
    }
    return with_dtype(dtype, [&](auto* type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        if (n_vocabulary < VEC) return launch(tiny_kernel<T>, a, dim3(static_cast<uint32_t>(ceil_div(n_tokens, 64))), dim3(64), hip_stream);
        if (cut.parts > 0) {
            auto of = [&](void (*parts)(DistillArgs), void (*slopes)(DistillArgs)) {
                const uint32_t n = static_cast<uint32_t>(cut.parts), rows = static_cast<uint32_t>(n_tokens);
                const int status = launch(parts, a, dim3(n, rows), dim3(PART), hip_stream);
                return status != MGWFBP_OK ? status : launch(slopes, a, dim3(d_dz == nullptr ? 1 : n, rows), dim3(PART), hip_stream, Entries<PART>::bytes(n_top));
            };
            if (cut.vecs == 1) return of(part_kernel<T, 1>, part_slope_kernel<T, 1>);
            if (cut.vecs == 2) return of(part_kernel<T, 2>, part_slope_kernel<T, 2>);
            if (cut.vecs == 4) return of(part_kernel<T, 4>, part_slope_kernel<T, 4>);
            return of(part_kernel<T, 8>, part_slope_kernel<T, 8>);
        }
        return with_shape<T>(n_vocabulary, n_top, d_labels != nullptr && n_top > 0 && temperature != 1.f, [&](auto s) {
            constexpr int THREADS = decltype(s)::threads;
            void (*kernel)(DistillArgs) = distill_kernel<T, THREADS, decltype(s)::vecs, decltype(s)::per_simd>;
            return launch(kernel, a, dim3(static_cast<uint32_t>(n_tokens)), dim3(THREADS), hip_stream, Entries<THREADS>::bytes(n_top));
        });
    });
}

}  // extern "C"
