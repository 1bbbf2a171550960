// Gated linear recurrence over the tokens of sequences, and its way back.
//
//   a = 1 / (1 + exp(-gate));  h[t] = a[t] * h[t-1] + c(a[t]) * x[t], for every channel by itself;  y = h
//   c = 1 (free), 1 - a (convex) or sqrt(1 - a^2) (unit);  h before a sequence's first token is first[s], behind its last one last[s]
//
//   D[t] = dy[t] + a[t+1] * D[t+1], with dlast[s] behind a sequence's last token;  dfirst[s] = a D at its first token
//   dx = c D;  dgate = D * a * (1 - a) * (h[t-1] + c'(a) x)
//
// A step is the map h -> a h + b, and such maps compose to maps of the same form: (A, B) then (a, b) is (a A, a B + b).  So a
// block of 128 tokens is cut into eight wavefronts of sixteen tokens each, a lane for a channel or two: every wavefront composes its
// own tokens in registers, the eight pairs meet in LDS, and with what comes in every wavefront goes through its tokens once
// more.  The data is read once and written once, in tokens and channels as they lie; the next block is on its way meanwhile.  A
// workgroup goes through the blocks of a sequence one after the other.  Where there are too few sequences and channels to fill the
// chip, sequences are cut into segments, whose maps a launch before finds (fold_kernel): gate and x (or dy) are read twice then.
//
// The way back needs h[t-1].  It is made again from gate and x and a kept state before each block of 128 tokens, 1/32 of a byte
// an element, instead of kept for every token: y may be thrown away, and h is not rounded.
//
// Sequences lie side by side, all of one length, or one behind the other between offsets.  In the latter form a sequence's first token
// drops what came before it wherever in a block it falls: its map has A = -0, which no product of gates is, and does not look at h, so
// that an infinity or NaN stays in its sequence.
//
// The gate's exponential is exp2(-|gate| log2 e), whose argument is rounded to binary32 twice: the smaller of a and 1 - a is off by
// 1.2e-7 |gate| + 3e-7 of itself, and 0 beyond |gate| = 87, where it is below 2^-126.  The larger one is 1 less the smaller, so that a share that stays for hundreds of tokens is off by little more
// than its rounding, which is to no side: by the reciprocal alone, which is to one, gradients of 37 sequences of some 900 tokens were
// off by 7e-7 of their norm and are by 2e-7.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "device_types.h"
#include "mgwfbp_layers.h"
#include "spans.h"

namespace {

using namespace ops;

constexpr int LANES = 64, BLOCK = MGWFBP_RECUR_BLOCK;

// How sequences lie in a unit of work: a sequence is one; several of one length share a block; or between offsets.
enum { ONE, EVEN, PACKED };
// Tokens up to which a lane goes through a sequence by itself.  Us forward and back, 1024 bfloat16 channels, that and blocks: 8 sequences of 8 tokens 6.8 and 7.3,
// 6.2 and 14.9; 256 of 6 6.7 and 10.4, 8.2 and 24.6; 4096 of 8 51 and 129, 76 and 131.  Twice as many: 256 of 16 13.9 and 22.9, 9.8 and 16.1.
constexpr int SHORT = 8;

struct RecurArgs {
    const void* gate;
    const void* x;
    const void* dy;
    const float* first;
    const float* dlast;
    const void* offsets;
    void* y;
    void* dgate;
    void* dx;
    float* last;
    float* dfirst;
    float* states;                       // [units][blocks][channels]
    float* maps;                         // [units][segments][2][channels]: A and B of a segment
    int64_t gate_stride, x_stride, dy_stride, y_stride, dgate_stride, dx_stride;
    int64_t channels, sequences, tokens, blocks;             // tokens and blocks of a unit: of a sequence, of those that share a block, or of all
    int64_t length, rows;                // EVEN: tokens of a sequence, and of all of them
    uint32_t slabs, segments, per_segment;                   // pieces of the channels; pieces of a unit, and their blocks
    int32_t offset_type;
    int32_t copied;                      // first is in the maps' last segment: the caller's may be overwritten by last
};

// The wavefront's number, as what it is: the same in all its lanes, so that what follows from it is computed once for them.
__device__ __forceinline__ int wave_of() { return __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x / LANES)); }

// CH neighbouring elements of a row, as bits: two of 16 bits share a register.
template <int BYTES> struct Bits;
template <> struct Bits<2> { typedef uint16_t type; };
template <> struct Bits<4> { typedef uint32_t type; };
template <typename T, int CH> struct Piece {
    typedef T vec __attribute__((ext_vector_type(CH), aligned(alignof(T))));
    typedef typename Bits<CH * sizeof(T)>::type bits;
    bits v;
    __device__ __forceinline__ void load(const T* p) { v = __builtin_bit_cast(bits, *reinterpret_cast<const vec*>(p)); }
    __device__ __forceinline__ void load(const T* p, int n) {            // the first n of them
        typedef typename Bits<sizeof(T)>::type one;
        v = 0;
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (i < n) v |= static_cast<bits>(static_cast<bits>(reinterpret_cast<const one*>(p)[i]) << (8 * sizeof(T) * i % 32));
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, v);
        else if constexpr (__is_same(T, __bf16)) return __builtin_bit_cast(float, i == 0 ? static_cast<uint32_t>(v) << 16 : static_cast<uint32_t>(v) & 0xffff0000u);
        else return static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(v >> (16 * i % 32))));
    }
};

// a and 1 - a of a gate, both to their own last digits.
__device__ __forceinline__ void logistic(float g, float& a, float& rest) {
    const float e = __builtin_amdgcn_exp2f(__builtin_fabsf(g) * -1.44269504088896341f);
    const float far = e * __builtin_amdgcn_rcpf(1.f + e), near = 1.f - far;
    a = g >= 0.f ? near : far;
    rest = g >= 0.f ? far : near;
}
template <int KIND> __device__ __forceinline__ float factor(float a, float rest) {
    if constexpr (KIND == MGWFBP_RECUR_FREE) return 1.f;
    else if constexpr (KIND == MGWFBP_RECUR_CONVEX) return rest;
    else return __builtin_amdgcn_sqrtf(__builtin_fmaf(rest, a, rest));
}
// d h[t] / d gate[t]
template <int KIND> __device__ __forceinline__ float slope(float a, float rest, float before, float x) {
    if constexpr (KIND == MGWFBP_RECUR_FREE) return a * rest * before;
    else if constexpr (KIND == MGWFBP_RECUR_CONVEX) return a * rest * (before - x);
    else return a * (rest * before - a * factor<KIND>(a, rest) * __builtin_amdgcn_rcpf(1.f + a) * x);     // dc/da = -a / c
}

// Where sequences begin that lie one behind the other: offsets [count], not decreasing.  All lanes of a wavefront ask together.
// Offsets are kept within 0 .. most, and every place that is read is one of the count, so wrong ones lead nowhere else.
struct Bounds {
    const void* p;
    int type, count, most, held;
    __device__ __forceinline__ int at(int i) const {
        const int64_t v = type == MGWFBP_I64 ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
        return static_cast<int>(min(max(v, static_cast<int64_t>(0)), static_cast<int64_t>(most)));
    }
    __device__ __forceinline__ void open(const RecurArgs& A) {
        p = A.offsets;
        type = A.offset_type;
        count = static_cast<int>(A.sequences) + 1;
        most = static_cast<int>(A.tokens);
        const int lane = threadIdx.x % LANES;
        held = at(min(lane, count - 1));                     // up to 63 sequences: all there is
    }
    // How many offsets are <= t: of 64 places at a time, so two or three waits for memory where there are thousands.
    __device__ __forceinline__ int up_to(int t) const {
        const int lane = threadIdx.x % LANES;
        if (count <= LANES) return __popcll(__ballot(lane < count && held <= t));
        int lo = 0, hi = count;                              // those before lo are, those from hi on are not
        while (hi - lo > LANES) {
            const int step = (hi - lo + LANES - 1) / LANES, i = lo + (lane + 1) * step - 1;
            const int k = __popcll(__ballot(i < hi && at(min(i, count - 1)) <= t));
            hi = min(hi, lo + (k + 1) * step - 1);
            lo += k * step;
        }
        return lo + __popcll(__ballot(lo + lane < hi && at(min(lo + lane, count - 1)) <= t));
    }
    __device__ __forceinline__ int sequence_of(int t) const { return min(max(up_to(t) - 1, 0), count - 2); }
    // Bit i: an offset is t0 + i, 0 <= i <= N.
    template <int N> __device__ __forceinline__ uint32_t marks(int t0) const {
        const int lane = threadIdx.x % LANES;
        uint32_t bits = 0;
        if (count <= LANES) {
            const int i = held - t0;
            const bool in = lane < count && i >= 0 && i <= N;
            if (__ballot(in) == 0) return 0;
            bits = in ? 1u << i : 0u;
        } else {
            const int from = up_to(t0 - 1), to = up_to(t0 + N);
            if (from >= to) return 0;
            for (int j = from + lane; j < to; j += LANES) {
                const int i = at(j) - t0;
                if (i >= 0 && i <= N) bits |= 1u << i;
            }
        }
#pragma unroll
        for (int d = LANES / 2; d > 0; d /= 2) bits |= static_cast<uint32_t>(__shfl_xor(static_cast<int>(bits), d));
        return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(bits)));
    }
};

// What a wavefront knows of its place: W of them share a block, N tokens each.
template <int MODE_, int CH_, int W> struct Place {
    static constexpr int MODE = MODE_;
    static constexpr int CH = CH_, N = BLOCK / W;
    static constexpr uint32_t ALL = static_cast<uint32_t>((uint64_t(1) << N) - 1);
    Bounds bounds;
    int64_t unit, base;                  // base: the unit's first row
    uint32_t c;                          // the lane's first channel
    int n;                               // and how many it has
    bool full;                           // all lanes have CH
    int begin, end;                      // tokens of the unit that are sequences'
    int length;                          // EVEN: of a sequence
    uint32_t segment, first_block, end_block;

    __device__ __forceinline__ void open(const RecurArgs& A) {
        // Workgroups go round the eight dies; each die takes a stretch of the work, so that it has whole rows, all their lines.
        constexpr uint32_t DIES = 8;
        const uint32_t die = blockIdx.x % DIES, share = gridDim.x / DIES, more = gridDim.x % DIES;
        const uint32_t work = die * share + min(die, more) + blockIdx.x / DIES;
        const uint32_t slab = work % A.slabs, rest = work / A.slabs;
        segment = rest % A.segments;
        unit = rest / A.segments;
        base = MODE == PACKED ? 0 : unit * A.tokens;
        c = (slab * LANES + threadIdx.x % LANES) * CH;
        n = static_cast<int>(max(static_cast<int64_t>(0), min(A.channels - c, static_cast<int64_t>(CH))));
        full = static_cast<int64_t>(slab + 1) * LANES * CH <= A.channels;
        begin = 0;
        end = static_cast<int>(A.tokens);
        if constexpr (MODE == EVEN) {
            end = static_cast<int>(min(A.tokens, A.rows - base));
            length = static_cast<int>(A.length);
        }
        if constexpr (MODE == PACKED) {
            bounds.open(A);
            begin = __builtin_amdgcn_readfirstlane(bounds.at(0));
            end = __builtin_amdgcn_readfirstlane(bounds.at(bounds.count - 1));
        }
        first_block = segment * A.per_segment;
        end_block = min(first_block + A.per_segment, static_cast<uint32_t>((end + BLOCK - 1) / BLOCK));
    }
    // The lane's distance from a row's first element, in bytes and 32 bits, made anew where it is used: memory instructions add it to an address
    // that all lanes share, if the compiler sees both; carried along in 64 bits it would cost an addition for every access.
    template <typename T> __device__ __forceinline__ uint32_t lane_bytes() const {
        uint32_t bytes = static_cast<uint32_t>(c * sizeof(T));
        asm volatile("" : "+v"(bytes));
        return bytes;
    }
    template <typename T> static __device__ __forceinline__ T* in(T* row, uint32_t bytes) {
        typedef std::conditional_t<std::is_const_v<T>, const char, char> byte;
        return reinterpret_cast<T*>(reinterpret_cast<byte*>(row) + bytes);
    }
    __device__ __forceinline__ int row(int t) const { return min(max(t, begin), max(end - 1, 0)); }      // one that may be read
    __device__ __forceinline__ bool whole(int t0) const { return full && t0 >= begin && t0 + N <= end; }
    // Bits of the N tokens from t0 on: a sequence's; and where they lie one behind the other, the first of one, the last of one.
    __device__ __forceinline__ void masks(int t0, uint32_t& valid, uint32_t& first, uint32_t& last) const {
        const int lo = min(max(begin - t0, 0), N), hi = min(max(end - t0, 0), N);
        valid = ALL >> (N - hi) & (ALL << lo) & ALL;
        first = last = 0;
        if constexpr (MODE != ONE) {
            uint32_t marks = 0;
            if constexpr (MODE == PACKED) {
                marks = bounds.template marks<N>(t0);
            } else {
                for (int t = (t0 + length - 1) / length * length; t <= t0 + N; t += length) marks |= 1u << (t - t0);
            }
            first = marks & valid;
            last = marks >> 1 & valid;
        }
    }
    __device__ __forceinline__ int64_t sequence_at(int t) const {
        if constexpr (MODE == PACKED) return bounds.sequence_of(t);
        else if constexpr (MODE == EVEN) return (base + t) / length;
        else return unit;
    }
    __device__ __forceinline__ void state(const RecurArgs& A, const float* from, int64_t sequence, float (&out)[CH]) const {
#pragma unroll
        for (int k = 0; k < CH; ++k) out[k] = from != nullptr && k < n ? from[sequence * A.channels + c + k] : 0.f;
    }
    __device__ __forceinline__ void put_state(const RecurArgs& A, float* to, int64_t sequence, const float (&in)[CH]) const {
        if (to == nullptr) return;
#pragma unroll
        for (int k = 0; k < CH; ++k)
            if (k < n) to[sequence * A.channels + c + k] = in[k];
    }
    // Sequences without tokens hand their state on.
    __device__ __forceinline__ void empty_sequences(const RecurArgs& A, const float* from, float* to) const {
        if constexpr (MODE == PACKED) {
            if (to == nullptr) return;
            for (int64_t s0 = wave_of() * LANES; s0 < A.sequences; s0 += W * LANES) {
                const int64_t s = s0 + threadIdx.x % LANES;
                uint64_t empty = __ballot(s < A.sequences && bounds.at(static_cast<int>(min(s, A.sequences - 1))) >= bounds.at(static_cast<int>(min(s + 1, A.sequences))));
                while (empty != 0) {
                    const int64_t at = s0 + __ffsll(static_cast<unsigned long long>(empty)) - 1;
                    empty &= empty - 1;
                    float h[CH];
                    state(A, from, at, h);
                    put_state(A, to, at, h);
                }
            }
        }
    }
};

// A wavefront's tokens of a block, as they are in memory.
template <typename T, typename P> struct Tokens {
    Piece<T, P::CH> v[P::N];
    __device__ __forceinline__ void load(const P& at, const void* from, int64_t stride, int t0) {
        if (at.whole(t0)) {
            const T* row = static_cast<const T*>(from) + (at.base + t0) * stride;
            const uint32_t bytes = at.template lane_bytes<T>();
#pragma unroll
            for (int i = 0; i < P::N; ++i, row += stride) v[i].load(at.in(row, bytes));
        } else {
#pragma unroll
            for (int i = 0; i < P::N; ++i) v[i].load(static_cast<const T*>(from) + (at.base + at.row(t0 + i)) * stride + at.c, at.n);
        }
    }
};

// A map that begins a sequence: it gives b whatever comes in.  A unit of one sequence needs none: it begins with what comes in.
constexpr float FRESH = -0.f;
template <int MODE> __device__ __forceinline__ bool is_fresh(float a) { return MODE != ONE && __builtin_bit_cast(uint32_t, a) == 0x80000000u; }
template <int MODE> __device__ __forceinline__ float through(float a, float b, float h) { return is_fresh<MODE>(a) ? b : __builtin_fmaf(a, h, b); }
// (a, b) and then (ma, mb), in (a, b)
template <int MODE> __device__ __forceinline__ void compose(float& a, float& b, float ma, float mb) {
    b = through<MODE>(ma, mb, b);
    a = is_fresh<MODE>(ma) ? FRESH : a * ma;               // a product of FRESH and a gate is FRESH again
}

// Maps of wavefronts in LDS, two blocks in turn, so that one barrier a block is enough.
template <int MODE, int CH, int W> struct Maps {
    float m[2][W][2][LANES * CH];
    __device__ __forceinline__ void put(uint32_t turn, int wave, const float (&a)[CH], const float (&b)[CH]) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            m[turn][wave][0][k * LANES + threadIdx.x % LANES] = a[k];
            m[turn][wave][1][k * LANES + threadIdx.x % LANES] = b[k];
        }
    }
    // h through the map of a wavefront.
    __device__ __forceinline__ void take(uint32_t turn, int wave, float (&h)[CH]) const {
#pragma unroll
        for (int k = 0; k < CH; ++k) h[k] = through<MODE>(m[turn][wave][0][k * LANES + threadIdx.x % LANES], m[turn][wave][1][k * LANES + threadIdx.x % LANES], h[k]);
    }
};

template <int CH> __device__ __forceinline__ void nothing_yet(float (&ma)[CH], float (&mb)[CH]) {
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        ma[k] = 1.f;
        mb[k] = 0.f;
    }
}

// h, which comes into a unit, through the maps of the segments before a workgroup's (or, on the way back, behind it); the wavefronts
// share them.
template <bool BACK, int MODE, int CH, int W> __device__ __forceinline__ void through_segments(const RecurArgs& A, const Place<MODE, CH, W>& at, Maps<MODE, CH, W>& room, float (&h)[CH]) {
    const int wave = wave_of();
    const int count = static_cast<int>(BACK ? A.segments - 1 - at.segment : at.segment);
    const int each = (count + W - 1) / W, from = min(wave * each, count), to = min(from + each, count);
    float a[CH], b[CH];
    nothing_yet(a, b);
#pragma unroll 4
    for (int i = from; i < to; ++i) {
        const int64_t s = at.unit * A.segments + (BACK ? A.segments - 1 - i : i);
        const float* const map = A.maps + s * 2 * A.channels + at.c;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const float ma = k < at.n ? map[k] : 1.f, mb = k < at.n ? map[A.channels + k] : 0.f;
            compose<MODE>(a[k], b[k], ma, mb);
        }
    }
    room.put(1, wave, a, b);
    __syncthreads();
    for (int w = 0; w < W; ++w) room.take(1, w, h);          // turn 1 is written again after another barrier
}

// The first state of a unit of one sequence.  `last` may be the same memory: a workgroup that has a whole unit has read it before its first
// barrier and writes the last state behind it; where there are more, fold_kernel has put it elsewhere.
template <int CH, int W> __device__ __forceinline__ void unit_first(const RecurArgs& A, const Place<ONE, CH, W>& at, float (&h)[CH]) {
    if (A.copied) {
        const float* const map = A.maps + (at.unit * A.segments + A.segments - 1) * 2 * A.channels + at.c;
#pragma unroll
        for (int k = 0; k < CH; ++k) h[k] = k < at.n ? map[k] : 0.f;
    } else {
        at.state(A, A.first, at.unit, h);
    }
}

// gate and x of a wavefront's tokens to the steps h -> a h + b; a token of no sequence changes nothing.
template <int KIND, typename T, typename P> __device__ __forceinline__ void steps_of(const Tokens<T, P>& gate, const Tokens<T, P>& x, uint32_t valid, float (&a)[P::N][P::CH],
                                                                                     float (&rest)[P::N][P::CH], float (&b)[P::N][P::CH]) {
#pragma unroll
    for (int i = 0; i < P::N; ++i)
#pragma unroll
        for (int k = 0; k < P::CH; ++k) {
            logistic(gate.v[i].get(k), a[i][k], rest[i][k]);
            b[i][k] = factor<KIND>(a[i][k], rest[i][k]) * x.v[i].get(k);
        }
    if (valid != P::ALL) {
        // taken here, so that the selections stay in the branch
        const uint32_t some = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(valid)));
#pragma unroll
        for (int i = 0; i < P::N; ++i)
#pragma unroll
            for (int k = 0; k < P::CH; ++k) {
                a[i][k] = some >> i & 1 ? a[i][k] : 1.f;
                b[i][k] = some >> i & 1 ? b[i][k] : 0.f;
            }
    }
}

// The map of a wavefront's tokens; reset(i, h) puts the state before token i, which begins a sequence, into h.
template <int N, int CH, typename F> __device__ __forceinline__ void compose_steps(const float (&a)[N][CH], const float (&b)[N][CH], uint32_t begins, F&& reset, float (&ma)[CH],
                                                                                   float (&mb)[CH]) {
    auto step = [&](int i) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            mb[k] = __builtin_fmaf(a[i][k], mb[k], b[i][k]);
            ma[k] *= a[i][k];
        }
    };
    if (begins == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) step(i);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (begins >> i & 1) {
            reset(i, mb);
#pragma unroll
            for (int k = 0; k < CH; ++k) ma[k] = FRESH;
        }
        step(i);
    }
}
// The same from the end, for what flows from a token to the one before it, g -> a (dy + g), a being 1 for tokens of no sequence.
template <int N, int CH, typename T, typename P, typename F> __device__ __forceinline__ void compose_flows(const float (&a)[N][CH], const Tokens<T, P>& dy, uint32_t valid, uint32_t ends,
                                                                                                          F&& reset, float (&ma)[CH], float (&mb)[CH]) {
    auto step = [&](int i, bool valid) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            mb[k] = a[i][k] * (mb[k] + (valid ? dy.v[i].get(k) : 0.f));
            ma[k] *= a[i][k];
        }
    };
    if (ends == 0 && valid == P::ALL) {
#pragma unroll
        for (int i = N - 1; i >= 0; --i) step(i, true);
        return;
    }
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
        if (ends >> i & 1) {
            reset(i, mb);
#pragma unroll
            for (int k = 0; k < CH; ++k) ma[k] = FRESH;
        }
        step(i, valid >> i & 1);
    }
}

// ---------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------

// 65543 tokens of 1024 binary16 channels, 403 MB: 83 to 87 us, 4.7 to 4.9 TB/s, with the segments' maps before it 154.  The vector units are at work in 57 % of the
// cycles (three transcendental functions an element), and four wavefronts a SIMD wait for 35 % of their time: neither is full.  32 x 128 tokens of 512 channels, in
// one block each, 5.7 us.
template <typename T, int KIND, int CH, int W, int MODE> __global__ __launch_bounds__(W * LANES) void scan_kernel(RecurArgs A) {
    typedef Place<MODE, CH, W> P;
    constexpr int N = P::N;
    __shared__ Maps<MODE, CH, W> maps;
    P at;
    at.open(A);
    const int wave = wave_of();
    if (at.segment == 0) at.empty_sequences(A, A.first, A.last);
    if (at.first_block >= at.end_block) return;
    Tokens<T, P> gate, x;
    int t0 = static_cast<int>(at.first_block) * BLOCK + wave * N;
    gate.load(at, A.gate, A.gate_stride, t0);
    x.load(at, A.x, A.x_stride, t0);
    float carry[CH] = {};
    if constexpr (MODE == ONE) unit_first(A, at, carry);
    if (at.segment > 0) through_segments<false>(A, at, maps, carry);
    for (uint32_t block = at.first_block; block < at.end_block; ++block, t0 += BLOCK) {
        const uint32_t turn = (block - at.first_block) % 2;
        uint32_t valid, begins, ends;
        at.masks(t0, valid, begins, ends);
        float a[N][CH], rest[N][CH], b[N][CH];
        steps_of<KIND>(gate, x, valid, a, rest, b);
        if (block + 1 < at.end_block) {
            gate.load(at, A.gate, A.gate_stride, t0 + BLOCK);
            x.load(at, A.x, A.x_stride, t0 + BLOCK);
        }
        // The step of a token that begins a sequence gives its state whatever comes in: its first state is read here and not again, since `last`
        // may be the same memory.
        if (begins != 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (!(begins >> i & 1)) continue;
                float first[CH];
                at.state(A, A.first, at.sequence_at(t0 + i), first);
                if (MODE == EVEN) at.put_state(A, A.states, at.sequence_at(t0 + i), first);
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    b[i][k] = __builtin_fmaf(a[i][k], first[k], b[i][k]);
                    a[i][k] = FRESH;
                }
            }
        }
        float ma[CH], mb[CH], h[CH];
        nothing_yet(ma, mb);
        if (begins == 0) {
            compose_steps(a, b, 0, [](int, float (&)[CH]) {}, ma, mb);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int k = 0; k < CH; ++k) compose<MODE>(ma[k], mb[k], a[i][k], b[i][k]);
        }
        maps.put(turn, wave, ma, mb);
        if constexpr (MODE == ONE) {                         // what came in is here, and not on its way, when another wavefront may write over it
#pragma unroll
            for (int k = 0; k < CH; ++k) asm volatile("" ::"v"(carry[k]));
        }
        __syncthreads();
        if (MODE != EVEN && A.states != nullptr && wave == 0 && t0 >= at.begin) {
#pragma unroll
            for (int k = 0; k < CH; ++k) h[k] = carry[k];
            if (begins & 1) at.state(A, A.first, at.sequence_at(t0), h);         // offsets: first is not last
            at.put_state(A, A.states, at.unit * A.blocks + block, h);
        }
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w == wave) {
#pragma unroll
                for (int k = 0; k < CH; ++k) h[k] = carry[k];
            }
            maps.take(turn, w, carry);
        }
        T* row = static_cast<T*>(A.y) + (at.base + t0) * A.y_stride;
        if (at.full && valid == P::ALL && (begins | ends) == 0) {
            const uint32_t bytes = at.template lane_bytes<T>();
#pragma unroll
            for (int i = 0; i < N; ++i, row += A.y_stride) {
#pragma unroll
                for (int k = 0; k < CH; ++k) h[k] = __builtin_fmaf(a[i][k], h[k], b[i][k]);
                store_some(at.in(row, bytes), h, CH);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i, row += A.y_stride) {
#pragma unroll
                for (int k = 0; k < CH; ++k) h[k] = through<MODE>(a[i][k], b[i][k], h[k]);
                if (valid >> i & 1) store_some(row + at.c, h, at.n);
                if (ends >> i & 1) at.put_state(A, A.last, at.sequence_at(t0 + i), h);
            }
        }
        // tokens behind a sequence's last one have changed nothing
        if (MODE == ONE && wave == W - 1 && block + 1 == A.blocks) at.put_state(A, A.last, at.unit, h);
    }
}

// ---------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------

// gate, x and dy in, dgate and dx out, a state for every 128 tokens: 32775 tokens of 1001 binary32 channels, 37 sequences one behind the other, 656 MB, 143 to 147 us,
// 4.5 TB/s; with the segments' maps 212.  Vector units 22 % of the cycles; two wavefronts a SIMD (256 workgroups), which wait for 53 % of their time.
// 8 x 512 tokens of 1024 bfloat16 channels 11 us and 4 for the maps.
template <typename T, int KIND, int CH, int W, int MODE> __global__ __launch_bounds__(W * LANES) void back_kernel(RecurArgs A) {
    typedef Place<MODE, CH, W> P;
    constexpr int N = P::N;
    __shared__ Maps<MODE, CH, W> forth, back;
    P at;
    at.open(A);
    const int wave = wave_of();
    if (at.segment == 0) at.empty_sequences(A, A.dlast, A.dfirst);
    if (at.first_block >= at.end_block) return;
    Tokens<T, P> gate, x, dy;
    float carry[CH] = {}, state[CH];
    int t0 = static_cast<int>(at.end_block - 1) * BLOCK + wave * N;
    gate.load(at, A.gate, A.gate_stride, t0);
    dy.load(at, A.dy, A.dy_stride, t0);
    x.load(at, A.x, A.x_stride, t0);
    if constexpr (MODE != EVEN) at.state(A, A.states, at.unit * A.blocks + at.end_block - 1, state);       // EVEN: every block begins a sequence
    else
#pragma unroll
        for (int k = 0; k < CH; ++k) state[k] = 0.f;
    if constexpr (MODE == ONE) at.state(A, A.dlast, at.unit, carry);
    if (at.segment + 1 < A.segments) through_segments<true>(A, at, back, carry);
    for (uint32_t block = at.end_block; block-- > at.first_block; t0 -= BLOCK) {
        const uint32_t turn = (at.end_block - 1 - block) % 2;
        uint32_t valid, begins, ends;
        at.masks(t0, valid, begins, ends);
        auto flow_in = [&](int i, float (&g)[CH]) { at.state(A, A.dlast, at.sequence_at(t0 + i), g); };
        auto state_in = [&](int i, float (&h)[CH]) { at.state(A, A.first, at.sequence_at(t0 + i), h); };
        float a[N][CH], rest[N][CH], before[N][CH];          // before: b, until the state before the token takes its place
        steps_of<KIND>(gate, x, valid, a, rest, before);
        if (block > at.first_block) gate.load(at, A.gate, A.gate_stride, t0 - BLOCK);        // the others are still needed
        float ma[CH], mb[CH];
        nothing_yet(ma, mb);
        compose_steps(a, before, begins, state_in, ma, mb);
        forth.put(turn, wave, ma, mb);
        nothing_yet(ma, mb);
        compose_flows(a, dy, valid, ends, flow_in, ma, mb);
        back.put(turn, wave, ma, mb);
        __syncthreads();
        float flow[CH];
        for (int w = 0; w < wave; ++w) forth.take(turn, w, state);
#pragma unroll
        for (int w = W - 1; w >= 0; --w) {
            if (w == wave) {
#pragma unroll
                for (int k = 0; k < CH; ++k) flow[k] = carry[k];
            }
            back.take(turn, w, carry);
        }
        auto forward = [&](int i) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const float b = before[i][k];
                before[i][k] = state[k];
                state[k] = __builtin_fmaf(a[i][k], state[k], b);
            }
        };
        auto backward = [&](int i, float (&dg)[CH], float (&dx)[CH]) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const float d = flow[k] + dy.v[i].get(k);
                dx[k] = factor<KIND>(a[i][k], rest[i][k]) * d;
                dg[k] = slope<KIND>(a[i][k], rest[i][k], before[i][k], x.v[i].get(k)) * d;
                flow[k] = a[i][k] * d;
            }
        };
        T* to_gate = static_cast<T*>(A.dgate) + (at.base + t0 + N - 1) * A.dgate_stride;
        T* to_x = static_cast<T*>(A.dx) + (at.base + t0 + N - 1) * A.dx_stride;
        if (at.full && valid == P::ALL && (begins | ends) == 0) {
            const uint32_t bytes = at.template lane_bytes<T>();
#pragma unroll
            for (int i = 0; i < N; ++i) forward(i);
#pragma unroll
            for (int i = N - 1; i >= 0; --i, to_gate -= A.dgate_stride, to_x -= A.dx_stride) {
                float dg[CH], dx[CH];
                backward(i, dg, dx);
                store_some(at.in(to_gate, bytes), dg, CH);
                store_some(at.in(to_x, bytes), dx, CH);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (begins >> i & 1) state_in(i, state);
                forward(i);
            }
#pragma unroll
            for (int i = N - 1; i >= 0; --i, to_gate -= A.dgate_stride, to_x -= A.dx_stride) {
                if (ends >> i & 1) flow_in(i, flow);
                if (!(valid >> i & 1)) continue;
                float dg[CH], dx[CH];
                backward(i, dg, dx);
                store_some(to_gate + at.c, dg, at.n);
                store_some(to_x + at.c, dx, at.n);
                if (begins >> i & 1) at.put_state(A, A.dfirst, at.sequence_at(t0 + i), flow);
            }
        }
        if (MODE == ONE && wave == 0 && block == 0) at.put_state(A, A.dfirst, at.unit, flow);
        if (block > at.first_block) {
            dy.load(at, A.dy, A.dy_stride, t0 - BLOCK);
            x.load(at, A.x, A.x_stride, t0 - BLOCK);
            if constexpr (MODE != EVEN) at.state(A, A.states, at.unit * A.blocks + block - 1, state);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// segments
// ---------------------------------------------------------------------------------------------

// The map of a segment: every wavefront composes its share of the tokens, N at a time.  On the way back it is the map of what
// flows from a token to the one before it.  The last segment's map (the first one's, on the way back) is
// nobody's, so it is not made; its place keeps the first state where that may be overwritten.  65543 tokens of 1024 binary16 channels, 268 MB: 75 to 79 us,
// 3.5 TB/s; vector units 49 % of the cycles, four wavefronts a SIMD that wait for 45 % of their time.  As much again is read by the launch behind it.  Workgroups of a block each that wait within one launch for the maps of the blocks before theirs read
// everything once; they were 154 -> 516 us forward and 214 -> 251 back here, since the some 500 workgroups that fit the chip are one stretch of the chain after the other,
// each with its loads, its wait and its stores by themselves; only wide binary32 rows gained on the way back (2 x 16384 tokens 184 -> 145).
template <typename T, int KIND, int CH, int W, int MODE, bool BACK> __global__ __launch_bounds__(W * LANES) void fold_kernel(RecurArgs A) {
    typedef Place<MODE, CH, W> P;
    constexpr int N = P::N;
    __shared__ Maps<MODE, CH, W> maps;
    P at;
    at.open(A);
    const int wave = wave_of();
    if (!BACK && MODE == ONE && A.copied && at.segment == A.segments - 1 && wave == 0) {
        float first[CH];
        at.state(A, A.first, at.unit, first);
        float* const map = A.maps + (at.unit * A.segments + at.segment) * 2 * A.channels + at.c;
#pragma unroll
        for (int k = 0; k < CH; ++k)
            if (k < at.n) map[k] = first[k];
    }
    if (at.segment == (BACK ? 0 : A.segments - 1)) return;
    float ma[CH], mb[CH];
    nothing_yet(ma, mb);
    const int pieces = static_cast<int>(A.per_segment);      // of a wavefront
    const int from = static_cast<int>(at.first_block) * BLOCK + wave * pieces * N;
    if (at.first_block < at.end_block) {
        const void* const other = BACK ? A.dy : A.x;
        const int64_t other_stride = BACK ? A.dy_stride : A.x_stride;
        Tokens<T, P> gate, x;
        auto start = [&](int p) { return from + (BACK ? pieces - 1 - p : p) * N; };
        gate.load(at, A.gate, A.gate_stride, start(0));
        x.load(at, other, other_stride, start(0));
        for (int p = 0; p < pieces; ++p) {
            const int t0 = start(p);
            uint32_t valid, begins, ends;
            at.masks(t0, valid, begins, ends);
            float a[N][CH], rest[N][CH], b[N][CH];
            steps_of<BACK ? MGWFBP_RECUR_FREE : KIND>(gate, x, valid, a, rest, b);
            auto reset = [&](int i, float (&h)[CH]) { at.state(A, BACK ? A.dlast : A.first, at.sequence_at(t0 + i), h); };
            if constexpr (BACK) compose_flows(a, x, valid, ends, reset, ma, mb);
            else compose_steps(a, b, begins, reset, ma, mb);
            if (p + 1 < pieces) {
                gate.load(at, A.gate, A.gate_stride, start(p + 1));
                x.load(at, other, other_stride, start(p + 1));
            }
        }
    }
    maps.put(0, wave, ma, mb);
    __syncthreads();
    if (wave != 0) return;
    const int lane = threadIdx.x % LANES;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        float a = 1.f, b = 0.f;
        for (int j = 0; j < W; ++j) {
            const int w = BACK ? W - 1 - j : j;
            compose<MODE>(a, b, maps.m[0][w][0][k * LANES + lane], maps.m[0][w][1][k * LANES + lane]);
        }
        if (k < at.n) {
            float* const map = A.maps + (at.unit * A.segments + at.segment) * 2 * A.channels + at.c + k;
            map[0] = a;
            map[A.channels] = b;
        }
    }
}

// ---------------------------------------------------------------------------------------------
// short sequences of one length
// ---------------------------------------------------------------------------------------------

constexpr int SHORT_THREADS = 256;

// A lane goes through eight channels of a sequence: a step of an answer is one token.  Bound by the launch (8 sequences of one token: 3.0 us, 3.9 the call); 4096 of
// 8 tokens and 1024 bfloat16 channels 51 us, 3.9 TB/s.
template <typename T, int KIND> __global__ __launch_bounds__(SHORT_THREADS) void short_scan_kernel(RecurArgs A) {
    const int64_t vecs = (A.channels + VEC - 1) / VEC, at = static_cast<int64_t>(blockIdx.x) * SHORT_THREADS + threadIdx.x;
    const int64_t s = at / vecs, c = (at - s * vecs) * VEC;
    if (s >= A.sequences) return;
    const int n = static_cast<int>(min(A.channels - c, static_cast<int64_t>(VEC)));
    const Raw8<float> first = load8(A.first != nullptr ? A.first + s * A.channels + c : nullptr, A.first != nullptr ? n : 0);
    float h[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) h[k] = get(first, k);
    if (A.states != nullptr && A.tokens > 0) store8(A.states + s * A.channels + c, h, n);
    const int64_t t0 = s * A.tokens;
    const int tokens = static_cast<int>(A.tokens);
    Raw8<T> gate, x, next_gate, next_x;
    const auto ask = [&](int i, Raw8<T>& gate_of, Raw8<T>& x_of) {
        gate_of = load8(static_cast<const T*>(A.gate) + (t0 + i) * A.gate_stride + c, i < tokens ? n : 0);
        x_of = load8(static_cast<const T*>(A.x) + (t0 + i) * A.x_stride + c, i < tokens ? n : 0);
    };
    ask(0, next_gate, next_x);
    for (int i = 0; i < tokens; ++i) {
        gate = next_gate;
        x = next_x;
        ask(i + 1, next_gate, next_x);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            float a, rest;
            logistic(get(gate, k), a, rest);
            h[k] = __builtin_fmaf(a, h[k], factor<KIND>(a, rest) * get(x, k));
        }
        store8(static_cast<T*>(A.y) + (t0 + i) * A.y_stride + c, h, n);
    }
    if (A.last != nullptr) store8(A.last + s * A.channels + c, h, n);
}

// Channels of a lane: four bytes of a row.
constexpr int channels_of(int64_t bytes) { return bytes == 4 ? 1 : 2; }

// Its way back: the states of up to MOST tokens stay in registers, for four tokens fewer of them: 4096 sequences of 1 token and 1024 bfloat16 channels 18 us, 24 with
// room for eight.
template <typename T, int KIND, int MOST> __global__ __launch_bounds__(SHORT_THREADS) void short_back_kernel(RecurArgs A) {
    constexpr int CH = channels_of(sizeof(T));
    const int64_t pieces = (A.channels + CH - 1) / CH, at = static_cast<int64_t>(blockIdx.x) * SHORT_THREADS + threadIdx.x;
    const int64_t s = at / pieces, c = (at - s * pieces) * CH;
    if (s >= A.sequences) return;
    const int n = static_cast<int>(min(A.channels - c, static_cast<int64_t>(CH))), tokens = static_cast<int>(A.tokens);
    Piece<T, CH> gate[MOST], x[MOST], dy[MOST];
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        const int64_t t = s * tokens + i;
        const int m = i < tokens ? n : 0;
        gate[i].load(static_cast<const T*>(A.gate) + t * A.gate_stride + c, m);
        x[i].load(static_cast<const T*>(A.x) + t * A.x_stride + c, m);
        dy[i].load(static_cast<const T*>(A.dy) + t * A.dy_stride + c, m);
    }
    float h[CH], flow[CH], before[MOST][CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        h[k] = A.first != nullptr && k < n ? A.first[s * A.channels + c + k] : 0.f;
        flow[k] = A.dlast != nullptr && k < n ? A.dlast[s * A.channels + c + k] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        if (i >= tokens) continue;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            float a, rest;
            logistic(gate[i].get(k), a, rest);
            before[i][k] = h[k];
            h[k] = __builtin_fmaf(a, h[k], factor<KIND>(a, rest) * x[i].get(k));
        }
    }
#pragma unroll
    for (int i = MOST - 1; i >= 0; --i) {
        if (i >= tokens) continue;
        float dg[CH], dx[CH];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            float a, rest;
            logistic(gate[i].get(k), a, rest);
            const float d = flow[k] + dy[i].get(k);
            dx[k] = factor<KIND>(a, rest) * d;
            dg[k] = slope<KIND>(a, rest, before[i][k], x[i].get(k)) * d;
            flow[k] = a * d;
        }
        const int64_t t = s * tokens + i;
        store_some(static_cast<T*>(A.dgate) + t * A.dgate_stride + c, dg, n);
        store_some(static_cast<T*>(A.dx) + t * A.dx_stride + c, dx, n);
    }
    if (A.dfirst != nullptr) store_some(A.dfirst + s * A.channels + c, flow, n);
}

// ---- host side -------------------------------------------------------------------------------

constexpr int64_t MOST_TOKENS = int64_t(1) << 26, MOST_CHANNELS = int64_t(1) << 23;

// Channels of a lane and wavefronts of a workgroup.  65543 binary16 tokens of 1024 channels, one channel a lane and two: forward 86 and 99 us, back 192 and 158, the maps of the way
// back 68 and 90.  Sixteen wavefronts of eight tokens are level.
constexpr int FOLD_CH = 1, SCAN_CH = 1;                      // back: channels_of
constexpr int FOLD_W = 8, SCAN_W = 8, BACK_W = 8;

// How the work is cut.
struct Cut {
    int mode;
    int64_t units, tokens, blocks, segments, per_segment;
};

// Sequences of up to EVEN_MOST tokens share a block.  Us together and each by itself, forward, back; 256 sequences of 1024 channels: 33 tokens, bfloat16 20 and 48,
// 50 and 87, binary32 27 and 48, 67 and 84; 64 tokens, bfloat16 27 and 43, 58 and 89, binary32 46 and 53, but 115 and 90; 65 tokens (a block each in both) bfloat16 45 and 42,
// 118 and 94, binary32 53 and 51, 129 and 88.  So the border is right but for the way back of binary32, whose is between 48 tokens (81 and 90) and 64.
constexpr int64_t EVEN_MOST = BLOCK / 2;
// Workgroups that are wanted.  Segments cost a launch and a second reading; 8 x 4096 tokens of 1024 bfloat16 channels whole, with 256, 512 and
// 1024 workgroups: forward 88, 76, 76, 74 us, back 198, 99, 103, 107; 65543 binary16 tokens 1315, 152, 158, 159 and 3272, 213, 235, 244.  Forward, few blocks are faster
// whole on half the compute units.  Whole and in segments, 1024 channels, us: 4 sequences of 512 tokens (64 workgroups) bfloat16 10.5 and 9.2, binary32 11.1 and 11.1; 7 of them (112)
// 11.1 and 12.7, 11.9 and 14.4; 8 (128) 11.2 and 12.9, 12.4 and 14.9; 16 (256) 12.7 and 18.3.  8 of 1024 (8 blocks) 18.6 and 18.9, 27.3 and 29.2; of 1152 (9 blocks) 20.5 and 20.4,
// 31 and 32; of 2048 39 and 35, 55 and 58.  With 192 workgroups and more, whole would be faster beyond 8 blocks, too: 12 of 2048 bfloat16 43 and 62.  Back, 8 of 512: bfloat16 22.8
// and 16.5, binary32 17.4 and 20.0.
constexpr int64_t FILL = 256, WHOLE_FILL = 128, WHOLE_BLOCKS = 8;

Cut cut_of(const mgwfbp_sequences& s, int64_t channels, int32_t dtype, bool back) {
    Cut c{};
    const int64_t length = s.d_offsets != nullptr ? s.n_tokens : s.n_tokens / s.n_sequences;
    c.mode = s.d_offsets != nullptr ? PACKED : length <= EVEN_MOST ? EVEN : ONE;
    const int64_t together = c.mode == EVEN ? std::max<int64_t>(1, BLOCK / std::max<int64_t>(length, 1)) : 1;
    c.units = c.mode == PACKED ? 1 : ceil_div(s.n_sequences, together);
    c.tokens = length * together;
    c.blocks = ceil_div(c.tokens, BLOCK);
    const int64_t slabs = ceil_div(channels, static_cast<int64_t>(LANES) * channels_of(dtype_bytes(dtype))), whole = c.units * slabs;
    c.segments = std::max<int64_t>(1, std::min(c.blocks, FILL / std::max<int64_t>(whole, 1)));
    if (!back && c.blocks <= WHOLE_BLOCKS && c.units * ceil_div(channels, LANES) >= WHOLE_FILL) c.segments = 1;
    c.per_segment = std::max<int64_t>(1, ceil_div(c.blocks, c.segments));
    c.segments = std::max<int64_t>(1, ceil_div(c.blocks, c.per_segment));
    return c;
}

bool sizes_ok(const mgwfbp_sequences* s, int64_t channels) {
    if (s == nullptr || s->n_sequences < 0 || s->n_sequences > MOST_TOKENS || s->n_tokens < 0 || s->n_tokens > MOST_TOKENS || channels < 0 || channels > MOST_CHANNELS)
        return false;
    if (s->d_offsets == nullptr) return s->n_sequences == 0 ? s->n_tokens == 0 : s->n_tokens % s->n_sequences == 0;
    return (s->offset_type == MGWFBP_I32 || s->offset_type == MGWFBP_I64) && is_aligned(s->d_offsets, s->offset_type == MGWFBP_I64 ? 8 : 4);
}
int64_t unit_tokens(const mgwfbp_sequences& s) { return s.d_offsets != nullptr ? s.n_tokens : s.n_sequences == 0 ? 0 : s.n_tokens / s.n_sequences; }
bool is_short(const mgwfbp_sequences& s) { return s.d_offsets == nullptr && unit_tokens(s) <= SHORT; }
bool is_kind(int32_t k) { return k == MGWFBP_RECUR_FREE || k == MGWFBP_RECUR_CONVEX || k == MGWFBP_RECUR_UNIT; }
bool side_ok(const void* p, int64_t tokens, int64_t channels, int64_t stride, int32_t dtype) {
    return tokens == 0 || (p != nullptr && is_aligned(p, dtype_bytes(dtype)) && is_matrix(tokens, channels, stride, dtype_bytes(dtype)));
}
bool states_ok(const float* p) { return is_aligned(p, 4); }

uint64_t workspace_of(const mgwfbp_sequences& s, int64_t channels, int32_t dtype) {
    if (s.n_sequences == 0 || channels == 0 || is_short(s)) return 0;
    uint64_t bytes = 0;
    for (const bool back : {false, true}) {
        const Cut c = cut_of(s, channels, dtype, back);
        if (c.segments > 1) bytes = std::max(bytes, static_cast<uint64_t>(c.units * c.segments * 2 * channels) * 4);
    }
    return bytes;
}

Span ends_span(const float* p, const mgwfbp_sequences& s, int64_t channels) { return vector_span(p, s.n_sequences * channels, 4); }
Span states_span(const float* p, const mgwfbp_sequences& s, int64_t channels) {
    return vector_span(p, (s.d_offsets != nullptr ? 1 : s.n_sequences) * ceil_div(unit_tokens(s), BLOCK) * channels, 4);
}
Span offsets_span(const mgwfbp_sequences& s) { return vector_span(s.d_offsets, s.n_sequences + 1, s.offset_type == MGWFBP_I64 ? 8 : 4); }

template <int K> struct Kind { static constexpr int value = K; };
template <typename F> int with_kind(int32_t kind, F&& f) {
    switch (kind) {
        case MGWFBP_RECUR_FREE: return f(Kind<MGWFBP_RECUR_FREE>());
        case MGWFBP_RECUR_CONVEX: return f(Kind<MGWFBP_RECUR_CONVEX>());
        case MGWFBP_RECUR_UNIT: return f(Kind<MGWFBP_RECUR_UNIT>());
        default: return MGWFBP_EINVAL;
    }
}

template <bool BACK> int run(const mgwfbp_sequences& s, int32_t kind, int32_t dtype, RecurArgs& a, void* workspace, uint64_t workspace_bytes, void* stream) {
    const int64_t channels = a.channels;
    a.sequences = s.n_sequences;
    a.tokens = a.length = unit_tokens(s);
    a.rows = s.n_tokens;
    a.offsets = s.d_offsets;
    a.offset_type = s.offset_type;
    if (is_short(s)) {
        const int64_t lanes = a.sequences * ceil_div(channels, BACK ? channels_of(dtype_bytes(dtype)) : VEC);
        const int64_t groups = ceil_div(lanes, SHORT_THREADS);
        if (groups >= (int64_t(1) << 31)) return MGWFBP_EINVAL;
        return with_dtype(dtype, [&](auto* type) {
            return with_kind(kind, [&](auto k) {
                typedef std::remove_pointer_t<decltype(type)> T;
                constexpr int K = decltype(k)::value;
                void (*kernel)(RecurArgs) = !BACK ? short_scan_kernel<T, K> : a.tokens <= SHORT / 2 ? short_back_kernel<T, K, SHORT / 2> : short_back_kernel<T, K, SHORT>;
                return launch(kernel, a, dim3(static_cast<uint32_t>(groups)), dim3(SHORT_THREADS), stream);
            });
        });
    }
    const Cut cut = cut_of(s, channels, dtype, BACK);
    a.tokens = cut.tokens;
    a.blocks = cut.blocks;
    a.segments = static_cast<uint32_t>(cut.segments);
    a.per_segment = static_cast<uint32_t>(cut.per_segment);
    if (cut.segments > 1) {
        if (workspace == nullptr || !is_aligned(workspace, 256) || workspace_bytes < workspace_of(s, channels, dtype)) return MGWFBP_EINVAL;
        a.maps = static_cast<float*>(workspace);
        a.copied = !BACK && cut.mode == ONE && a.first != nullptr && a.first == a.last;
    }
    return with_dtype(dtype, [&](auto* type) {
        return with_kind(kind, [&](auto k) {
            typedef std::remove_pointer_t<decltype(type)> T;
            constexpr int K = decltype(k)::value, FCH = FOLD_CH, FW = FOLD_W, SCH = BACK ? channels_of(sizeof(T)) : SCAN_CH, SW = BACK ? BACK_W : SCAN_W;
            auto start = [&](void (*one)(RecurArgs), void (*even)(RecurArgs), void (*packed)(RecurArgs), int ch, int waves) {
                a.slabs = static_cast<uint32_t>(ceil_div(channels, static_cast<int64_t>(LANES) * ch));
                const int64_t groups = cut.units * cut.segments * a.slabs;
                if (groups >= (int64_t(1) << 31)) return static_cast<int>(MGWFBP_EINVAL);
                return launch(cut.mode == PACKED ? packed : cut.mode == EVEN ? even : one, a, dim3(static_cast<uint32_t>(groups)), dim3(waves * LANES), stream);
            };
            if (cut.segments > 1) {
                const int status = start(fold_kernel<T, K, FCH, FW, ONE, BACK>, nullptr, fold_kernel<T, K, FCH, FW, PACKED, BACK>, FCH, FW);       // a unit of EVEN is a block
                if (status != MGWFBP_OK) return status;
            }
            if constexpr (BACK) return start(back_kernel<T, K, SCH, SW, ONE>, back_kernel<T, K, SCH, SW, EVEN>, back_kernel<T, K, SCH, SW, PACKED>, SCH, SW);
            else return start(scan_kernel<T, K, SCH, SW, ONE>, scan_kernel<T, K, SCH, SW, EVEN>, scan_kernel<T, K, SCH, SW, PACKED>, SCH, SW);
        });
    });
}

}  // namespace

extern "C" {

int mgwfbp_recur_states(const mgwfbp_sequences* sequences, int64_t* rows_out) {
    if (!sizes_ok(sequences, 0) || rows_out == nullptr) return MGWFBP_EINVAL;
    *rows_out = (sequences->d_offsets != nullptr ? 1 : sequences->n_sequences) * ceil_div(unit_tokens(*sequences), BLOCK);
    return MGWFBP_OK;
}

int mgwfbp_recur_workspace(const mgwfbp_sequences* sequences, int64_t n_channels, int32_t dtype, uint64_t* bytes_out) {
    if (!sizes_ok(sequences, n_channels) || !is_dtype(dtype) || bytes_out == nullptr) return MGWFBP_EINVAL;
    *bytes_out = workspace_of(*sequences, n_channels, dtype);
    return MGWFBP_OK;
}

int mgwfbp_recur(const mgwfbp_sequences* sequences, int64_t n_channels, int32_t kind, int32_t dtype, const void* d_gate, int64_t gate_stride,
                 const void* d_x, int64_t x_stride, const float* d_first, void* d_y, int64_t y_stride, float* d_last, float* d_states,
                 void* d_workspace, uint64_t workspace_bytes, void* hip_stream) {
    if (!sizes_ok(sequences, n_channels) || !is_dtype(dtype) || !is_kind(kind)) return MGWFBP_EINVAL;
    const int64_t tokens = sequences->n_tokens;
    if (sequences->n_sequences == 0 || n_channels == 0) return MGWFBP_OK;
    if (!side_ok(d_gate, tokens, n_channels, gate_stride, dtype) || !side_ok(d_x, tokens, n_channels, x_stride, dtype) ||
        !side_ok(d_y, tokens, n_channels, y_stride, dtype) || !states_ok(d_first) || !states_ok(d_last) || !states_ok(d_states) ||
        !is_matrix(sequences->n_sequences, n_channels, n_channels, 4))
        return MGWFBP_EINVAL;
    const int64_t bytes = dtype_bytes(dtype);
    const uint32_t Y = 1, LAST = 2;
    if (tangled({matrix_span(d_y, tokens, n_channels, y_stride, bytes), ends_span(d_last, *sequences, n_channels), states_span(d_states, *sequences, n_channels),
                 vector_span(d_workspace, static_cast<int64_t>(workspace_of(*sequences, n_channels, dtype)), 1)},
                {{matrix_span(d_gate, tokens, n_channels, gate_stride, bytes), Y},
                 {matrix_span(d_x, tokens, n_channels, x_stride, bytes), Y},
                 {ends_span(d_first, *sequences, n_channels), sequences->d_offsets == nullptr ? LAST : 0},
                 {offsets_span(*sequences), 0}}))
        return MGWFBP_EINVAL;
    RecurArgs a{};
    a.gate = d_gate;
    a.x = d_x;
    a.first = d_first;
    a.y = d_y;
    a.last = d_last;
    a.states = d_states;
    a.gate_stride = gate_stride;
    a.x_stride = x_stride;
    a.y_stride = y_stride;
    a.channels = n_channels;
    return run<false>(*sequences, kind, dtype, a, d_workspace, workspace_bytes, hip_stream);
}

int mgwfbp_recur_backward(const mgwfbp_sequences* sequences, int64_t n_channels, int32_t kind, int32_t dtype, const void* d_gate, int64_t gate_stride,
                          const void* d_x, int64_t x_stride, const float* d_first, const float* d_states, const void* d_dy, int64_t dy_stride,
                          const float* d_dlast, void* d_dgate, int64_t dgate_stride, void* d_dx, int64_t dx_stride, float* d_dfirst,
                          void* d_workspace, uint64_t workspace_bytes, void* hip_stream) {
    if (!sizes_ok(sequences, n_channels) || !is_dtype(dtype) || !is_kind(kind)) return MGWFBP_EINVAL;
    const int64_t tokens = sequences->n_tokens;
    if (sequences->n_sequences == 0 || n_channels == 0) return MGWFBP_OK;
    if (!side_ok(d_gate, tokens, n_channels, gate_stride, dtype) || !side_ok(d_x, tokens, n_channels, x_stride, dtype) ||
        !side_ok(d_dy, tokens, n_channels, dy_stride, dtype) || !side_ok(d_dgate, tokens, n_channels, dgate_stride, dtype) ||
        !side_ok(d_dx, tokens, n_channels, dx_stride, dtype) || !states_ok(d_first) || !states_ok(d_states) || !states_ok(d_dlast) || !states_ok(d_dfirst) ||
        (tokens > 0 && !is_short(*sequences) && d_states == nullptr) || !is_matrix(sequences->n_sequences, n_channels, n_channels, 4))
        return MGWFBP_EINVAL;
    const int64_t bytes = dtype_bytes(dtype);
    const uint32_t DGATE = 1, DX = 2;
    if (tangled({matrix_span(d_dgate, tokens, n_channels, dgate_stride, bytes), matrix_span(d_dx, tokens, n_channels, dx_stride, bytes),
                 ends_span(d_dfirst, *sequences, n_channels), vector_span(d_workspace, static_cast<int64_t>(workspace_of(*sequences, n_channels, dtype)), 1)},
                {{matrix_span(d_gate, tokens, n_channels, gate_stride, bytes), DGATE | DX},
                 {matrix_span(d_x, tokens, n_channels, x_stride, bytes), DGATE | DX},
                 {matrix_span(d_dy, tokens, n_channels, dy_stride, bytes), DGATE | DX},
                 {ends_span(d_first, *sequences, n_channels), 0},
                 {ends_span(d_dlast, *sequences, n_channels), 0},
                 {states_span(d_states, *sequences, n_channels), 0},
                 {offsets_span(*sequences), 0}}))
        return MGWFBP_EINVAL;
    RecurArgs a{};
    a.gate = d_gate;
    a.x = d_x;
    a.dy = d_dy;
    a.first = d_first;
    a.dlast = d_dlast;
    a.dgate = d_dgate;
    a.dx = d_dx;
    a.dfirst = d_dfirst;
    a.states = const_cast<float*>(d_states);
    a.gate_stride = gate_stride;
    a.x_stride = x_stride;
    a.dy_stride = dy_stride;
    a.dgate_stride = dgate_stride;
    a.dx_stride = dx_stride;
    a.channels = n_channels;
    return run<true>(*sequences, kind, dtype, a, d_workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
