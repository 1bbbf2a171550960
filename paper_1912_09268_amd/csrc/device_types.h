// Element types of the training operators (embed.hip, act8.hip, act_linear.hip): what a mgwfbp_dtype is on the device,
// and vectors of eight elements that are loaded and stored at any element's address.  gfx950 executes accesses that
// are aligned to less than their size with the same 16-byte instructions, so no alignment needs a form of its own; the
// end of a row that is no multiple of eight is taken element by element.
#ifndef MGWFBP_DEVICE_TYPES_H
#define MGWFBP_DEVICE_TYPES_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "mgwfbp_layers.h"

namespace ops {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4e __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8e __attribute__((ext_vector_type(8), aligned(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8e __attribute__((ext_vector_type(8), aligned(2)));

constexpr int VEC = 8;   // elements that a lane takes at a time: 16 bytes of a 16-bit type

template <typename T> struct Vec8;
template <> struct Vec8<__bf16> { typedef bf16x8e type; };
template <> struct Vec8<_Float16> { typedef f16x8e type; };

// What eight elements are in memory, and as they are held between the load and the conversion.
template <typename T> struct Raw8 { typename Vec8<T>::type v; };
template <> struct Raw8<float> { f32x4e lo, hi; };

template <typename T> __device__ __forceinline__ Raw8<T> load8(const T* p) {
    Raw8<T> r;
    if constexpr (sizeof(T) == 4) {
        r.lo = *reinterpret_cast<const f32x4e*>(p);
        r.hi = *reinterpret_cast<const f32x4e*>(p + 4);
    } else {
        r.v = *reinterpret_cast<const typename Vec8<T>::type*>(p);
    }
    return r;
}

// The first n of eight elements, zeros behind them; nothing else is read.
template <typename T> __device__ __forceinline__ Raw8<T> load8(const T* p, int n) {
    if (n >= VEC) return load8(p);
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const T x = i < n ? p[i] : static_cast<T>(0.f);
        if constexpr (sizeof(T) == 4) {
            if (i < 4) r.lo[i] = x; else r.hi[i - 4] = x;
        } else {
            r.v[i] = x;
        }
    }
    return r;
}

template <typename T> __device__ __forceinline__ float get(const Raw8<T>& r, int i) {
    if constexpr (sizeof(T) == 4) return i < 4 ? r.lo[i] : r.hi[i - 4];
    else return static_cast<float>(r.v[i]);
}

// A binary32 result to T, nearest even.  For binary16 the compiler would put the last multiplication and the conversion into one
// instruction with one rounding, in one form of a kernel and not in another; results are binary32 first in all of them.
template <typename T> __device__ __forceinline__ T rounded(float x) {
    if constexpr (__is_same(T, _Float16)) asm("" : "+v"(x));
    return static_cast<T>(x);
}

// Eight results, rounded where T has 16 bits.
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&x)[VEC]) {
    if constexpr (sizeof(T) == 4) {
        const f32x4e lo = {x[0], x[1], x[2], x[3]}, hi = {x[4], x[5], x[6], x[7]};
        *reinterpret_cast<f32x4e*>(p) = lo;
        *reinterpret_cast<f32x4e*>(p + 4) = hi;
    } else {
        typename Vec8<T>::type v;
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = rounded<T>(x[i]);
        *reinterpret_cast<typename Vec8<T>::type*>(p) = v;
    }
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&x)[VEC], int n) {
    if (n >= VEC) return store8(p, x);
#pragma unroll
    for (int i = 0; i < VEC; ++i)
        if (i < n) p[i] = rounded<T>(x[i]);
}

// The first n of W results, W elements of T being 16 bytes or fewer; STREAM: past the caches.
template <bool STREAM = false, typename T, int W> __device__ __forceinline__ void store_some(T* p, const float (&x)[W], int n) {
    if (n >= W) {
        typedef T vec __attribute__((ext_vector_type(W), aligned(alignof(T))));
        vec v;
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = rounded<T>(x[i]);
        if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<vec*>(p));
        else *reinterpret_cast<vec*>(p) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < W; ++i)
        if (i < n) p[i] = rounded<T>(x[i]);
}

// ---- host side -------------------------------------------------------------------------------

inline bool is_dtype(int32_t t) { return t == MGWFBP_F32 || t == MGWFBP_BF16 || t == MGWFBP_F16; }
inline int64_t dtype_bytes(int32_t t) { return t == MGWFBP_F32 ? 4 : 2; }

// Calls f with a null pointer to the element type of dtype t.
template <typename F> int with_dtype(int32_t t, F&& f) {
    switch (t) {
        case MGWFBP_F32: return f(static_cast<float*>(nullptr));
        case MGWFBP_BF16: return f(static_cast<__bf16*>(nullptr));
        case MGWFBP_F16: return f(static_cast<_Float16*>(nullptr));
        default: return MGWFBP_EINVAL;
    }
}

// A matrix of `rows` rows that start `stride` elements apart and hold `width` elements: its last byte has an offset that
// fits 62 bits, so that no address computed from it wraps.
inline bool is_matrix(int64_t rows, int64_t width, int64_t stride, int64_t elem_bytes) {
    if (rows < 0 || width < 0) return false;
    if (rows == 0 || width == 0) return true;
    if (rows > 1 && stride < width) return false;
    if (width > (int64_t(1) << 40)) return false;
    return rows <= 1 || (stride <= (int64_t(1) << 40) && rows <= (int64_t(1) << 59) / (stride * elem_bytes));
}
inline bool is_aligned(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0; }

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Records a failed HIP call for mgwfbp_layers_last_hip_error() on this thread.
int note(hipError_t e);

// Launch of `kernel` with its one argument structure.
template <typename A> int launch(void (*kernel)(A), const A& args, dim3 grid, dim3 block, void* stream) {
    void* list[] = {const_cast<A*>(&args)};
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, list, 0, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) (void)hipGetLastError();        // reported here, not to whoever asks next
    return note(e);
}

}  // namespace ops

#endif
