// What the layer operators share (grem_layer_norm.hip, grem_checkpoint.hip, grem_neighbour_mean.hip, grem_linear.hip): the three
// value types, loads and stores of runs of values at any alignment, checkpoint groups, sums over lanes.
#ifndef GREM_LAYERS_HIP_H
#define GREM_LAYERS_HIP_H

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "grem.h"

namespace {

using bf16 = __bf16;
using f16 = _Float16;

// Rows up to 2^30 (a launch takes fewer than 2^32 threads), widths up to 2^20 values: a row's place is computed in 64 bits, a
// place inside it in 32.
constexpr int64_t kLayerMaxRows = 1 << 30;
constexpr int64_t kLayerMaxCols = 1 << 20;

// A run of V values at the alignment of one: the hardware takes vector loads at any multiple of the element, so odd strides and
// odd bases cost cache lines, not instructions.  It is loaded as whole words and taken apart afterwards: a run that may end
// early has two ways of being loaded, and values that meet from two ways one by one are waited for where they meet.
template <class T, int V> struct Words {
    static constexpr int bytes = V * (int)sizeof(T), count = bytes / 4;
    typedef uint32_t type __attribute__((ext_vector_type(count)));
    struct __attribute__((packed, aligned(alignof(T)))) Place {
        type w;
    };
};

template <class T, int V> using WordsOf = typename Words<T, V>::type;

// values [c, c + V) of a row of d, zero from d on; EVEN: V divides d, so that a run is whole or absent
template <class T, int V, bool EVEN> __device__ __forceinline__ WordsOf<T, V> load_words(const T* __restrict__ row, int c, int d)
{
    using W = Words<T, V>;
    if constexpr (EVEN) {
        typename W::type w = {};
        if (c < d) w = ((const typename W::Place*)(row + c))->w;
        return w;
    } else {
        if (c + V <= d) return ((const typename W::Place*)(row + c))->w;
        T v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = c + i < d ? row[c + i] : (T)0;
        typename W::type w;
        __builtin_memcpy(&w, v, W::bytes);
        return w;
    }
}

// a run that is known to be whole
template <class T, int V> __device__ __forceinline__ WordsOf<T, V> whole_words(const T* __restrict__ at)
{
    return ((const typename Words<T, V>::Place*)at)->w;
}

template <class T, int V> __device__ __forceinline__ void to_floats(const WordsOf<T, V>& w, float (&f)[V])
{
    T v[V];
    __builtin_memcpy(v, &w, Words<T, V>::bytes);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = (float)v[i];
}

template <class T, int V, bool EVEN = false> __device__ __forceinline__ void load_floats(const T* __restrict__ row, int c, int d, float (&f)[V])
{
    to_floats<T, V>(load_words<T, V, EVEN>(row, c, d), f);
}

// rounded to T, to nearest even: the one rounding of an output that is computed in 32 bits
template <class T, int V, bool EVEN = false> __device__ __forceinline__ void store_floats(T* __restrict__ row, int c, int d, const float (&f)[V])
{
    using W = Words<T, V>;
    T v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (T)f[i];
    if (EVEN || c + V <= d) {
        typename W::type w;
        __builtin_memcpy(&w, v, W::bytes);
        ((typename W::Place*)(row + c))->w = w;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (c + i < d) row[c + i] = v[i];
    }
}

// ---- checkpoint groups: 32 columns share an exponent, a value is code * 2^(byte - 130) ------------------------------
constexpr int kCkGroup = 32;
constexpr int kCkBias = 130;
constexpr int kCkNotFinite = 255;

// 2^(byte - 130), NaN for a group that is not finite (whose codes are 0): code * scale is the value, exactly
__device__ __forceinline__ float ck_scale(int byte)
{
    // 2^(byte - 130) has exponent field byte - 3; from 3 down it is a number below the normal ones
    const uint32_t bits = byte > 3 ? (uint32_t)(byte - 3) << 23 : 1u << (19 + byte);
    return __uint_as_float(byte == kCkNotFinite ? 0x7FC00000u : bits);
}

// Rows of values, or of a checkpoint's codes and exponent bytes.
struct Rows {
    const void* data;
    int64_t stride;
    const uint8_t* exponents;
    int64_t exponent_stride;
};

// A run of a row on its way: its words, and the exponent byte where it is a checkpoint's (V divides 32 and c is a multiple of V, so one
// serves the run).
template <class T, bool CK, int V> struct Held {
    WordsOf<T, V> w;
    template <bool EVEN> __device__ __forceinline__ void load(const Rows& x, int64_t r, int c, int d)
    {
        w = load_words<T, V, EVEN>((const T*)x.data + r * x.stride, c, d);
    }
    __device__ __forceinline__ void floats(float (&f)[V]) const { to_floats<T, V>(w, f); }
};

template <class T, int V> struct Held<T, true, V> {
    WordsOf<int8_t, V> w;
    int byte;
    template <bool EVEN> __device__ __forceinline__ void load(const Rows& x, int64_t r, int c, int d)
    {
        byte = kCkBias;
        if (c < d) byte = x.exponents[r * x.exponent_stride + c / kCkGroup];
        w = load_words<int8_t, V, EVEN>((const int8_t*)x.data + r * x.stride, c, d);
    }
    __device__ __forceinline__ void floats(float (&f)[V]) const
    {
        const float scale = ck_scale(byte);
        to_floats<int8_t, V>(w, f);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] *= scale;
    }
};

// sum over groups of W neighbouring lanes, in every lane of the group
template <int W> __device__ __forceinline__ float lanes_sum(float x)
{
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// ---- columns' sums ------------------------------------------------------------------------------------------------------
//
// What the workgroups of a pass over the rows leave, `parts` rows of `width` sums, is added up by workgroups of 1,024 threads that take 16
// columns each: 64 threads a column, then those in order (1,024 rows of 2,048 columns: 26 us with 256 threads, 6 with 1,024).
constexpr int kJoinBlock = 1024, kJoinCols = 16, kJoinSlices = kJoinBlock / kJoinCols;

// the total of column c in threads 0 .. 15; sums: kJoinSlices rows of kJoinCols + 1
__device__ __forceinline__ float join_columns(const float* __restrict__ partial, int parts, int64_t width, int64_t c, float (*sums)[kJoinCols + 1])
{
    const int slice = threadIdx.x / kJoinCols, col = threadIdx.x % kJoinCols;
    float s = 0.0f;
    if (c < width)
#pragma unroll 4
        for (int p = slice; p < parts; p += kJoinSlices) s += partial[(size_t)p * (size_t)width + c];
    sums[slice][col] = s;
    __syncthreads();
    float total = 0.0f;
    if (threadIdx.x < kJoinCols)
#pragma unroll
        for (int i = 0; i < kJoinSlices; ++i) total += sums[i][threadIdx.x];
    return total;
}

// ---- argument checks -------------------------------------------------------------------------------------------------
inline int layer_size(int32_t type) { return type == GREM_F32 ? 4 : type == GREM_BF16 || type == GREM_F16 ? 2 : 0; }

inline bool layer_rows_ok(const void* p, int64_t stride, int64_t n, int64_t d, int size)
{
    return n == 0 || (p && (uintptr_t)p % (uintptr_t)size == 0 && stride >= d);
}

// (null is aligned)
inline bool layer_aligned(const void* p, int to) { return (uintptr_t)p % (uintptr_t)to == 0; }

// a workspace of at least `need` bytes; one that is not needed is not looked at
inline int layer_space(const void* workspace, size_t bytes, size_t need)
{
    if (need == 0) return GREM_OK;
    if (!workspace || bytes < need) return GREM_ERR_NOMEM;
    return layer_aligned(workspace, 256) ? GREM_OK : GREM_ERR_ARG;
}

inline bool layer_ck_ok(const grem_rows* x, int64_t n, int64_t d)
{
    return n == 0 || (x->data && x->stride >= d && x->exponent_stride >= (d + kCkGroup - 1) / kCkGroup);
}

inline bool layer_source_ok(const grem_rows* x, int64_t n, int64_t d, int size)
{
    return x && (x->exponents ? layer_ck_ok(x, n, d) : layer_rows_ok(x->data, x->stride, n, d, size));
}

inline Rows layer_rows(const grem_rows* x) { return Rows{x->data, x->stride, x->exponents, x->exponent_stride}; }

inline int layer_launched() { return hipGetLastError() == hipSuccess ? GREM_OK : GREM_ERR_HIP; }

inline size_t layer_align(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// f(T{}) for the type's C++ type
template <class F> inline void layer_typed(int32_t type, F f)
{
    if (type == GREM_F32) f(float{});
    else if (type == GREM_BF16) f(bf16{});
    else f(f16{});
}

template <class F> inline void layer_either(bool even, F f)
{
    if (even) f(std::true_type{});
    else f(std::false_type{});
}

}  // namespace

#endif
