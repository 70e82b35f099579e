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
// odd bases cost cache lines, not instructions.
template <class T, int V> struct __attribute__((packed, aligned(alignof(T)))) Run { T v[V]; };

template <class T, int V> __device__ __forceinline__ void load_run(const T* __restrict__ p, T (&v)[V])
{
    const Run<T, V> r = *(const Run<T, V>*)p;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = r.v[i];
}

template <class T, int V> __device__ __forceinline__ void store_run(T* __restrict__ p, const T (&v)[V])
{
    Run<T, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) r.v[i] = v[i];
    *(Run<T, V>*)p = r;
}

// values [c, c + V) of a row of d, as floats; zero from d on
template <class T, int V> __device__ __forceinline__ void load_floats(const T* __restrict__ row, int c, int d, float (&f)[V])
{
    T v[V];
    if (c + V <= d) {
        load_run<T, V>(row + c, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = c + i < d ? row[c + i] : (T)0.0f;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = (float)v[i];
}

// rounded to T, to nearest even: the one rounding of an output that is computed in 32 bits
template <class T, int V> __device__ __forceinline__ void store_floats(T* __restrict__ row, int c, int d, const float (&f)[V])
{
    T v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (T)f[i];
    if (c + V <= d) {
        store_run<T, V>(row + c, v);
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

__device__ __forceinline__ float ck_value(int code, int byte)
{
    return byte == kCkNotFinite ? __builtin_nanf("") : ldexpf((float)code, byte - kCkBias);
}

// Rows of values, or of a checkpoint's codes and exponent bytes.
struct Rows {
    const void* data;
    int64_t stride;
    const uint8_t* exponents;
    int64_t exponent_stride;
};

// values [c, c + V) of row r, in floats; V divides 32 and c is a multiple of V, so one exponent serves them all
template <class T, bool CK, int V> __device__ __forceinline__ void load_row(const Rows& x, int64_t r, int c, int d, float (&f)[V])
{
    if constexpr (!CK) {
        load_floats<T, V>((const T*)x.data + r * x.stride, c, d, f);
    } else {
        if (c >= d) {
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = 0.0f;
            return;
        }
        const int byte = x.exponents[r * x.exponent_stride + c / kCkGroup];
        float q[V];
        load_floats<int8_t, V>((const int8_t*)x.data + r * x.stride, c, d, q);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = c + i < d ? ck_value((int)q[i], byte) : 0.0f;
    }
}

// sum over groups of W neighbouring lanes, in every lane of the group
template <int W> __device__ __forceinline__ float lanes_sum(float x)
{
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// ---- argument checks -------------------------------------------------------------------------------------------------
inline int layer_size(int32_t type) { return type == GREM_F32 ? 4 : type == GREM_BF16 || type == GREM_F16 ? 2 : 0; }

inline bool layer_rows_ok(const void* p, int64_t stride, int64_t n, int64_t d, int size)
{
    return n == 0 || (p && (uintptr_t)p % (uintptr_t)size == 0 && stride >= d);
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

}  // namespace

#endif
