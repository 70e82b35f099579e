// Activation checkpoints in 8 bits, for gfx950: rows of values in groups of 32 columns, a group kept as 32 codes of 8 bits
// and one byte for its exponent.
//   e = the least whole number with |x| <= 127 * 2^e in the group, in [-130, 122];  code = x / 2^e to the nearest, ties to even
//   value = code * 2^e
// The scale is a power of two: x / 2^e is exact, so the codes are the same whatever the precision they are found in, and
// code * 2^e has at most 7 significant bits: it is exact in bfloat16 and, in its normal range, in half precision.  A matrix product takes
// a checkpoint as it stands, with no second rounding.  (A scale of absmax / 127 would be up to one bit finer and would round again
// when it is multiplied out.)
//
// Bound by memory: eight columns a thread, whole rows a workgroup.  1M x 256 bfloat16 there and back: 314 us, 5.2 TB/s (a copy: 4.9-5.4).
#include "grem_layers.hip.h"

namespace {

constexpr int kCkBlock = 256;
constexpr int kCkPer = 8;                       // columns a thread: four lanes make a group

// bits of the largest |x|: the exponent byte; 255 where a NaN or an infinity is among them
__device__ __forceinline__ int ck_byte(uint32_t most)
{
    if (most >= 0x7F800000u) return kCkNotFinite;
    const int e = (int)(most >> 23) - 126 - 7 + ((most & 0x7FFFFFu) > 0x7E0000u ? 1 : 0);       // 1.mantissa > 2 * 127/128
    return (e < -kCkBias ? -kCkBias : e) + kCkBias;
}

// At the last binade of the type 64 * 2^e would be its 2^(largest exponent + 1): the codes stop at 63.
template <class T> constexpr int ck_top() { return (__is_same(T, f16) ? 10 : 122) + kCkBias; }

template <class T, bool EVEN>
__global__ __launch_bounds__(kCkBlock) void k_ck_pack(const T* __restrict__ x, int64_t ldx, int64_t n, int d, uint32_t per_row,
                                                      uint32_t rows, int8_t* __restrict__ codes, int64_t ldc,
                                                      uint8_t* __restrict__ exponents, int64_t lde)
{
    const int64_t first = (int64_t)blockIdx.x * rows;
    const uint32_t here = n - first < rows ? (uint32_t)(n - first) : rows;
    const uint32_t items = (here * per_row + 63u) & ~63u;              // whole waves: the groups' lanes work together
    for (uint32_t i = threadIdx.x; i < items; i += kCkBlock) {
        const uint32_t q = i / per_row, r = q < here ? q : here - 1;
        const int c = (int)(i - q * per_row) * kCkPer;
        float f[kCkPer];
        load_floats<T, kCkPer, EVEN>(x + (first + r) * ldx, c, d, f);
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < kCkPer; ++j) {
            const uint32_t b = __float_as_uint(f[j]) & 0x7FFFFFFFu;
            most = most > b ? most : b;
        }
        uint32_t other = (uint32_t)__shfl_xor((int)most, 1);
        most = most > other ? most : other;
        other = (uint32_t)__shfl_xor((int)most, 2);
        most = most > other ? most : other;
        if (q >= here) continue;
        const int byte = ck_byte(most);
        if ((i & 3u) == 0u && c < d) exponents[(first + r) * lde + c / kCkGroup] = (uint8_t)byte;
        const float limit = byte == ck_top<T>() ? 63.0f : 127.0f;
        float code[kCkPer];
#pragma unroll
        for (int j = 0; j < kCkPer; ++j) {
            const float v = rintf(ldexpf(f[j], kCkBias - byte));
            code[j] = byte == kCkNotFinite ? 0.0f : fminf(fmaxf(v, -limit), limit);
        }
        if (c < d) store_floats<int8_t, kCkPer, EVEN>(codes + (first + r) * ldc, c, d, code);
    }
}

template <class T, bool EVEN>
__global__ __launch_bounds__(kCkBlock) void k_ck_unpack(Rows x, int64_t n, int d, uint32_t per_row, uint32_t rows,
                                                        T* __restrict__ y, int64_t ldy)
{
    const int64_t first = (int64_t)blockIdx.x * rows;
    const uint32_t here = n - first < rows ? (uint32_t)(n - first) : rows;
    for (uint32_t i = threadIdx.x; i < here * per_row; i += kCkBlock) {
        const uint32_t r = i / per_row;
        const int c = (int)(i - r * per_row) * kCkPer;
        Held<T, true, kCkPer> h;
        h.template load<EVEN>(x, first + r, c, d);
        float f[kCkPer];
        h.floats(f);
        if (c < d) store_floats<T, kCkPer, EVEN>(y + (first + r) * ldy, c, d, f);
    }
}

// rows of a workgroup: about 4,096 runs of 8 columns, whole rows, and at most what 2^31 workgroups need
struct CkShape {
    uint32_t per_row, rows, grid;
};

CkShape ck_shape(int64_t n, int64_t d)
{
    CkShape s;
    s.per_row = (uint32_t)((d + kCkGroup - 1) / kCkGroup) * (kCkGroup / kCkPer);
    s.rows = s.per_row >= 4096 ? 1 : 4096 / s.per_row;
    while (s.rows > 1 && (n + s.rows - 1) / s.rows < 2048) s.rows = (s.rows + 1) / 2;
    s.grid = (uint32_t)((n + s.rows - 1) / s.rows);
    return s;
}

}  // namespace

extern "C" int grem_checkpoint_pack(int32_t type, int64_t n, int64_t d, const void* x, int64_t ldx, int8_t* codes, int64_t ldc,
                                    uint8_t* exponents, int64_t lde, void* stream)
{
    const int size = layer_size(type);
    if (!size || n < 0 || n > kLayerMaxRows || d < 1 || d > kLayerMaxCols || !layer_rows_ok(x, ldx, n, d, size) ||
        !layer_rows_ok(codes, ldc, n, d, 1) || !layer_rows_ok(exponents, lde, n, (d + kCkGroup - 1) / kCkGroup, 1))
        return GREM_ERR_ARG;
    if (n == 0) return GREM_OK;
    const CkShape s = ck_shape(n, d);
    layer_typed(type, [&](auto t) {
        using T = decltype(t);
        layer_either(d % kCkPer == 0, [&](auto even) {
            hipLaunchKernelGGL((k_ck_pack<T, decltype(even)::value>), dim3(s.grid), dim3(kCkBlock), 0, (hipStream_t)stream, (const T*)x, ldx, n,
                               (int)d, s.per_row, s.rows, codes, ldc, exponents, lde);
        });
    });
    return layer_launched();
}

extern "C" int grem_checkpoint_unpack(int32_t type, int64_t n, int64_t d, const grem_rows* x, void* y, int64_t ldy, void* stream)
{
    const int size = layer_size(type);
    if (!size || n < 0 || n > kLayerMaxRows || d < 1 || d > kLayerMaxCols || !x || (n && !x->exponents) || !layer_ck_ok(x, n, d) ||
        !layer_rows_ok(y, ldy, n, d, size))
        return GREM_ERR_ARG;
    if (n == 0) return GREM_OK;
    const CkShape s = ck_shape(n, d);
    layer_typed(type, [&](auto t) {
        using T = decltype(t);
        layer_either(d % kCkPer == 0, [&](auto even) {
            hipLaunchKernelGGL((k_ck_unpack<T, decltype(even)::value>), dim3(s.grid), dim3(kCkBlock), 0, (hipStream_t)stream, layer_rows(x), n,
                               (int)d, s.per_row, s.rows, (T*)y, ldy);
        });
    });
    return layer_launched();
}
