// Layer norm over the rows of an (n, d) matrix and its backward pass, for gfx950.
//   mu = sum x / d,  r = 1 / sqrt(sum (x - mu)^2 / d + eps),  xh = (x - mu) r,  y = xh * gamma + beta
//   t = dy * gamma,  dx = r (t - sum t / d - xh * sum (t xh) / d),  dgamma = sum over rows of dy * xh,  dbeta = of dy
// Everything is held in 32 bits; an output is rounded to its type once.
//
// Both passes are bound by memory (a dozen operations a value).  A group of L lanes (16, 32, 64 or the 256 of a workgroup, the fewest that
// hold a row in at most 4 runs of 16 bytes a lane) takes a row, keeps it in registers, and the variance is summed about the mean: x is read
// once and no digits cancel.  The backward pass walks rows with the columns' two sums in registers, too; a workgroup leaves one partial row of
// each, and k_ln_join adds those in a fixed order (no atomics: the same bytes on every run).
// 1M x 256 bfloat16: 221 to 244 us from one way of timing to another, 4.9 to 4.4 TB/s; the backward pass of 262,144 x 1,024 from 8 bits 262 to 268 us,
// 5.2 to 5.0 TB/s (a copy: 4.9-5.4).
#include "grem_layers.hip.h"

namespace {

constexpr int kLnBlock = 256;
// Workgroups of the backward pass, at most; each leaves 8d bytes.  Three a CU where a row fills a wave or more (1,024 of them end in a second
// round that is mostly empty, 301 us for 280 at 262,144 x 1,024); narrow rows are few bytes a wave and need eight a CU under way
// (500,000 x 100: 111 us for 124; 1M x 256 would lose by them, 326 us for 288).
constexpr int64_t kLnNarrow = 128;
constexpr int ln_groups(int64_t d) { return d <= kLnNarrow ? 2048 : 768; }

template <class T> constexpr int kLnV = 16 / (int)sizeof(T);

// Sum over the L lanes that share a row; sums: a word per wave.  Two sets that take turns: whoever writes one has passed the barrier of
// the other, and so has everyone who still read the one.
template <int L> __device__ __forceinline__ float ln_sum(float x, float* sums)
{
    if constexpr (L <= 64) {
        return lanes_sum<L>(x);
    } else {
        x = lanes_sum<64>(x);
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = x;
        __syncthreads();
        return sums[0] + sums[1] + sums[2] + sums[3];
    }
}

template <class T, int V, bool EVEN = false> __device__ __forceinline__ void ln_param(const T* __restrict__ p, int c, int d, float none, float (&f)[V])
{
    if (p) {
        load_floats<T, V, EVEN>(p, c, d, f);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = none;
    }
}

template <class T, bool EVEN, int L, int C>
__global__ __launch_bounds__(kLnBlock) void k_ln_forward(const T* __restrict__ x, int64_t ldx, int64_t n, int d,
                                                         const T* __restrict__ gamma, const T* __restrict__ beta, float eps,
                                                         T* __restrict__ y, int64_t ldy, float* __restrict__ mean,
                                                         float* __restrict__ rstd)
{
    constexpr int V = kLnV<T>;
    __shared__ float sums[2][4];
    const int lane = threadIdx.x % L;
    for (int64_t base = (int64_t)blockIdx.x * (kLnBlock / L); base < n; base += (int64_t)gridDim.x * (kLnBlock / L)) {
        const int64_t row = base + threadIdx.x / L;
        const int64_t r = row < n ? row : n - 1;
        WordsOf<T, V> w[C];
#pragma unroll
        for (int k = 0; k < C; ++k) w[k] = load_words<T, V, EVEN>(x + r * ldx, (k * L + lane) * V, d);
        float f[C][V];
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < C; ++k) {
            to_floats<T, V>(w[k], f[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) s += f[k][i];
        }
        const float mu = ln_sum<L>(s, sums[0]) / (float)d;
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < C; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                f[k][i] -= mu;
                s += (k * L + lane) * V + i < d ? f[k][i] * f[k][i] : 0.0f;
            }
        const float rs = 1.0f / sqrtf(ln_sum<L>(s, sums[1]) / (float)d + eps);
        if (row >= n) continue;
        if (lane == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = rs;
        }
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const int c = (k * L + lane) * V;
            if (c >= d) continue;
            float g[V], b[V];
            ln_param<T, V, EVEN>(gamma, c, d, 1.0f, g);
            ln_param<T, V, EVEN>(beta, c, d, 0.0f, b);
#pragma unroll
            for (int i = 0; i < V; ++i) f[k][i] = f[k][i] * rs * g[i] + b[i];
            store_floats<T, V, EVEN>(y + row * ldy, c, d, f[k]);
        }
    }
}

// rows too wide for registers: a workgroup a row, three walks over it (the second and third from the caches)
template <class T>
__global__ __launch_bounds__(kLnBlock) void k_ln_forward_wide(const T* __restrict__ x, int64_t ldx, int64_t n, int d,
                                                              const T* __restrict__ gamma, const T* __restrict__ beta, float eps,
                                                              T* __restrict__ y, int64_t ldy, float* __restrict__ mean,
                                                              float* __restrict__ rstd)
{
    constexpr int V = kLnV<T>;
    __shared__ float sums[2][4];
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T* in = x + row * ldx;
        float s = 0.0f;
        for (int c = threadIdx.x * V; c < d; c += kLnBlock * V) {
            float f[V];
            load_floats<T, V>(in, c, d, f);
#pragma unroll
            for (int i = 0; i < V; ++i) s += f[i];
        }
        const float mu = ln_sum<kLnBlock>(s, sums[0]) / (float)d;
        s = 0.0f;
        for (int c = threadIdx.x * V; c < d; c += kLnBlock * V) {
            float f[V];
            load_floats<T, V>(in, c, d, f);
#pragma unroll
            for (int i = 0; i < V; ++i) s += c + i < d ? (f[i] - mu) * (f[i] - mu) : 0.0f;
        }
        const float rs = 1.0f / sqrtf(ln_sum<kLnBlock>(s, sums[1]) / (float)d + eps);
        if (threadIdx.x == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = rs;
        }
        for (int c = threadIdx.x * V; c < d; c += kLnBlock * V) {
            float f[V], g[V], b[V];
            load_floats<T, V>(in, c, d, f);
            ln_param<T, V>(gamma, c, d, 1.0f, g);
            ln_param<T, V>(beta, c, d, 0.0f, b);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = (f[i] - mu) * rs * g[i] + b[i];
            store_floats<T, V>(y + row * ldy, c, d, f);
        }
    }
}

// partial: per workgroup d sums of dy * xh, then d sums of dy
template <class T, bool CK, bool EVEN, int L, int C>
__global__ __launch_bounds__(kLnBlock) void k_ln_backward(const T* __restrict__ dy, int64_t lddy, Rows x, int64_t n, int d,
                                                          const float* __restrict__ mean, const float* __restrict__ rstd,
                                                          const T* __restrict__ gamma, T* __restrict__ dx, int64_t lddx,
                                                          float* __restrict__ partial)
{
    constexpr int V = kLnV<T>, R = kLnBlock / L;
    __shared__ float sums[2][4];
    __shared__ float columns[R > 1 ? (R - 1) * L * C * V : 1];
    const int lane = threadIdx.x % L, slot = threadIdx.x / L;
    float g[C][V], dg[C][V], db[C][V];
#pragma unroll
    for (int k = 0; k < C; ++k) {
        ln_param<T, V>(gamma, (k * L + lane) * V, d, 1.0f, g[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) dg[k][i] = db[k][i] = 0.0f;
    }
    for (int64_t base = (int64_t)blockIdx.x * R; base < n; base += (int64_t)gridDim.x * R) {
        const int64_t row = base + slot, r = row < n ? row : n - 1;
        const float mu = mean[r], rs = rstd[r];
        WordsOf<T, V> wt[C];
        Held<T, CK, V> wx[C];
#pragma unroll
        for (int k = 0; k < C; ++k) {
            wt[k] = load_words<T, V, EVEN>(dy + r * lddy, (k * L + lane) * V, d);
            wx[k].template load<EVEN>(x, r, (k * L + lane) * V, d);
        }
        float xh[C][V], t[C][V];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const int c = (k * L + lane) * V;
            to_floats<T, V>(wt[k], t[k]);
            wx[k].floats(xh[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xh[k][i] = c + i < d ? (xh[k][i] - mu) * rs : 0.0f;
                if (row < n) {
                    dg[k][i] += t[k][i] * xh[k][i];
                    db[k][i] += t[k][i];
                }
                t[k][i] *= g[k][i];
                s1 += t[k][i];
                s2 += t[k][i] * xh[k][i];
            }
        }
        s1 = ln_sum<L>(s1, sums[0]) / (float)d;
        s2 = ln_sum<L>(s2, sums[1]) / (float)d;
        if (row >= n) continue;
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const int c = (k * L + lane) * V;
            if (c >= d) continue;
#pragma unroll
            for (int i = 0; i < V; ++i) t[k][i] = rs * (t[k][i] - s1 - xh[k][i] * s2);
            if (dx) store_floats<T, V, EVEN>(dx + row * lddx, c, d, t[k]);
        }
    }
    if (!partial) return;
    // the workgroup's rows, slot by slot
    float* out = partial + (size_t)blockIdx.x * 2 * (size_t)d;
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        if constexpr (R > 1) {
            __syncthreads();
            if (slot > 0)
#pragma unroll
                for (int k = 0; k < C; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) columns[((slot - 1) * L + lane) * (C * V) + k * V + i] = which ? db[k][i] : dg[k][i];
            __syncthreads();
        }
        if (slot > 0) continue;
#pragma unroll
        for (int k = 0; k < C; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (k * L + lane) * V + i;
                float v = which ? db[k][i] : dg[k][i];
                if constexpr (R > 1)
                    for (int q = 0; q < R - 1; ++q) v += columns[(q * L + lane) * (C * V) + k * V + i];
                if (c < d) out[which * (size_t)d + c] = v;
            }
    }
}

// rows too wide for registers: dx, a workgroup a row
template <class T, bool CK>
__global__ __launch_bounds__(kLnBlock) void k_ln_backward_wide(const T* __restrict__ dy, int64_t lddy, Rows x, int64_t n, int d,
                                                               const float* __restrict__ mean, const float* __restrict__ rstd,
                                                               const T* __restrict__ gamma, T* __restrict__ dx, int64_t lddx)
{
    constexpr int V = kLnV<T>;
    __shared__ float sums[2][4];
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const float mu = mean[row], rs = rstd[row];
        float s1 = 0.0f, s2 = 0.0f;
        auto pair = [&](int c, float (&t)[V], float (&xh)[V]) {
            float g[V];
            load_floats<T, V>(dy + row * lddy, c, d, t);
            Held<T, CK, V> h;
            h.template load<false>(x, row, c, d);
            h.floats(xh);
            ln_param<T, V>(gamma, c, d, 1.0f, g);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xh[i] = c + i < d ? (xh[i] - mu) * rs : 0.0f;
                t[i] *= g[i];
            }
        };
        for (int c = threadIdx.x * V; c < d; c += kLnBlock * V) {
            float t[V], xh[V];
            pair(c, t, xh);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s1 += c + i < d ? t[i] : 0.0f;
                s2 += t[i] * xh[i];
            }
        }
        s1 = ln_sum<kLnBlock>(s1, sums[0]) / (float)d;
        s2 = ln_sum<kLnBlock>(s2, sums[1]) / (float)d;
        for (int c = threadIdx.x * V; c < d; c += kLnBlock * V) {
            float t[V], xh[V];
            pair(c, t, xh);
#pragma unroll
            for (int i = 0; i < V; ++i) t[i] = rs * (t[i] - s1 - xh[i] * s2);
            store_floats<T, V>(dx + row * lddx, c, d, t);
        }
    }
}

// ... and the columns' sums: a workgroup takes kLnBlock runs of columns and every gridDim.y-th row
template <class T, bool CK>
__global__ __launch_bounds__(kLnBlock) void k_ln_columns_wide(const T* __restrict__ dy, int64_t lddy, Rows x, int64_t n, int d,
                                                              const float* __restrict__ mean, const float* __restrict__ rstd,
                                                              float* __restrict__ partial)
{
    constexpr int V = kLnV<T>;
    const int c = (int)(blockIdx.x * kLnBlock + threadIdx.x) * V;
    if (c >= d) return;
    float dg[V], db[V];
#pragma unroll
    for (int i = 0; i < V; ++i) dg[i] = db[i] = 0.0f;
    for (int64_t r = blockIdx.y; r < n; r += gridDim.y) {
        const float mu = mean[r], rs = rstd[r];
        float t[V], xh[V];
        load_floats<T, V>(dy + r * lddy, c, d, t);
        Held<T, CK, V> h;
        h.template load<false>(x, r, c, d);
        h.floats(xh);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            dg[i] += t[i] * ((xh[i] - mu) * rs);
            db[i] += t[i];
        }
    }
    float* out = partial + (size_t)blockIdx.y * 2 * (size_t)d;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (c + i < d) {
            out[c + i] = dg[i];
            out[(size_t)d + c + i] = db[i];
        }
}

// partial: rows of d sums for gamma and d for beta
template <class T>
__global__ __launch_bounds__(kJoinBlock) void k_ln_join(const float* __restrict__ partial, int parts, int d, T* __restrict__ dgamma,
                                                        T* __restrict__ dbeta)
{
    __shared__ float sums[kJoinSlices][kJoinCols + 1];
    const int64_t c = (int64_t)blockIdx.x * kJoinCols + threadIdx.x % kJoinCols;
    const float total = join_columns(partial, parts, 2 * (int64_t)d, c, sums);
    if (threadIdx.x >= kJoinCols || c >= 2 * (int64_t)d) return;
    if (c < d) {
        if (dgamma) dgamma[c] = (T)total;
    } else {
        if (dbeta) dbeta[c - d] = (T)total;
    }
}

// (a launch takes fewer than 2^32 threads)
unsigned ln_grid(int64_t groups) { return (unsigned)(groups < (1 << 22) ? groups : 1 << 22); }

struct LnL16 { static constexpr int L = 16, C = 1; };
struct LnL32 { static constexpr int L = 32, C = 1; };
struct LnL64 { static constexpr int L = 64, C = 1; };
struct LnL64x2 { static constexpr int L = 64, C = 2; };
struct LnL64x4 { static constexpr int L = 64, C = 4; };
struct LnL256x2 { static constexpr int L = 256, C = 2; };
struct LnL256x4 { static constexpr int L = 256, C = 4; };

// f(shape) for the smallest shape that holds a row of d values in registers; false if none does
template <class T, class F> bool ln_shaped(int64_t d, F f)
{
    constexpr int V = kLnV<T>;
    if (d <= 16 * V) f(LnL16{});
    else if (d <= 32 * V) f(LnL32{});
    else if (d <= 64 * V) f(LnL64{});
    else if (d <= 128 * V) f(LnL64x2{});
    else if (d <= 256 * V) f(LnL64x4{});
    else if (d <= 512 * V) f(LnL256x2{});
    else if (d <= 1024 * V) f(LnL256x4{});
    else return false;
    return true;
}

}  // namespace

extern "C" int grem_layer_norm(int32_t type, int64_t n, int64_t d, const void* x, int64_t ldx, const void* gamma, const void* beta,
                               double eps, void* y, int64_t ldy, float* mean, float* rstd, void* stream_)
{
    const int size = layer_size(type);
    if (!size || n < 0 || n > kLayerMaxRows || d < 1 || d > kLayerMaxCols || !(eps >= 0.0) || !layer_rows_ok(x, ldx, n, d, size) ||
        !layer_rows_ok(y, ldy, n, d, size) || (uintptr_t)gamma % size || (uintptr_t)beta % size ||
        !layer_aligned(mean, 4) || !layer_aligned(rstd, 4))
        return GREM_ERR_ARG;
    if (n == 0) return GREM_OK;
    hipStream_t stream = (hipStream_t)stream_;
    layer_typed(type, [&](auto t) {
        using T = decltype(t);
        const bool held = ln_shaped<T>(d, [&](auto shape) {
            constexpr int L = decltype(shape)::L, C = decltype(shape)::C;
            layer_either(d % kLnV<T> == 0, [&](auto even) {
                hipLaunchKernelGGL((k_ln_forward<T, decltype(even)::value, L, C>), dim3(ln_grid((n * L + kLnBlock - 1) / kLnBlock)),
                                   dim3(kLnBlock), 0, stream, (const T*)x, ldx, n, (int)d, (const T*)gamma, (const T*)beta, (float)eps, (T*)y,
                                   ldy, mean, rstd);
            });
        });
        if (!held)
            hipLaunchKernelGGL((k_ln_forward_wide<T>), dim3(ln_grid(n)), dim3(kLnBlock), 0, stream, (const T*)x, ldx, n, (int)d,
                               (const T*)gamma, (const T*)beta, (float)eps, (T*)y, ldy, mean, rstd);
    });
    return layer_launched();
}

extern "C" size_t grem_layer_norm_backward_bytes(int64_t n, int64_t d)
{
    if (n < 0 || n > kLayerMaxRows || d < 1 || d > kLayerMaxCols) return 0;
    return layer_align((size_t)(n < ln_groups(d) ? n : ln_groups(d)) * 2 * (size_t)d * sizeof(float));
}

extern "C" int grem_layer_norm_backward(int32_t type, int64_t n, int64_t d, const void* dy, int64_t lddy, const grem_rows* x,
                                        const float* mean, const float* rstd, const void* gamma, void* dx, int64_t lddx,
                                        void* dgamma, void* dbeta, void* workspace, size_t workspace_bytes, void* stream_)
{
    const int size = layer_size(type);
    if (!size || n < 0 || n > kLayerMaxRows || d < 1 || d > kLayerMaxCols || !layer_rows_ok(dy, lddy, n, d, size) ||
        !layer_source_ok(x, n, d, size) || (n && (!mean || !rstd)) || (dx && !layer_rows_ok(dx, lddx, n, d, size)) ||
        (uintptr_t)gamma % size || (uintptr_t)dgamma % size || (uintptr_t)dbeta % size || !layer_aligned(mean, 4) || !layer_aligned(rstd, 4))
        return GREM_ERR_ARG;
    const bool params = dgamma || dbeta;
    if (!dx && !params) return GREM_OK;
    if (n == 0 && !params) return GREM_OK;
    if (const int rc = layer_space(workspace, workspace_bytes, params ? grem_layer_norm_backward_bytes(n, d) : 0)) return rc;
    hipStream_t stream = (hipStream_t)stream_;
    float* partial = params ? (float*)workspace : nullptr;
    layer_typed(type, [&](auto t) {
        using T = decltype(t);
        auto run = [&](auto packed) {
            constexpr bool CK = decltype(packed)::value;
            int parts = (int)(n < ln_groups(d) ? n : ln_groups(d));
            if (n) {
                const bool held = ln_shaped<T>(d, [&](auto shape) {
                    constexpr int L = decltype(shape)::L, C = decltype(shape)::C;
                    const int64_t groups = (n * L + kLnBlock - 1) / kLnBlock;
                    parts = (int)(groups < ln_groups(d) ? groups : ln_groups(d));
                    layer_either(d % kLnV<T> == 0, [&](auto even) {
                        hipLaunchKernelGGL((k_ln_backward<T, CK, decltype(even)::value, L, C>), dim3((unsigned)parts), dim3(kLnBlock), 0, stream,
                                           (const T*)dy, lddy, layer_rows(x), n, (int)d, mean, rstd, (const T*)gamma, (T*)dx, lddx, partial);
                    });
                });
                if (!held && dx)
                    hipLaunchKernelGGL((k_ln_backward_wide<T, CK>), dim3(ln_grid(n)), dim3(kLnBlock), 0, stream, (const T*)dy, lddy,
                                       layer_rows(x), n, (int)d, mean, rstd, (const T*)gamma, (T*)dx, lddx);
                if (!held && params) {
                    if (parts > 256) parts = 256;
                    hipLaunchKernelGGL((k_ln_columns_wide<T, CK>), dim3((unsigned)((d + kLnBlock * kLnV<T> - 1) / (kLnBlock * kLnV<T>)), (unsigned)parts),
                                       dim3(kLnBlock), 0, stream, (const T*)dy, lddy, layer_rows(x), n, (int)d, mean, rstd, partial);
                }
            }
            if (params)
                hipLaunchKernelGGL((k_ln_join<T>), dim3((unsigned)((2 * d + kJoinCols - 1) / kJoinCols)), dim3(kJoinBlock), 0, stream, partial, parts, (int)d,
                                   (T*)dgamma, (T*)dbeta);
        };
        if (n && x->exponents) run(std::integral_constant<bool, true>{});
        else run(std::integral_constant<bool, false>{});
    });
    return layer_launched();
}
