// The product of one or two inputs with a weight matrix, with bias, activation and residual in its epilogue, and its backward pass,
// for gfx950.
//   z = [a | b] w^T + bias,  out = act(z) + residual
//   dz = dout * act'(z),  [da | db] = dz w,  dw = dz^T [a | b],  dbias = sum over rows of dz
// a and b are read where they are: the columns of a are the first steps of the product's long axis, those of b the rest, so a vertex's
// own row and its neighbours' mean need not be copied next to each other.
//
// Sums are held in 32 bits in the matrix cores' registers; z, out and the gradients are rounded once each.  dz is rounded to the
// inputs' type before its two products, which take 16-bit operands (its error, half a step of that type, is of the size of the outputs' own).
#include "grem_layers.hip.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// acc += A B for 16 x 16 of the output and 16 bytes of the long axis per lane: 32 values of 16 bits in one instruction, or 16 floats in
// four.  Lane l holds row (l & 15) of either operand and the run of the long axis that starts at 16 bytes * (l >> 4); the
// order inside the long axis is free as long as both operands share it.
template <class T> __device__ __forceinline__ void mma(f32x4& acc, u32x4 a, u32x4 b)
{
    if constexpr (__is_same(T, bf16)) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    } else if constexpr (__is_same(T, f16)) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
    } else {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], acc, 0, 0, 0);
    }
}

// ---- activations ---------------------------------------------------------------------------------------------------------
template <int ACT> __device__ __forceinline__ float act(float z)
{
    if constexpr (ACT == GREM_ACT_RELU) return z > 0.0f ? z : z == z ? 0.0f : z;
    if constexpr (ACT == GREM_ACT_GELU) return 0.5f * z * erfcf(-0.70710678118654752f * z);
    if constexpr (ACT == GREM_ACT_SILU) return z / (1.0f + expf(-z));
    return z;
}

template <int ACT> __device__ __forceinline__ float act_slope(float z)
{
    if constexpr (ACT == GREM_ACT_RELU) return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
    if constexpr (ACT == GREM_ACT_GELU)
        return 0.5f * erfcf(-0.70710678118654752f * z) + z * 0.39894228040143268f * expf(-0.5f * z * z);
    if constexpr (ACT == GREM_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    return 1.0f;
}

template <class F> void by_act(int32_t a, F f)
{
    switch (a) {
        case GREM_ACT_RELU: f(std::integral_constant<int, GREM_ACT_RELU>{}); break;
        case GREM_ACT_GELU: f(std::integral_constant<int, GREM_ACT_GELU>{}); break;
        case GREM_ACT_SILU: f(std::integral_constant<int, GREM_ACT_SILU>{}); break;
        default: f(std::integral_constant<int, GREM_ACT_NONE>{}); break;
    }
}

// ---- out = [a | b] w^T ----------------------------------------------------------------------------------------------------
//
// A workgroup computes BM rows by BN features, four waves in a square.  Steps of 128 bytes of the long axis (64 values of 16 bits, 32
// floats) are staged through LDS in two buffers: while one is multiplied, the next step's loads are under way to registers.
// LDS rows are 128 bytes, 8 chunks of 16; chunk c of row r lies at c ^ key(r), so that the 16 rows that an operand read touches
// spread over the banks.
//
// The weights are the first operand: an accumulator's four registers then run along a row of the output, and which feature stands in
// which row of the operand is free: tile i, row 4g + r is feature 4 * tiles * g + 4 i + r of the wave's, so that a lane's
// features are side by side and leave in 16-byte stores.
struct Product {
    const void *a, *b, *w;
    int64_t lda, ldb, ldw, n;
    int ka, kb, m;
};

struct Epilogue {
    const void *bias, *residual;
    void *out, *pre;                // features [0, split) of a row
    void *out2;                     // features from split on
    int64_t ldr, ldo, ldp, ldo2;
    int split;
};

constexpr int kLinBlock = 256;
constexpr int kLinStep = 128;       // bytes

// 16 bytes of a row's values from k on, zero from d on
template <class T> __device__ __forceinline__ u32x4 chunk_of(const T* row, int k, int d)
{
    constexpr int V = 16 / (int)sizeof(T);
    T v[V];
    if (k + V <= d) {
        load_run<T, V>(row + k, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = k + i < d ? row[k + i] : (T)0.0f;
    }
    u32x4 r;
    __builtin_memcpy(&r, v, 16);
    return r;
}

template <int NT> __device__ __forceinline__ int weight_key(int r) { return (r & 3) | (((r / (4 * NT)) & 1) << 2); }

template <class T, int BM, int BN, int ACT, bool SPLIT>
__global__ __launch_bounds__(kLinBlock) void k_lin_product(Product p, Epilogue e)
{
    constexpr int V = 16 / (int)sizeof(T), K = kLinStep / (int)sizeof(T);
    constexpr int MT = BM / 32, NT = BN / 32;               // 16 x 16 tiles of a wave: rows, features
    constexpr int LA = BM / 32, LW = BN / 32;               // chunks a thread stages
    __shared__ u32x4 sx[2][BM * 8], sw[2][BN * 8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, rho = lane & 15;
    const int64_t row0 = (int64_t)blockIdx.x * BM;
    const int col0 = (int)blockIdx.y * BN;
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
    const int sr = threadIdx.x >> 3, sc = threadIdx.x & 7;
    const int steps_a = (p.ka + K - 1) / K, steps = steps_a + (p.kb + K - 1) / K;

    int64_t xrow[LA];
    int wrow[LW];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int64_t r = row0 + i * 32 + sr;
        xrow[i] = r < p.n ? r : p.n - 1;
    }
#pragma unroll
    for (int i = 0; i < LW; ++i) {
        const int c = col0 + i * 32 + sr;
        wrow[i] = c < p.m ? c : p.m - 1;
    }
    u32x4 rx[LA], rw[LW];
    auto load = [&](int step) {
        const bool first = step < steps_a;
        const T* x = (const T*)(first ? p.a : p.b);
        const int64_t ld = first ? p.lda : p.ldb;
        const int k = (first ? step : step - steps_a) * K + sc * V, d = first ? p.ka : p.kb;
        const T* w = (const T*)p.w + (first ? 0 : p.ka);
#pragma unroll
        for (int i = 0; i < LA; ++i) rx[i] = chunk_of<T>(x + xrow[i] * ld, k, d);
#pragma unroll
        for (int i = 0; i < LW; ++i) rw[i] = chunk_of<T>(w + wrow[i] * p.ldw, k, d);
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < LA; ++i) sx[buf][(i * 32 + sr) * 8 + (sc ^ (sr & 7))] = rx[i];
#pragma unroll
        for (int i = 0; i < LW; ++i) {
            const int r = i * 32 + sr;
            sw[buf][r * 8 + (sc ^ weight_key<NT>(r))] = rw[i];
        }
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (steps > 0) {
        load(0);
        store(0);
    }
    __syncthreads();
    for (int s = 0; s < steps; ++s) {
        const int buf = s & 1;
        if (s + 1 < steps) load(s + 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 fx[MT], fw[NT];
            const int c = h * 4 + g;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int r = wm + i * 16 + rho;
                fx[i] = sx[buf][r * 8 + (c ^ (r & 7))];
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int r = wn + (rho >> 2) * (4 * NT) + j * 4 + (rho & 3);
                fw[j] = sw[buf][r * 8 + (c ^ weight_key<NT>(r))];
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) mma<T>(acc[i][j], fw[j], fx[i]);
        }
        if (s + 1 < steps) store(buf ^ 1);
        __syncthreads();
    }

    // lane (g, rho): row wm + 16 i + rho, features wn + 4 NT g .. + 4 NT
    const int f0 = col0 + wn + g * (4 * NT);
    if (f0 >= p.m) return;
    float bias[4 * NT];
#pragma unroll
    for (int j = 0; j < 4 * NT; ++j) bias[j] = !SPLIT && e.bias && f0 + j < p.m ? (float)((const T*)e.bias)[f0 + j] : 0.0f;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t row = row0 + wm + i * 16 + rho;
        if (row >= p.n) continue;
#pragma unroll
        for (int q = 0; q < 4 * NT; q += V) {
            const int f = f0 + q;
            if (f >= p.m) continue;
            float z[V];
#pragma unroll
            for (int t = 0; t < V; ++t) z[t] = acc[i][(q + t) / 4][(q + t) % 4] + bias[q + t];
            if constexpr (SPLIT) {
                if (f + V <= e.split) {
                    if (e.out) store_floats<T, V>((T*)e.out + row * e.ldo, f, p.m, z);
                } else if (f >= e.split) {
                    if (e.out2) store_floats<T, V>((T*)e.out2 + row * e.ldo2, f - e.split, p.m - e.split, z);
                } else {
#pragma unroll
                    for (int t = 0; t < V; ++t) {
                        if (f + t < e.split) {
                            if (e.out) ((T*)e.out)[row * e.ldo + f + t] = (T)z[t];
                        } else if (f + t < p.m && e.out2) {
                            ((T*)e.out2)[row * e.ldo2 + f + t - e.split] = (T)z[t];
                        }
                    }
                }
            } else {
                if (e.pre) store_floats<T, V>((T*)e.pre + row * e.ldp, f, p.m, z);
                float r[V];
                if (e.residual) load_floats<T, V>((const T*)e.residual + row * e.ldr, f, p.m, r);
#pragma unroll
                for (int t = 0; t < V; ++t) z[t] = act<ACT>(z[t]) + (e.residual ? r[t] : 0.0f);
                store_floats<T, V>((T*)e.out + row * e.ldo, f, p.m, z);
            }
        }
    }
}

// ---- dw = dz^T [a | b] ----------------------------------------------------------------------------------------------------
//
// The long axis is the rows: a workgroup takes BM features of dz by BN columns of a or of b and a stretch of rows, and leaves its sums in
// 32 bits; k_lin_join adds the stretches in order.  Both operands lie with the long axis across their rows.  They are staged as
// they lie, and the reads from LDS turn them: for 16 bits the transposing read gives lane rho of 16 lanes four rows of column rho, where
// the lanes' addresses cover 4 rows of 16 columns; floats are read one by one.  A checkpoint's codes become values on the
// way to LDS, exactly.
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T> constexpr int kLinRows = kLinStep / (int)sizeof(T);        // rows of a step

template <class T, bool CK> __device__ __forceinline__ u32x4 source_chunk(const Rows& x, int64_t r, int c, int d)
{
    if constexpr (!CK) {
        return c < d ? chunk_of<T>((const T*)x.data + r * x.stride, c, d) : u32x4{0, 0, 0, 0};
    } else {
        constexpr int V = 16 / (int)sizeof(T);
        float f[V];
        load_row<T, true, V>(x, r, c, d, f);
        T v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (T)f[i];
        u32x4 q;
        __builtin_memcpy(&q, v, 16);
        return q;
    }
}

template <class T, bool CK, int BM, int BN>
__global__ __launch_bounds__(kLinBlock) void k_lin_weight(const T* __restrict__ dz, int64_t lddz, Rows a, Rows b, int64_t n, int ka,
                                                          int kb, int m, int tiles_a, int64_t stretch, float* __restrict__ partial)
{
    constexpr int V = 16 / (int)sizeof(T), R = kLinRows<T>;
    constexpr int MT = BM / 32, NT = BN / 32;
    constexpr int CM = BM / V, CN = BN / V;                          // chunks of a row
    constexpr int LM = R * CM / kLinBlock, LN = R * CN / kLinBlock;  // chunks a thread stages
    // rows are padded by 32 bytes (16 bits) or 64 (floats): the reads of one instruction then cover all banks evenly
    constexpr int PM = CM + (sizeof(T) == 2 ? 2 : 4), PN = CN + (sizeof(T) == 2 ? 2 : 4);
    __shared__ u32x4 sz[2][R * PM], sx[2][R * PN];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, rho = lane & 15;
    const int col0 = (int)blockIdx.x * BM;                           // of dz
    const bool first = (int)blockIdx.y < tiles_a;
    const Rows x = first ? a : b;
    const int k0 = (first ? (int)blockIdx.y : (int)blockIdx.y - tiles_a) * BN, kd = first ? ka : kb;
    const int64_t lo = (int64_t)blockIdx.z * stretch, hi = lo + stretch < n ? lo + stretch : n;
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);

    u32x4 rz[LM], rx[LN];
    auto load = [&](int64_t from) {
#pragma unroll
        for (int i = 0; i < LM; ++i) {
            const int q = i * kLinBlock + (int)threadIdx.x, r = q / CM, c = col0 + (q % CM) * V;
            rz[i] = from + r < hi && c < m ? chunk_of<T>(dz + (from + r) * lddz, c, m) : u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < LN; ++i) {
            const int q = i * kLinBlock + (int)threadIdx.x, r = q / CN, c = k0 + (q % CN) * V;
            rx[i] = from + r < hi ? source_chunk<T, CK>(x, from + r, c, kd) : u32x4{0, 0, 0, 0};
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < LM; ++i) {
            const int q = i * kLinBlock + (int)threadIdx.x;
            sz[buf][(q / CM) * PM + q % CM] = rz[i];
        }
#pragma unroll
        for (int i = 0; i < LN; ++i) {
            const int q = i * kLinBlock + (int)threadIdx.x;
            sx[buf][(q / CN) * PN + q % CN] = rx[i];
        }
    };
    // 16 columns from `col` on by half h of the step's rows
    auto operand = [&](const u32x4* s, int pitch, int col, int h) {
        if constexpr (sizeof(T) == 2) {
            const char* p = (const char*)s + (size_t)(h * 32 + g * 8 + (rho >> 2)) * (size_t)(pitch * 16) + (size_t)(col + (rho & 3) * 4) * 2;
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
            const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + (size_t)(4 * pitch * 16)));
            u32x4 out;
            __builtin_memcpy(&out, &u, 8);
            __builtin_memcpy((char*)&out + 8, &v, 8);
            return out;
        } else {
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = ((const float*)s)[(h * 16 + i * 4 + g) * (pitch * 4) + col + rho];
            return __builtin_bit_cast(u32x4, v);
        }
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (lo < hi) {
        load(lo);
        store(0);
    }
    __syncthreads();
    int buf = 0;
    for (int64_t from = lo; from < hi; from += R, buf ^= 1) {
        const bool more = from + R < hi;
        if (more) load(from + R);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 fz[MT], fx[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i) fz[i] = operand(sz[buf], PM, wm + i * 16, h);
#pragma unroll
            for (int j = 0; j < NT; ++j) fx[j] = operand(sx[buf], PN, wn + j * 16, h);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) mma<T>(acc[i][j], fx[j], fz[i]);
        }
        if (more) store(buf ^ 1);
        __syncthreads();
    }
    // lane (g, rho): feature col0 + wm + 16 i + rho, columns wn + 16 j + 4 g .. + 4
    const int width = ka + kb, base = first ? k0 : ka + k0;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int f = col0 + wm + i * 16 + rho;
        if (f >= m) continue;
        float* out = partial + ((size_t)blockIdx.z * (size_t)m + (size_t)f) * (size_t)width + base;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int c = wn + j * 16 + g * 4;
            float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (k0 + c < kd) store_floats<float, 4>(out, c, kd - k0, v);
        }
    }
}

// dw[f][c] = sum over the stretches, in order
template <class T>
__global__ __launch_bounds__(kLinBlock) void k_lin_join(const float* __restrict__ partial, int stretches, int64_t values, int width,
                                                        T* __restrict__ dw, int64_t lddw)
{
    for (int64_t i = (int64_t)blockIdx.x * kLinBlock + threadIdx.x; i < values; i += (int64_t)gridDim.x * kLinBlock) {
        float s = 0.0f;
        for (int q = 0; q < stretches; ++q) s += partial[(int64_t)q * values + i];
        dw[i / width * lddw + i % width] = (T)s;
    }
}

// ---- dz and dbias ---------------------------------------------------------------------------------------------------------
//
// One pass over dout and z: dz rounded to its type, and the columns' sums of the unrounded dz, a partial row per workgroup
// (its 256 threads are 32 runs of columns by 8 rows).
constexpr int kLinDzCols = 32, kLinDzRows = 8;

template <class T, int ACT>
__global__ __launch_bounds__(kLinBlock) void k_lin_slope(const T* __restrict__ dout, int64_t ldd, const T* __restrict__ pre, int64_t ldp,
                                                         int64_t n, int m, T* __restrict__ dz, int64_t lddz,
                                                         float* __restrict__ partial)
{
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ float sums[kLinDzRows][kLinDzCols * V + 1];
    const int col = threadIdx.x % kLinDzCols, slot = threadIdx.x / kLinDzCols;
    const int c = ((int)blockIdx.y * kLinDzCols + col) * V;
    float s[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = 0.0f;
    if (c < m)
        for (int64_t r = (int64_t)blockIdx.x * kLinDzRows + slot; r < n; r += (int64_t)gridDim.x * kLinDzRows) {
            float f[V], z[V];
            load_floats<T, V>(dout + r * ldd, c, m, f);
            if constexpr (ACT != GREM_ACT_NONE) {
                load_floats<T, V>(pre + r * ldp, c, m, z);
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] *= act_slope<ACT>(z[i]);
                store_floats<T, V>(dz + r * lddz, c, m, f);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] += f[i];
        }
    if (!partial) return;
#pragma unroll
    for (int i = 0; i < V; ++i) sums[slot][col * V + i] = s[i];
    __syncthreads();
    for (int i = threadIdx.x; i < kLinDzCols * V; i += kLinBlock) {
        const int at = (int)blockIdx.y * kLinDzCols * V + i;
        float t = 0.0f;
#pragma unroll
        for (int q = 0; q < kLinDzRows; ++q) t += sums[q][i];
        if (at < m) partial[(size_t)blockIdx.x * (size_t)m + at] = t;
    }
}

// dbias: a workgroup takes 16 columns, 16 threads a column, then those in order
template <class T>
__global__ __launch_bounds__(kLinBlock) void k_lin_bias(const float* __restrict__ partial, int parts, int m, T* __restrict__ dbias)
{
    __shared__ float sums[16][17];
    const int c = (int)blockIdx.x * 16 + (threadIdx.x & 15), q = threadIdx.x >> 4;
    float s = 0.0f;
    if (c < m)
        for (int p = q; p < parts; p += 16) s += partial[(size_t)p * (size_t)m + c];
    sums[q][threadIdx.x & 15] = s;
    __syncthreads();
    if (threadIdx.x >= 16 || c >= m) return;
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) total += sums[i][threadIdx.x];
    dbias[c] = (T)total;
}

// w (m x width) turned: wt (width x m), so that dz w is a product of the first kind
template <class T>
__global__ __launch_bounds__(kLinBlock) void k_lin_turn(const T* __restrict__ w, int64_t ldw, int m, int width, T* __restrict__ wt, int64_t ldt)
{
    __shared__ T tile[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int c0 = (int)blockIdx.x * 32, f0 = (int)blockIdx.y * 32;
#pragma unroll
    for (int i = 0; i < 32; i += 8)
        if (f0 + y + i < m && c0 + x < width) tile[y + i][x] = w[(int64_t)(f0 + y + i) * ldw + c0 + x];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 32; i += 8)
        if (c0 + y + i < width && f0 + x < m) wt[(int64_t)(c0 + y + i) * ldt + f0 + x] = tile[x][y + i];
}

// ---- host ------------------------------------------------------------------------------------------------------------------
template <class T, bool SPLIT> void lin_product(const Product& p, const Epilogue& e, int32_t activation, hipStream_t stream)
{
    constexpr int BM = 128, BN = 128;
    const dim3 grid((unsigned)((p.n + BM - 1) / BM), (unsigned)((p.m + BN - 1) / BN));
    if constexpr (SPLIT)
        hipLaunchKernelGGL((k_lin_product<T, BM, BN, GREM_ACT_NONE, true>), grid, dim3(kLinBlock), 0, stream, p, e);
    else
        by_act(activation, [&](auto a) {
            hipLaunchKernelGGL((k_lin_product<T, BM, BN, decltype(a)::value, false>), grid, dim3(kLinBlock), 0, stream, p, e);
        });
}

// the backward pass's workspace
struct LinSpace {
    int64_t lddz, ldt, stretch;
    int stretches, parts;
    size_t o_dz, o_wt, o_dw, o_bias, bytes;
};

LinSpace lin_space(int size, int64_t n, int64_t m, int64_t ka, int64_t kb, int32_t activation)
{
    LinSpace s;
    const int64_t V = 16 / size, rows = kLinStep / size;
    size_t off = 0;
    auto carve = [&](size_t bytes) { const size_t at = off; off += layer_align(bytes); return at; };
    s.lddz = (m + V - 1) / V * V;
    s.ldt = s.lddz;
    s.o_dz = carve(activation == GREM_ACT_NONE ? 0 : (size_t)n * (size_t)s.lddz * size);
    s.o_wt = carve((size_t)(ka + kb) * (size_t)s.ldt * size);
    // stretches of rows: enough workgroups for two a CU, and no shorter than 8 steps
    const int64_t tiles = ((m + 127) / 128) * ((ka + 127) / 128 + (kb + 127) / 128);
    int64_t want = tiles ? (512 + tiles - 1) / tiles : 1;
    const int64_t most = (n + 8 * rows - 1) / (8 * rows);
    if (want > most) want = most;
    if (want < 1) want = 1;
    s.stretch = (n + want - 1) / want;
    s.stretch = (s.stretch + rows - 1) / rows * rows;
    if (s.stretch < rows) s.stretch = rows;
    s.stretches = (int)((n + s.stretch - 1) / s.stretch);
    if (s.stretches < 1) s.stretches = 1;
    s.o_dw = carve((size_t)s.stretches * (size_t)m * (size_t)(ka + kb) * 4);
    s.parts = (int)((n + kLinDzRows - 1) / kLinDzRows);
    if (s.parts > 1024) s.parts = 1024;
    s.o_bias = carve((size_t)s.parts * (size_t)m * 4);
    s.bytes = off;
    return s;
}

bool lin_shape_ok(int64_t n, int64_t m, int64_t ka, int64_t kb)
{
    return n >= 0 && n <= kLayerMaxRows && m >= 1 && m <= kLayerMaxCols && ka >= 1 && ka <= kLayerMaxCols && kb >= 0 && kb <= kLayerMaxCols;
}

bool act_ok(int32_t a) { return a >= GREM_ACT_NONE && a <= GREM_ACT_SILU; }

}  // namespace

extern "C" int grem_linear(int32_t type, int64_t n, int64_t m, const void* a, int64_t lda, int64_t ka, const void* b, int64_t ldb,
                           int64_t kb, const void* w, int64_t ldw, const void* bias, int32_t activation, const void* residual,
                           int64_t ldr, void* out, int64_t ldo, void* pre, int64_t ldp, void* stream)
{
    const int size = layer_size(type);
    if (!size || !lin_shape_ok(n, m, ka, kb) || !act_ok(activation) || !layer_rows_ok(a, lda, n, ka, size) ||
        (kb && !layer_rows_ok(b, ldb, n, kb, size)) || !layer_rows_ok(w, ldw, m, ka + kb, size) || (uintptr_t)bias % size ||
        (residual && !layer_rows_ok(residual, ldr, n, m, size)) || !layer_rows_ok(out, ldo, n, m, size) ||
        (pre && !layer_rows_ok(pre, ldp, n, m, size)))
        return GREM_ERR_ARG;
    if (n == 0) return GREM_OK;
    const Product p{a, b, w, lda, ldb, ldw, n, (int)ka, (int)kb, (int)m};
    const Epilogue e{bias, residual, out, pre, nullptr, ldr, ldo, ldp, 0, 0};
    layer_typed(type, [&](auto t) { lin_product<decltype(t), false>(p, e, activation, (hipStream_t)stream); });
    return layer_launched();
}

extern "C" size_t grem_linear_backward_bytes(int32_t type, int64_t n, int64_t m, int64_t ka, int64_t kb, int32_t activation)
{
    const int size = layer_size(type);
    return !size || !lin_shape_ok(n, m, ka, kb) || !act_ok(activation) ? 0 : lin_space(size, n, m, ka, kb, activation).bytes;
}

extern "C" int grem_linear_backward(int32_t type, int64_t n, int64_t m, const void* dout, int64_t ldd, int32_t activation, const void* pre,
                                    int64_t ldp, const grem_rows* a, int64_t ka, const grem_rows* b, int64_t kb, const void* w,
                                    int64_t ldw, void* da, int64_t ldda, void* db, int64_t lddb, void* dw, int64_t lddw, void* dbias,
                                    void* workspace, size_t workspace_bytes, void* stream_)
{
    const int size = layer_size(type);
    if (!size || !lin_shape_ok(n, m, ka, kb) || !act_ok(activation) || !layer_rows_ok(dout, ldd, n, m, size) ||
        (activation != GREM_ACT_NONE && !layer_rows_ok(pre, ldp, n, m, size)) || (kb == 0 && db) ||
        ((da || db) && !layer_rows_ok(w, ldw, m, ka + kb, size)) || (da && !layer_rows_ok(da, ldda, n, ka, size)) ||
        (db && !layer_rows_ok(db, lddb, n, kb, size)) || (uintptr_t)dbias % size)
        return GREM_ERR_ARG;
    if (dw && (!layer_rows_ok(dw, lddw, m, ka + kb, size) || !layer_source_ok(a, n, ka, size) || (kb && !layer_source_ok(b, n, kb, size)) ||
               (kb && n && !a->exponents != !b->exponents)))
        return GREM_ERR_ARG;
    if (!da && !db && !dw && !dbias) return GREM_OK;
    const LinSpace s = lin_space(size, n, m, ka, kb, activation);
    if (s.bytes && (!workspace || workspace_bytes < s.bytes)) return GREM_ERR_NOMEM;
    if (n == 0 && !dw && !dbias) return GREM_OK;
    hipStream_t stream = (hipStream_t)stream_;
    uint8_t* ws = (uint8_t*)workspace;
    layer_typed(type, [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / (int)sizeof(T);
        const T* dz = (const T*)dout;
        int64_t lddz = ldd;
        float* bias_parts = dbias ? (float*)(ws + s.o_bias) : nullptr;
        if (n && (activation != GREM_ACT_NONE || dbias)) {
            T* made = (T*)(ws + s.o_dz);
            by_act(activation, [&](auto act) {
                hipLaunchKernelGGL((k_lin_slope<T, decltype(act)::value>), dim3((unsigned)s.parts, (unsigned)((m + kLinDzCols * V - 1) / (kLinDzCols * V))),
                                   dim3(kLinBlock), 0, stream, (const T*)dout, ldd, (const T*)pre, ldp, n, (int)m, made, s.lddz, bias_parts);
            });
            if (activation != GREM_ACT_NONE) {
                dz = made;
                lddz = s.lddz;
            }
        }
        if (dbias)
            hipLaunchKernelGGL((k_lin_bias<T>), dim3((unsigned)((m + 15) / 16)), dim3(kLinBlock), 0, stream, bias_parts, n ? s.parts : 0, (int)m,
                               (T*)dbias);
        if (n && (da || db)) {
            T* wt = (T*)(ws + s.o_wt);
            hipLaunchKernelGGL((k_lin_turn<T>), dim3((unsigned)((ka + kb + 31) / 32), (unsigned)((m + 31) / 32)), dim3(kLinBlock), 0, stream,
                               (const T*)w, ldw, (int)m, (int)(ka + kb), wt, s.ldt);
            const Product p{dz, nullptr, wt, lddz, 0, s.ldt, n, (int)m, 0, (int)(ka + kb)};
            const Epilogue e{nullptr, nullptr, da, nullptr, db, 0, ldda, 0, lddb, (int)ka};
            lin_product<T, true>(p, e, GREM_ACT_NONE, stream);
        }
        if (dw) {
            float* parts = (float*)(ws + s.o_dw);
            const int tiles_a = (int)((ka + 127) / 128), tiles_b = (int)((kb + 127) / 128);
            const dim3 grid((unsigned)((m + 127) / 128), (unsigned)(tiles_a + tiles_b), (unsigned)s.stretches);
            const Rows xa = n ? layer_rows(a) : Rows{}, xb = n && kb ? layer_rows(b) : Rows{};
            if (n && a->exponents)
                hipLaunchKernelGGL((k_lin_weight<T, true, 128, 128>), grid, dim3(kLinBlock), 0, stream, dz, lddz, xa, xb, n, (int)ka, (int)kb,
                                   (int)m, tiles_a, s.stretch, parts);
            else
                hipLaunchKernelGGL((k_lin_weight<T, false, 128, 128>), grid, dim3(kLinBlock), 0, stream, dz, lddz, xa, xb, n, (int)ka, (int)kb,
                                   (int)m, tiles_a, s.stretch, parts);
            const int64_t values = m * (ka + kb), groups = (values + kLinBlock - 1) / kLinBlock;
            hipLaunchKernelGGL((k_lin_join<T>), dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(kLinBlock), 0, stream, parts, s.stretches, values,
                               (int)(ka + kb), (T*)dw, lddw);
        }
    });
    return layer_launched();
}
