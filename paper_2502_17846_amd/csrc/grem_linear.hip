// The product of one or two inputs with a weight matrix, with bias, activation and residual in its epilogue, and its backward pass,
// for gfx950.
//   z = [a | b] w^T + bias,  out = act(z) + residual
//   dz = dout * act'(z),  [da | db] = dz w,  dw = dz^T [a | b],  dbias = sum over rows of dz
// a and b are read where they are: the columns of a are the first steps of the product's long axis, those of b the rest, so a vertex's
// own row and its neighbours' mean need not be copied next to each other.
//
// Sums are held in 32 bits in the matrix cores' registers; z, out and the gradients are rounded once each.  With an activation dz is rounded to
// the inputs' type before its two products, whose operands are 16 bits wide: a second error of the size of the outputs' own rounding, independent
// of it, so that da, db and dw are off by 1.41 times as much (of their norm: half precision 2.9e-4 for 2.1e-4, bfloat16 2.35e-3 for 1.66e-3).
// Two operands for dz, its rounding and what that left, would take it away and double the products.
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
//
// exp(-z^2/2) and the normal distribution function.  The tail, 1 - Phi(x) for x = |z|, is exp(-x^2/2) * (c1 t + .. + cn t^n) with
// t = 1 / (1 + q x): Mills' ratio is smooth in t and goes to 0 with it, so a polynomial without a constant follows it to infinity, and small
// values of GELU keep their digits.  The c are least maximum relative errors over x >= 0 (reweighted least squares against erfc in 64 bits): n = 9
// is off by 1.3e-7 of the tail, n = 7 by 3.5e-6, a hundredth of a half step of the 16-bit types, which take it.  The square's and the
// exponent's roundings grow as x^2: 32-bit types carry them along (without them 4e-6 at x = 10).  With evaluation: 9 half steps of 32 bits at
// most, on average 0.66 for |z| < 3, and 2^-16.6.  (The math library's erfc takes three times the instructions, and with them an epilogue's time
// outgrew its product's: 262,144 x 512 by 256 took 280 us with it.)
struct Normal {
    float density, below;           // exp(-z^2/2), Phi(z)
};

template <class T> __device__ __forceinline__ Normal normal_at(float z)
{
    const float x = fabsf(z), near = fminf(x, 20.0f), s = near * near;       // (exp(-200) is 0)
    constexpr float scale = -0.72134752044448170f;                           // -log2(e) / 2
    const float power = s * scale;
    float e = __builtin_amdgcn_exp2f(power), poly;
    if constexpr (sizeof(T) == 4) {
        const float rest = __builtin_fmaf(s, scale, -power) + __builtin_fmaf(near, near, -s) * scale + s * (float)(-0.72134752044448170 - (double)scale);
        e = __builtin_fmaf(e, rest * 0.69314718055994531f, e);
        const float t = __builtin_amdgcn_rcpf(1.0f + 0.2827f * x);
        poly = t * (0.112780996f + t * (0.112777829f + t * (0.103879213f + t * (0.0842417628f + t * (0.0708082244f + t * (-0.00295902393f +
               t * (0.0849074423f + t * (-0.0915424824f + t * 0.0251060724f))))))));
    } else {
        const float t = __builtin_amdgcn_rcpf(1.0f + 0.2792f * x);
        poly = t * (0.111384295f + t * (0.111439563f + t * (0.101470783f + t * (0.0954858735f + t * (0.0223157033f + t * (0.10880512f +
               t * -0.0509027466f))))));
    }
    const float tail = e * poly;
    return Normal{e, z > 0.0f ? 1.0f - tail : tail};
}

// 1 / (1 + exp(-z)): 0 and 1 at the ends, where exp leaves its range
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f)); }

template <class T, int ACT> __device__ __forceinline__ float act(float z)
{
    if constexpr (ACT == GREM_ACT_RELU) return z > 0.0f ? z : z == z ? 0.0f : z;
    if constexpr (ACT == GREM_ACT_GELU) return z * normal_at<T>(z).below;
    if constexpr (ACT == GREM_ACT_SILU) return z * sigmoid(z);
    return z;
}

template <class T, int ACT> __device__ __forceinline__ float act_slope(float z)
{
    if constexpr (ACT == GREM_ACT_RELU) return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
    if constexpr (ACT == GREM_ACT_GELU) {
        const Normal a = normal_at<T>(z);
        return a.below + z * 0.39894228040143268f * a.density;
    }
    if constexpr (ACT == GREM_ACT_SILU) {
        const float s = sigmoid(z);
        return s * (1.0f + z * (1.0f - s));
    }
    return 1.0f;
}

template <class F> __host__ __device__ __forceinline__ void by_act(int32_t a, F f)
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
// which row of the operand is free: a lane gets runs of V features (16 bytes) whose four neighbours' runs lie beside its own, so that a
// store instruction writes 64 bytes of each of 16 rows.
struct Product {
    const void *a, *b, *w;
    int64_t lda, ldb, ldw, n;
    int ka, kb, m, tiles_m;
};

struct Epilogue {
    const void *bias, *residual;
    void *out, *pre;                // features [0, split) of a row
    void *out2;                     // features from split on
    int64_t ldr, ldo, ldp, ldo2;
    int split, act;
};

constexpr int kLinBlock = 256;
constexpr int kLinStep = 128;       // bytes

// BM rows (of the output's n, or features of dz) by BN, of which a wave takes WM by WN
template <int BM_, int BN_, int WM_, int WN_> struct LinTile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, stages = 2, threads = BM / WM * (BN / WN) * 64;
    static constexpr int lds = stages * (BM + BN) * kLinStep, per_cu = 160 * 1024 / lds, waves_per_simd = per_cu * threads / 256;
};

// Workgroups go to the eight chiplets in turn.  Those that share a block of rows are given numbers eight apart, so that they run on
// one chiplet and the rows come from its L2.
struct LinPlace {
    int64_t row;
    int col;
};

__device__ __forceinline__ LinPlace lin_place(uint32_t id, int cols)
{
    const uint32_t chiplet = id & 7u, local = id >> 3;
    return LinPlace{(int64_t)(local / (uint32_t)cols) * 8 + chiplet, (int)(local % (uint32_t)cols)};
}

// 16 bytes at the alignment of a value
struct __attribute__((packed, aligned(2))) Chunk {
    u32x4 v;
};

// 16 bytes of a row's values from k on, zero from d on; WHOLE: the caller knows that they end before d.  (Where that is
// known for all lanes there must be no branch on it: the two ways' values would meet element by element, which waits for the load.)
template <class T, bool WHOLE = false> __device__ __forceinline__ u32x4 chunk_of(const T* row, int k, int d)
{
    constexpr int V = 16 / (int)sizeof(T);
    if constexpr (WHOLE) return ((const Chunk*)(row + k))->v;
    if (k + V <= d) return ((const Chunk*)(row + k))->v;
    T v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = k + i < d ? row[k + i] : (T)0.0f;
    u32x4 r;
    __builtin_memcpy(&r, v, 16);
    return r;
}

// A row's last run, where d is no multiple of V, is read as the V values that end at d, in one load, and moved down by the `over` values that
// belong to the run before (a run beyond d: by V or more, nothing is left of it).  Loads stay under way until the runs are stored to LDS.
template <class T> __device__ __forceinline__ int run_over(int k, int d)
{
    constexpr int V = 16 / (int)sizeof(T);
    return k > d - V ? k - (d - V) : 0;
}

template <int BITS> __device__ __forceinline__ u32x4 moved_down(u32x4 v, int over)
{
    const int bits = over * BITS;
    uint64_t w[2];
    __builtin_memcpy(w, &v, 16);
    const uint64_t from_high = bits < 64 ? w[1] << 1 << (63 - bits) : w[1] >> (bits & 63);
    const uint64_t low = bits < 64 ? w[0] >> bits | from_high : bits < 128 ? from_high : 0ull;
    const uint64_t high = bits < 64 ? w[1] >> bits : 0ull;
    w[0] = low;
    w[1] = high;
    u32x4 r;
    __builtin_memcpy(&r, w, 16);
    return r;
}

// where row rho of the weights' operand j stands among a wave's features, and what tells the rows apart that are read together
template <class T> __device__ __forceinline__ int weight_row(int j, int rho)
{
    constexpr int V = 16 / (int)sizeof(T), J = V / 4;
    return j / J * (4 * V) + (rho >> 2) * V + j % J * 4 + (rho & 3);
}

template <class T> __device__ __forceinline__ int weight_key(int r) { return (r & 3) | ((r / (16 / (int)sizeof(T))) & 1) << 2; }

// What a lane holds at the end: rows row_of + 16 i, features f0 + 4 V q .. + V.  whole: the workgroup's tile lies inside the output.
template <class T, int MT, int NT, bool SPLIT>
__device__ __forceinline__ void lin_epilogue(const f32x4 (&acc)[MT][NT], const Product& p, const Epilogue& e, int64_t row_of, int f0,
                                             bool whole)
{
    constexpr int V = 16 / (int)sizeof(T);
    if (f0 >= p.m) return;
    float bias[4 * NT];
#pragma unroll
    for (int j = 0; j < 4 * NT; ++j) {
        const int f = f0 + j / V * (4 * V) + j % V;
        bias[j] = !SPLIT && e.bias && f < p.m ? (float)((const T*)e.bias)[f] : 0.0f;
    }
    constexpr int Q = 4 * NT / V, part = MT < 4 ? MT : 4;
    auto rows = [&](auto all, auto activation) {
        constexpr bool WHOLE = decltype(all)::value;
        constexpr int ACT = decltype(activation)::value;
#pragma unroll
        for (int i0 = 0; i0 < MT; i0 += part) {
            // (the residual of four rows at a time, all under way before the first is used: `out` may be the residual itself, so the
            // compiler may not move a load before a store)
            u32x4 res[part][Q];
            if constexpr (!SPLIT) {
                if (e.residual)
#pragma unroll
                    for (int i = 0; i < part; ++i)
#pragma unroll
                        for (int q = 0; q < Q; ++q) {
                            const int64_t row = row_of + (i0 + i) * 16;
                            const int f = f0 + q * (4 * V);
                            res[i][q] = WHOLE || (row < p.n && f < p.m) ? chunk_of<T, WHOLE>((const T*)e.residual + row * e.ldr, f, p.m)
                                                                        : u32x4{0, 0, 0, 0};
                        }
            }
#pragma unroll
            for (int i = 0; i < part; ++i) {
                const int64_t row = row_of + (i0 + i) * 16;
                if (!WHOLE && row >= p.n) continue;
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    const int f = f0 + q * (4 * V);
                    if (!WHOLE && f >= p.m) continue;
                    const int end = WHOLE ? f + V : p.m;
                    float z[V];
#pragma unroll
                    for (int t = 0; t < V; ++t) z[t] = acc[i0 + i][(q * V + t) / 4][t % 4] + bias[q * V + t];
                    if constexpr (SPLIT) {
                        if (f + V <= e.split) {
                            if (e.out) store_floats<T, V>((T*)e.out + row * e.ldo, f, end, z);
                        } else if (f >= e.split) {
                            if (e.out2) store_floats<T, V>((T*)e.out2 + row * e.ldo2, f - e.split, end - e.split, z);
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
                        if (e.pre) store_floats<T, V>((T*)e.pre + row * e.ldp, f, end, z);
                        T r[V];
                        __builtin_memcpy(r, &res[i][q], 16);
#pragma unroll
                        for (int t = 0; t < V; ++t) z[t] = act<T, ACT>(z[t]) + (e.residual ? (float)r[t] : 0.0f);
                        store_floats<T, V>((T*)e.out + row * e.ldo, f, end, z);
                    }
                }
            }
        }
    };
    if constexpr (SPLIT) {
        if (whole) rows(std::true_type{}, std::integral_constant<int, GREM_ACT_NONE>{});
        else rows(std::false_type{}, std::integral_constant<int, GREM_ACT_NONE>{});
    } else {
        by_act(e.act, [&](auto activation) {
            if (whole) rows(std::true_type{}, activation);
            else rows(std::false_type{}, activation);
        });
    }
}

template <class T, class Tile, bool SPLIT>
__global__ __launch_bounds__(Tile::threads) void k_lin_product(Product p, Epilogue e)
{
    constexpr int BM = Tile::BM, BN = Tile::BN;
    constexpr int V = 16 / (int)sizeof(T), K = kLinStep / (int)sizeof(T);
    constexpr int MT = Tile::WM / 16, NT = Tile::WN / 16;   // 16 x 16 tiles of a wave: rows, features
    constexpr int RS = Tile::threads / 8;                   // rows that the workgroup stages at a time
    constexpr int LA = BM / RS, LW = BN / RS;               // chunks a thread stages
    __shared__ u32x4 sx[2][BM * 8], sw[2][BN * 8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, rho = lane & 15;
    const LinPlace at = lin_place(blockIdx.x, p.tiles_m);
    const int64_t row0 = at.row * BM;
    if (row0 >= p.n) return;
    const int col0 = at.col * BN;
    const int wm = wave / (BN / Tile::WN) * Tile::WM, wn = wave % (BN / Tile::WN) * Tile::WN;
    const int sr = threadIdx.x >> 3, sc = threadIdx.x & 7;
    const int steps_a = (p.ka + K - 1) / K, steps = steps_a + (p.kb + K - 1) / K;

    int64_t xrow[LA];
    int wrow[LW];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int64_t r = row0 + i * RS + sr;
        xrow[i] = r < p.n ? r : p.n - 1;
    }
#pragma unroll
    for (int i = 0; i < LW; ++i) {
        const int c = col0 + i * RS + sr;
        wrow[i] = c < p.m ? c : p.m - 1;
    }
    u32x4 rx[LA], rw[LW];
    int over = 0;
    bool ragged = false;
    auto load = [&](int step) {
        const bool first = step < steps_a;
        const T* x = (const T*)(first ? p.a : p.b);
        const int64_t ld = first ? p.lda : p.ldb;
        const int k = (first ? step : step - steps_a) * K + sc * V, d = first ? p.ka : p.kb;
        const T* w = (const T*)p.w + (first ? 0 : p.ka);
        auto all = [&](auto whole) {
            constexpr bool W = decltype(whole)::value;
#pragma unroll
            for (int i = 0; i < LA; ++i) rx[i] = chunk_of<T, W>(x + xrow[i] * ld, k, d);
#pragma unroll
            for (int i = 0; i < LW; ++i) rw[i] = chunk_of<T, W>(w + wrow[i] * p.ldw, k, d);
        };
        over = 0;
        ragged = false;
        if (k - sc * V + K <= d) {
            all(std::true_type{});
        } else if (d >= V) {
            over = run_over<T>(k, d);
            ragged = true;
#pragma unroll
            for (int i = 0; i < LA; ++i) rx[i] = chunk_of<T, true>(x + xrow[i] * ld, k - over, d);
#pragma unroll
            for (int i = 0; i < LW; ++i) rw[i] = chunk_of<T, true>(w + wrow[i] * p.ldw, k - over, d);
        } else {
            all(std::false_type{});
        }
    };
    auto store = [&](int buf) {
        if (ragged) {
#pragma unroll
            for (int i = 0; i < LA; ++i) rx[i] = moved_down<8 * (int)sizeof(T)>(rx[i], over);
#pragma unroll
            for (int i = 0; i < LW; ++i) rw[i] = moved_down<8 * (int)sizeof(T)>(rw[i], over);
        }
#pragma unroll
        for (int i = 0; i < LA; ++i) sx[buf][(i * RS + sr) * 8 + (sc ^ (sr & 7))] = rx[i];
#pragma unroll
        for (int i = 0; i < LW; ++i) {
            const int r = i * RS + sr;
            sw[buf][r * 8 + (sc ^ weight_key<T>(r))] = rw[i];
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
                const int r = wn + weight_row<T>(j, rho);
                fw[j] = sw[buf][r * 8 + (c ^ weight_key<T>(r))];
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) mma<T>(acc[i][j], fw[j], fx[i]);
        }
        if (s + 1 < steps) store(buf ^ 1);
        __syncthreads();
    }

    lin_epilogue<T, MT, NT, SPLIT>(acc, p, e, row0 + wm + rho, col0 + wn + g * V,
                                       row0 + BM <= p.n && col0 + BN <= p.m);
}

// The same product where every run of 16 bytes is whole and aligned: the steps go from memory straight to LDS, into two buffers.  When a step's
// first half has been multiplied its second half is in registers and its buffer free: the step after the next is sent for then, between the second
// half's products, and waited for in the middle of the next step, half a step to one step later.  A wave's load instruction fills 8 rows of 128 bytes, in order of its lanes: chunk c of row r lies at c ^ key(r) because the lane
// at that place asked for chunk c.  Beyond the end of the long axis a lane asks for zeros.
//
// What bounds it is that path: 65,536 x 2,048 by 1,024 takes 208 us without the loads and 223 without the products, and took 286 with a step's
// loads sent at once, because a wave that sends them stands until the memory pipeline has taken them all; dealt out between the
// products 264 to 270 (1,040 to 1,020 TFLOP/s).  Four or five steps of 64 bytes under way are slower than two of 128 (338 and 348 us for 300).
// A workgroup takes tiles one after the other, and the next one's first steps come while one is stored.
typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void mem_void;
static __device__ __align__(16) const uint32_t lin_zeros[4] = {0, 0, 0, 0};

template <int N> __device__ __forceinline__ void wait_loads_but()
{
    static_assert(N < 64, "");
    // vmcnt = N, and LDS reads all done (a buffer is overwritten after the next barrier)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4 | 0 << 8);
    asm volatile("" ::: "memory");
}

template <class T, class Tile, bool SPLIT>
__global__ __launch_bounds__(Tile::threads) __attribute__((amdgpu_waves_per_eu(Tile::waves_per_simd))) void k_lin_direct(Product p, Epilogue e, uint32_t total)
{
    constexpr int BM = Tile::BM, BN = Tile::BN, S = Tile::stages, waves = Tile::threads / 64;
    constexpr int V = 16 / (int)sizeof(T), C = kLinStep / 16, K = C * V;   // values of a run; runs and values of a step
    constexpr int MT = Tile::WM / 16, NT = Tile::WN / 16;
    constexpr int RW = 64 / C;                                         // rows that a load instruction fills
    constexpr int LX = BM / RW / waves, LW = BN / RW / waves;          // load instructions of a wave and step
    __shared__ u32x4 stage[S][(BM + BN) * C];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, rho = lane & 15;
    const int wm = wave / (BN / Tile::WN) * Tile::WM, wn = wave % (BN / Tile::WN) * Tile::WN;
    const int steps = (p.ka + K - 1) / K + (p.kb + K - 1) / K;
    if (lin_place(blockIdx.x, p.tiles_m).row * BM >= p.n) return;
    auto key_x = [](int r) { return r & 7; };
    auto key_w = [](int r) { return weight_key<T>(r); };

    // The lane's place in what its load instructions bring: row r of the first one, `gap` rows from each to the next (a multiple of what the
    // keys look at, so that a lane's columns are the same in all); the rows' places are computed anew for every load (a row and a stride in
    // bytes are numbers of 24 bits), the registers are wanted for the sums.
    constexpr int gap = RW * waves;
    static_assert(gap % 32 == 0 && S == 2, "");
    const int r0 = wave * RW + lane / C, xc = ((lane % C) ^ key_x(r0)) * V, wc = ((lane % C) ^ key_w(r0)) * V;
    // What is loaded: the steps of this workgroup's tiles, one after the other, a step and a half ahead of the products; where the next one
    // starts, in its source of width d, and zeros once the tiles have ended.
    const char *x = nullptr, *w = nullptr;
    int k = 0, d = 0, last_x = 0, last_w = 0;
    uint32_t ldx = 0, coming = blockIdx.x;
    const uint32_t ldw = (uint32_t)p.ldw * (uint32_t)sizeof(T);
    bool second = false;                       // of [a | b]
    auto next_source = [&]() {
        k = 0;
        if (d > 0 && !second && p.kb) {
            second = true;
            const LinPlace at = lin_place(coming - gridDim.x, p.tiles_m);
            x = (const char*)((const T*)p.b + at.row * BM * p.ldb);
            w = (const char*)((const T*)p.w + (int64_t)at.col * BN * p.ldw + p.ka);
            ldx = (uint32_t)p.ldb * (uint32_t)sizeof(T);
            d = p.kb;
            return;
        }
        second = false;
        d = 0;
        const LinPlace at = lin_place(coming, p.tiles_m);
        const int64_t row = at.row * BM;
        const int col = at.col * BN;
        if (coming >= total || row >= p.n) return;
        coming += gridDim.x;
        last_x = p.n - row < BM ? (int)(p.n - row) - 1 : BM - 1;
        last_w = p.m - col < BN ? p.m - col - 1 : BN - 1;
        x = (const char*)((const T*)p.a + row * p.lda);
        w = (const char*)((const T*)p.w + (int64_t)col * p.ldw);
        ldx = (uint32_t)p.lda * (uint32_t)sizeof(T);
        d = p.ka;
    };
    // load instruction i of a step, into buffer `to`
    auto load = [&](u32x4* to, int i) {
        const bool rows = i < LX;
        const int q = rows ? i : i - LX, at = r0 + q * gap, last = rows ? last_x : last_w, c = rows ? xc : wc;
        const void* from = (rows ? x : w) + (size_t)k * sizeof(T) +
                           (__umul24((uint32_t)(at < last ? at : last), rows ? ldx : ldw) + (uint32_t)c * (uint32_t)sizeof(T));
        from = k + c < d ? from : lin_zeros;
        __builtin_amdgcn_global_load_lds((mem_void*)from, (lds_void*)(to + wave * 64 + (rows ? 0 : BM * C) + q * waves * 64), 16, 0, 0);
    };

    // Operands: the rows' are read again for the next half step as soon as the last product with them is under way, the weights' have two
    // sets of registers.
    constexpr int J = V / 4;
    const int wr = weight_row<T>(0, rho), px0 = (wm + rho) * C, pw0 = BM * C + (wn + wr) * C;
    const int px[2] = {px0 + (g ^ key_x(rho)), px0 + ((4 + g) ^ key_x(rho))}, pw[2] = {pw0 + (g ^ key_w(wr)), pw0 + ((4 + g) ^ key_w(wr))};
    u32x4 fx[MT], fw[2][NT];
    f32x4 acc[MT][NT];
    auto read_x = [&](const u32x4* from, int h, int i) { fx[i] = from[px[h] + i * 16 * C]; };
    auto read_w = [&](const u32x4* from, int h) {
#pragma unroll
        for (int j = 0; j < NT; ++j) fw[h][j] = from[pw[h] + (j / J * (4 * V) + j % J * 4) * C];
    };
    // Half h of a step, with the next half's rows from `next` and, where LOADS, a step's loads into `to`, dealt out between the products: sent
    // at once they hold up the wave until the memory pipeline has taken them all.
    auto multiply = [&](int h, const u32x4* next, u32x4* to, auto loads) {
        constexpr bool LOADS = decltype(loads)::value;
        constexpr int each = (LX + LW + MT - 1) / MT;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int j = 0; j < NT; ++j) mma<T>(acc[i][j], fw[h][j], fx[i]);
            read_x(next, h ^ 1, i);
            if constexpr (LOADS)
#pragma unroll
                for (int q = i * each; q < (i + 1) * each; ++q)
                    if (q < LX + LW) load(to, q);
            __builtin_amdgcn_sched_barrier(0);     // as written
        }
    };

    auto wait = [&](auto wait_loads) {
        wait_loads();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // Loads and stores end in order.  A tile's second step was loaded before the tile before it was stored: the wait for it leaves the stores
    // under way.  stored: how many store instructions there were at least (whole tiles; 0 where that is not known).
    constexpr int stores = MT * NT * 4 / V;
    int stored = 0, now = 0;
    for (int q = 0; q < 2; ++q) {
        if (k >= d) next_source();
#pragma unroll
        for (int i = 0; i < LX + LW; ++i) load(stage[q], i);
        k += K;
    }
    wait([] { wait_loads_but<LX + LW>(); });
    for (uint32_t id = blockIdx.x; id < total; id += gridDim.x) {
        const LinPlace at = lin_place(id, p.tiles_m);
        const int64_t row0 = at.row * BM;
        const int col0 = at.col * BN;
        if (row0 >= p.n) break;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        read_w(stage[now], 0);
#pragma unroll
        for (int i = 0; i < MT; ++i) read_x(stage[now], 0, i);
        for (int s = 0; s < steps; ++s) {
            u32x4* here = stage[now];
            now ^= 1;
            const u32x4* next = stage[now];
            read_w(here, 1);
            multiply(0, here, nullptr, std::false_type{});
            // everyone has read this step's second half, and the next step has come
            wait([&] {
                if (s > 0) wait_loads_but<0>();
                else if (stored >= 2 * stores && 2 * stores < 64) wait_loads_but<2 * stores < 64 ? 2 * stores : 0>();
                else if (stored >= stores) wait_loads_but<stores>();
                else wait_loads_but<0>();
            });
            if (k >= d) next_source();
            read_w(next, 0);
            multiply(1, next, here, std::true_type{});
            k += K;
            asm volatile("" ::: "memory");             // (the reads stay on this side of the next wait)
        }
        const bool whole = row0 + BM <= p.n && col0 + BN <= p.m;
        lin_epilogue<T, MT, NT, SPLIT>(acc, p, e, row0 + wm + rho, col0 + wn + g * V, whole);
        if (SPLIT) stored = whole && e.out && e.out2 ? stores : 0;
        else stored = !whole ? 0 : e.pre ? 2 * stores : stores;
    }
    wait_loads_but<0>();                                // (zeros that are on their way: LDS is another workgroup's after the end)
}

// ---- dw = dz^T [a | b] ----------------------------------------------------------------------------------------------------
//
// 65,536 rows, 1,024 features by 2,048 columns from 8 bits, half precision: 307 us at the least, 344 for the median of twenty launches (895 and 798
// TFLOP/s); the operands' way through registers (where codes become values) and the turning reads, not the products, bound it.  In floats 2,006
// and 2,033 us, 137 and 135 of 154 TFLOP/s: there the products do.
// The long axis is the rows: a workgroup takes BM features of dz by BN columns of a or of b and a stretch of rows, and leaves its sums in
// 32 bits; k_lin_join adds the stretches in order.  Both operands lie with the long axis across their rows.  They are staged as
// they lie, and the reads from LDS turn them: for 16 bits the transposing read gives lane rho of 16 lanes four rows of column rho, where
// the lanes' addresses cover 4 rows of 16 columns; floats are read one by one.  A checkpoint's codes become values on the
// way to LDS, exactly.
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T> constexpr int kLinRows = kLinStep / (int)sizeof(T);        // rows of a step

// A run of columns of one row on its way to LDS: 16 bytes of values, or as many codes with their exponent.  The codes are turned into
// values when they are stored, a step later: the loads stay under way meanwhile.  WHOLE as above.
template <class T, bool CK> struct Staged {
    u32x4 v;
    template <bool WHOLE> __device__ __forceinline__ void load(const Rows& x, int64_t r, int c, int d)
    {
        v = WHOLE || c < d ? chunk_of<T, WHOLE>((const T*)x.data + r * x.stride, c, d) : u32x4{0, 0, 0, 0};
    }
    // the run at column c, read from `over` columns before it
    __device__ __forceinline__ void load_over(const Rows& x, int64_t r, int c, int, int over) { v = chunk_of<T, true>((const T*)x.data + r * x.stride, c - over, 0); }
    __device__ __forceinline__ void move_down(int over) { v = moved_down<8 * (int)sizeof(T)>(v, over); }
    __device__ __forceinline__ void clear() { v = u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ u32x4 values() const { return v; }
};

template <class T> struct Staged<T, true> {
    static constexpr int V = 16 / (int)sizeof(T);
    typedef uint32_t Codes __attribute__((ext_vector_type(V / 4)));
    struct __attribute__((packed, aligned(1))) Run8 {
        Codes q;
    };
    Codes q;
    int byte;
    template <bool WHOLE> __device__ __forceinline__ void load(const Rows& x, int64_t r, int c, int d)
    {
        const int8_t* row = (const int8_t*)x.data + r * x.stride;
        if constexpr (WHOLE) {
            byte = x.exponents[r * x.exponent_stride + c / kCkGroup];
            q = ((const Run8*)(row + c))->q;
            return;
        }
        clear();
        if (c >= d) return;
        byte = x.exponents[r * x.exponent_stride + c / kCkGroup];
        int8_t v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = c + i < d ? row[c + i] : (int8_t)0;
        __builtin_memcpy(&q, v, V);
    }
    __device__ __forceinline__ void load_over(const Rows& x, int64_t r, int c, int d, int over)
    {
        byte = x.exponents[r * x.exponent_stride + (c < d ? c : d - 1) / kCkGroup];
        q = ((const Run8*)((const int8_t*)x.data + r * x.stride + (c - over)))->q;
    }
    __device__ __forceinline__ void move_down(int over)
    {
        uint64_t w = 0;
        __builtin_memcpy(&w, &q, V);
        w = over < V ? w >> (8 * over) : 0ull;
        __builtin_memcpy(&q, &w, V);
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < V / 4; ++i) q[i] = 0u;
        byte = kCkBias;
    }
    __device__ __forceinline__ u32x4 values() const
    {
        const float scale = ck_scale(byte);
        T v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (T)((float)((int32_t)(q[i / 4] << (24 - 8 * (i % 4))) >> 24) * scale);
        u32x4 out;
        __builtin_memcpy(&out, v, 16);
        return out;
    }
};

template <class T, bool CK, class Tile>
__global__ __launch_bounds__(Tile::threads) void k_lin_weight(const T* __restrict__ dz, int64_t lddz, Rows a, Rows b, int64_t n, int ka,
                                                              int kb, int m, int tiles_a, int64_t stretch, float* __restrict__ partial)
{
    constexpr int BM = Tile::BM, BN = Tile::BN, threads = Tile::threads;
    constexpr int V = 16 / (int)sizeof(T), R = kLinRows<T>;
    constexpr int MT = Tile::WM / 16, NT = Tile::WN / 16;
    constexpr int CM = BM / V, CN = BN / V;                      // chunks of a row
    constexpr int LM = R * CM / threads, LN = R * CN / threads;  // chunks a thread stages
    // rows are padded by 32 bytes (16 bits) or 64 (floats): the reads of one instruction then cover all banks evenly
    constexpr int PM = CM + (sizeof(T) == 2 ? 2 : 4), PN = CN + (sizeof(T) == 2 ? 2 : 4);
    __shared__ u32x4 sz[2][R * PM], sx[2][R * PN];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, rho = lane & 15;
    const int col0 = (int)blockIdx.x * BM;                           // of dz
    const bool first = (int)blockIdx.y < tiles_a;
    const Rows x = first ? a : b;
    const int k0 = (first ? (int)blockIdx.y : (int)blockIdx.y - tiles_a) * BN, kd = first ? ka : kb;
    const int64_t lo = (int64_t)blockIdx.z * stretch, hi = lo + stretch < n ? lo + stretch : n;
    const int wm = wave / (BN / Tile::WN) * Tile::WM, wn = wave % (BN / Tile::WN) * Tile::WN;

    u32x4 rz[LM];
    Staged<T, CK> rx[LN];
    const bool cols_whole = col0 + BM <= m && k0 + BN <= kd, wide = m >= V && kd >= V;
    static_assert(threads % CM == 0 && threads % CN == 0, "");          // a thread's runs all start at one column
    const int cz = col0 + ((int)threadIdx.x % CM) * V, cx = k0 + ((int)threadIdx.x % CN) * V;
    const int oz = wide ? run_over<T>(cz, m) : 0, ox = wide ? run_over<T>(cx, kd) : 0;
    bool ragged = false;
    auto load = [&](int64_t from) {
        auto all = [&](auto whole) {
            constexpr bool W = decltype(whole)::value;
#pragma unroll
            for (int i = 0; i < LM; ++i) {
                const int q = i * threads + (int)threadIdx.x, r = q / CM, c = col0 + (q % CM) * V;
                rz[i] = W || (from + r < hi && c < m) ? chunk_of<T, W>(dz + (from + r) * lddz, c, m) : u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < LN; ++i) {
                const int q = i * threads + (int)threadIdx.x, r = q / CN, c = k0 + (q % CN) * V;
                if (W || from + r < hi) rx[i].template load<W>(x, from + r, c, kd);
                else rx[i].clear();
            }
        };
        ragged = false;
        if (cols_whole && from + R <= hi) {
            all(std::true_type{});
        } else if (wide && from + R <= hi) {
            ragged = true;
#pragma unroll
            for (int i = 0; i < LM; ++i) rz[i] = chunk_of<T, true>(dz + (from + (i * threads + (int)threadIdx.x) / CM) * lddz, cz - oz, m);
#pragma unroll
            for (int i = 0; i < LN; ++i) rx[i].load_over(x, from + (i * threads + (int)threadIdx.x) / CN, cx, kd, ox);
        } else {
            all(std::false_type{});
        }
    };
    auto store = [&](int buf) {
        if (ragged) {
#pragma unroll
            for (int i = 0; i < LM; ++i) rz[i] = moved_down<8 * (int)sizeof(T)>(rz[i], oz);
#pragma unroll
            for (int i = 0; i < LN; ++i) rx[i].move_down(ox);
        }
#pragma unroll
        for (int i = 0; i < LM; ++i) {
            const int q = i * threads + (int)threadIdx.x;
            sz[buf][(q / CM) * PM + q % CM] = rz[i];
        }
#pragma unroll
        for (int i = 0; i < LN; ++i) {
            const int q = i * threads + (int)threadIdx.x;
            sx[buf][(q / CN) * PN + q % CN] = rx[i].values();
        }
    };
    // 16 columns from `col` on by half h of the step's rows
    auto operand = [&](const u32x4* s, int pitch, int col, int h) {
        if constexpr (sizeof(T) == 2) {
            const char* p = (const char*)s + (size_t)(h * 32 + g * 4 + (rho >> 2)) * (size_t)(pitch * 16) + (size_t)(col + (rho & 3) * 4) * 2;
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
            const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + (size_t)(16 * pitch * 16)));
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

// ---- dz and dbias ---------------------------------------------------------------------------------------------------------
//
// One pass over dout and z: dz rounded to its type, and the columns' sums of the unrounded dz, a partial row per workgroup
// (its 256 threads are 32 runs of columns by 8 rows).
constexpr int kLinDzCols = 32, kLinDzRows = 8;

template <class T> struct Slope {
    const T *dout, *pre;
    T* dz;
    int64_t ldd, ldp, lddz, n;
    float* partial;                 // or NULL
    int m, parts, across;           // workgroups over the rows, over the columns
};

template <class T, bool EVEN, int ACT> __device__ __forceinline__ void lin_slope(const Slope<T>& p, int part, int piece)
{
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ float sums[kLinDzRows][kLinDzCols * V + 1];
    const int col = threadIdx.x % kLinDzCols, slot = threadIdx.x / kLinDzCols, m = p.m;
    const int c = (piece * kLinDzCols + col) * V;
    float s[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = 0.0f;
    if (c < m)
        for (int64_t r = (int64_t)part * kLinDzRows + slot; r < p.n; r += (int64_t)p.parts * kLinDzRows) {
            float f[V], z[V];
            const WordsOf<T, V> wf = load_words<T, V, EVEN>(p.dout + r * p.ldd, c, m);
            WordsOf<T, V> wz;
            if constexpr (ACT != GREM_ACT_NONE) wz = load_words<T, V, EVEN>(p.pre + r * p.ldp, c, m);
            to_floats<T, V>(wf, f);
            if constexpr (ACT != GREM_ACT_NONE) {
                to_floats<T, V>(wz, z);
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] *= act_slope<T, ACT>(z[i]);
                store_floats<T, V, true>(p.dz + r * p.lddz, c, m, f);          // (zeros up to lddz)
            }
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] += f[i];
        }
    if (!p.partial) return;
#pragma unroll
    for (int i = 0; i < V; ++i) sums[slot][col * V + i] = s[i];
    __syncthreads();
    for (int i = threadIdx.x; i < kLinDzCols * V; i += kLinBlock) {
        const int at = piece * kLinDzCols * V + i;
        float t = 0.0f;
#pragma unroll
        for (int q = 0; q < kLinDzRows; ++q) t += sums[q][i];
        if (at < m) p.partial[(size_t)part * (size_t)m + at] = t;
    }
}

// w (m x width) turned: wt (width x m, zeros up to ldt), so that dz w is a product of the first kind; dz and wt are both filled up with zeros to
// whole runs, and the product takes those as well
template <class T> struct Turn {
    const T* w;
    T* wt;
    int64_t ldw, ldt;
    int m, width;
    uint32_t across, tiles;         // tiles of 32 along the width, and in all
};

// (a launch takes fewer than 2^32 threads: beyond this many tiles, 2^30 weights, a workgroup takes several)
constexpr uint32_t kLinTurns = 1 << 20;

template <class T> __device__ __forceinline__ void lin_turn(const Turn<T>& p, uint32_t first, uint32_t turns)
{
    __shared__ T tile[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    for (uint32_t piece = first; piece < p.tiles; piece += turns) {
        const int c0 = (int)(piece % p.across) * 32, f0 = (int)(piece / p.across) * 32;
        if (piece != first) __syncthreads();
#pragma unroll
        for (int i = 0; i < 32; i += 8)
            if (f0 + y + i < p.m && c0 + x < p.width) tile[y + i][x] = p.w[(int64_t)(f0 + y + i) * p.ldw + c0 + x];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 32; i += 8)
            if (c0 + y + i < p.width && f0 + x < p.ldt) p.wt[(int64_t)(c0 + y + i) * p.ldt + f0 + x] = f0 + x < p.m ? tile[x][y + i] : (T)0.0f;
    }
}

// What the products wait for, in one launch: the turned weights' workgroups first, dz's after them.
template <class T, bool EVEN, int ACT>
__global__ __launch_bounds__(kLinBlock) void k_lin_prepare(Slope<T> slope, Turn<T> turn, uint32_t turns)
{
    if (blockIdx.x < turns) {
        lin_turn<T>(turn, blockIdx.x, turns);
    } else {
        const uint32_t at = blockIdx.x - turns;
        lin_slope<T, EVEN, ACT>(slope, (int)(at / (uint32_t)slope.across), (int)(at % (uint32_t)slope.across));
    }
}

// The partial sums of both parameters, added up in order: dbias by the first workgroups, 16 columns each, dw[f][c] = the sum over the
// stretches by the others.
template <class T>
__global__ __launch_bounds__(kJoinBlock) void k_lin_join(const float* __restrict__ bias_parts, int parts, int m, T* __restrict__ dbias, uint32_t biases,
                                                         const float* __restrict__ partial, int stretches, int64_t values, int width,
                                                         T* __restrict__ dw, int64_t lddw)
{
    if (blockIdx.x < biases) {
        __shared__ float sums[kJoinSlices][kJoinCols + 1];
        const int64_t c = (int64_t)blockIdx.x * kJoinCols + threadIdx.x % kJoinCols;
        const float total = join_columns(bias_parts, parts, m, c, sums);
        if (threadIdx.x < kJoinCols && c < m) dbias[c] = (T)total;
        return;
    }
    for (int64_t i = (int64_t)(blockIdx.x - biases) * kJoinBlock + threadIdx.x; i < values; i += (int64_t)(gridDim.x - biases) * kJoinBlock) {
        float s = 0.0f;
#pragma unroll 4
        for (int q = 0; q < stretches; ++q) s += partial[(int64_t)q * values + i];
        dw[i / width * lddw + i % width] = (T)s;
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------
constexpr int64_t kLinMostStride = 1 << 23;                  // bytes

template <class T, bool SPLIT> void lin_product(const Product& p, const Epilogue& e, hipStream_t stream)
{
    // where all runs of 16 bytes are whole and aligned, and a block's rows lie within 2^31 bytes: straight to LDS
    const uint64_t places = (uint64_t)p.a | (uint64_t)p.w | (uint64_t)(p.kb ? p.b : nullptr) |
                            (uint64_t)((p.lda | p.ldw | p.ka | (p.kb ? p.ldb | p.kb : 0)) * (int64_t)sizeof(T));
    const int64_t most = kLinMostStride / (int64_t)sizeof(T);
    const bool direct = places % 16 == 0 && p.lda < most && p.ldw < most && (p.kb == 0 || p.ldb < most);
    auto run = [&](auto tile) {
        using Tile = decltype(tile);
        Product q = p;
        q.tiles_m = (int)((p.m + Tile::BN - 1) / Tile::BN);
        const int64_t blocks = (p.n + Tile::BM - 1) / Tile::BM;
        const uint32_t total = (uint32_t)((blocks + 7) / 8 * 8 * q.tiles_m), once = 256u * Tile::per_cu;
        if (direct) hipLaunchKernelGGL((k_lin_direct<T, Tile, SPLIT>), dim3(total < once ? total : once), dim3(Tile::threads), 0, stream, q, e, total);
        else hipLaunchKernelGGL((k_lin_product<T, Tile, SPLIT>), dim3(total), dim3(Tile::threads), 0, stream, q, e);
    };
    // the largest tile of which there are enough for the CUs
    auto tiles = [&](int64_t t) { return ((p.n + t - 1) / t) * ((p.m + t - 1) / t); };
    // (floats: four times the instructions a step, so that the smaller tile's loads are hidden too)
    if constexpr (sizeof(T) == 2)
        if (p.m > 128 && tiles(256) >= 192) return run(LinTile<256, 256, 128, 64>{});
    // (and beyond 2^29 rows of few features: a launch takes fewer than 2^32 threads)
    if ((p.m > 64 || p.n > (1 << 29)) && tiles(128) >= 192) run(LinTile<128, 128, 64, 64>{});
    else run(LinTile<64, 64, 32, 32>{});
}

// the backward pass's workspace
struct LinSpace {
    int64_t lddz, ldt, stretch;
    int stretches, parts, tile;
    size_t o_dz, o_wt, o_dw, o_bias, bytes;
};

int lin_weight_tile(int64_t n, int64_t m, int64_t ka, int64_t kb)
{
    return n >= 4096 && m > 128 && (ka > 128 || kb > 128) ? 256 : 128;
}

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
    s.tile = lin_weight_tile(n, m, ka, kb);
    const int64_t t = s.tile, tiles = ((m + t - 1) / t) * ((ka + t - 1) / t + (kb + t - 1) / t);
    const int64_t groups = t == 256 ? 256 : 512;
    int64_t want = groups / tiles;
    const int64_t most = (n + 8 * rows - 1) / (8 * rows);
    if (want > most) want = most;
    if (want < 1) want = 1;
    s.stretch = (n + want - 1) / want;
    s.stretch = (s.stretch + rows - 1) / rows * rows;
    if (s.stretch < rows) s.stretch = rows;
    s.stretches = (int)((n + s.stretch - 1) / s.stretch);
    if (s.stretches < 1) s.stretches = 1;
    s.o_dw = carve((size_t)s.stretches * (size_t)m * (size_t)(ka + kb) * 4);
    // workgroups of the pass that makes dz: about 2,048, over all columns
    const int64_t across = (m + kLinDzCols * V - 1) / (kLinDzCols * V), down = (2048 + across - 1) / across;
    s.parts = (int)((n + kLinDzRows - 1) / kLinDzRows);
    if (s.parts > down) s.parts = (int)down;
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
    const Product p{a, b, w, lda, ldb, ldw, n, (int)ka, (int)kb, (int)m, 0};
    const Epilogue e{bias, residual, out, pre, nullptr, ldr, ldo, ldp, 0, 0, activation};
    layer_typed(type, [&](auto t) { lin_product<decltype(t), false>(p, e, (hipStream_t)stream); });
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
    if (const int rc = layer_space(workspace, workspace_bytes, s.bytes)) return rc;
    if (n == 0 && !dw && !dbias) return GREM_OK;
    hipStream_t stream = (hipStream_t)stream_;
    uint8_t* ws = (uint8_t*)workspace;
    layer_typed(type, [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / (int)sizeof(T);
        const T* dz = (const T*)dout;
        int64_t lddz = ldd;
        float* bias_parts = dbias ? (float*)(ws + s.o_bias) : nullptr;
        float* parts = (float*)(ws + s.o_dw);
        T* wt = (T*)(ws + s.o_wt);
        const bool slopes = n && (activation != GREM_ACT_NONE || dbias), turned = n && (da || db);
        if (slopes || turned) {
            T* made = (T*)(ws + s.o_dz);
            const int across = (int)((m + kLinDzCols * V - 1) / (kLinDzCols * V));
            const uint32_t wide = (uint32_t)((ka + kb + 31) / 32), tiles = wide * (uint32_t)((m + 31) / 32);
            const Slope<T> slope{(const T*)dout, (const T*)pre, made, ldd, ldp, s.lddz, n, bias_parts, (int)m, s.parts, across};
            const Turn<T> turn{(const T*)w, wt, ldw, s.ldt, (int)m, (int)(ka + kb), wide, tiles};
            const uint32_t turns = !turned ? 0u : tiles < kLinTurns ? tiles : kLinTurns;
            const uint32_t grid = turns + (slopes ? (uint32_t)s.parts * (uint32_t)across : 0u);
            by_act(activation, [&](auto act) {
                layer_either(m % V == 0, [&](auto even) {
                    hipLaunchKernelGGL((k_lin_prepare<T, decltype(even)::value, decltype(act)::value>), dim3(grid), dim3(kLinBlock), 0, stream, slope,
                                       turn, turns);
                });
            });
            if (activation != GREM_ACT_NONE) {
                dz = made;
                lddz = s.lddz;
            }
        }
        if (turned) {
            const int inner = activation != GREM_ACT_NONE ? (int)s.lddz : (int)m;
            const Product p{dz, nullptr, wt, lddz, 0, s.ldt, n, inner, 0, (int)(ka + kb), 0};
            const Epilogue e{nullptr, nullptr, da, nullptr, db, 0, ldda, 0, lddb, (int)ka, GREM_ACT_NONE};
            lin_product<T, true>(p, e, stream);
        }
        if (dw) {
            const Rows xa = n ? layer_rows(a) : Rows{}, xb = n && kb ? layer_rows(b) : Rows{};
            auto weight = [&](auto packed, auto tile) {
                using Tile = decltype(tile);
                const int tiles_a = (int)((ka + Tile::BN - 1) / Tile::BN), tiles_b = (int)((kb + Tile::BN - 1) / Tile::BN);
                hipLaunchKernelGGL((k_lin_weight<T, decltype(packed)::value, Tile>),
                                   dim3((unsigned)((m + Tile::BM - 1) / Tile::BM), (unsigned)(tiles_a + tiles_b), (unsigned)s.stretches),
                                   dim3(Tile::threads), 0, stream, dz, lddz, xa, xb, n, (int)ka, (int)kb, (int)m, tiles_a, s.stretch, parts);
            };
            auto by_tile = [&](auto packed) {
                if (s.tile == 256) weight(packed, LinTile<256, 256, 128, 64>{});
                else weight(packed, LinTile<128, 128, 64, 64>{});
            };
            if (n && a->exponents) by_tile(std::integral_constant<bool, true>{});
            else by_tile(std::integral_constant<bool, false>{});
        }
        if (dw || dbias) {
            const uint32_t biases = dbias ? (uint32_t)((m + kJoinCols - 1) / kJoinCols) : 0u;
            const int64_t values = dw ? m * (ka + kb) : 0, groups = (values + kJoinBlock - 1) / kJoinBlock;
            hipLaunchKernelGGL((k_lin_join<T>), dim3(biases + (unsigned)(groups < 2048 ? groups : 2048)), dim3(kJoinBlock), 0, stream, bias_parts,
                               n ? s.parts : 0, (int)m, (T*)dbias, biases, parts, s.stretches, values, (int)(ka + kb), (T*)dw, lddw);
        }
    });
    return layer_launched();
}
