// The mean of the neighbours' rows over a CSR graph, inside the partitions of a labelling, and its gradient, for gfx950.
//   N(v) = entries u of row v with labels[u] = labels[v] >= 0 (without labels: all entries), as stored, loops and duplicates included
//   out[v] = sum of x[u] over N(v) / |N(v)|, zero where N(v) is empty
//   dx[u]  = sum over the v that have u in N(v) of dout[v] / |N(v)|: the same walk over the transposed graph with a weight per entry
//
// The rows are gathered: an entry costs a row of d values from wherever it lies, and what bounds the kernels is how many such reads are
// under way and how many of them the caches serve.  A wave takes a vertex.  64 entries at a time it reads columns and labels, moves the
// entries that count to the front (a permutation of the lanes, so rows of other partitions are never touched), and then L lanes read
// a neighbour's row, 16 bytes each, 64/L neighbours side by side and four such sets under way.  Sums are held in 32 bits per lane and
// joined over the wave at the end.
// Rows of more than `segment` entries go on a list, are summed in segments by as many waves, and joined in order: no atomics on
// values, the same bytes on every run.
#include "grem_layers.hip.h"

namespace {

constexpr int kNmBlock = 256;
constexpr int kNmWaves = kNmBlock / 64;
constexpr int64_t kNmSegment = 512;             // entries a wave takes alone, at least
constexpr int64_t kNmMostSegments = 65536;      // longer segments rather than more of them

struct NmItem {
    int32_t row, segment;
};
struct NmLong {
    int32_t row, first, count, unused;
};

template <class T> constexpr int kNmV = 16 / (int)sizeof(T);

__device__ __forceinline__ int64_t nm_start(const void* __restrict__ rowptr, int bits, int64_t v)
{
    return bits == 64 ? ((const int64_t*)rowptr)[v] : (int64_t)((const int32_t*)rowptr)[v];
}

// Adds up the counted entries of [lo, hi) for columns [c0, c0 + L*V*C); every lane ends with the sums of its columns over its own
// neighbours.  Returns how many entries counted.
template <class T, bool EVEN, bool WEIGHTED, int L, int C>
__device__ __forceinline__ int nm_walk(const int32_t* __restrict__ colidx, int64_t lo, int64_t hi, const int32_t* __restrict__ labels, int32_t mine,
                                       const int32_t* __restrict__ counts, const T* __restrict__ x, int64_t ldx, int c0, int d,
                                       float (&acc)[C][kNmV<T>])
{
    constexpr int V = kNmV<T>, G = 64 / L, U = 4;
    const int lane = threadIdx.x & 63, part = lane / L, c = c0 + (lane % L) * V;
    int total = 0;
    for (int64_t base = lo; base < hi; base += 64) {
        const int64_t e = base + lane;
        int32_t u = e < hi ? colidx[e] : 0;
        bool keep = e < hi;
        if (labels && keep) keep = labels[u] == mine;
        const unsigned long long mask = __ballot(keep), below = (1ull << lane) - 1ull;
        const int kept = __popcll(mask);
        total += kept;
        if (kept == 0) continue;
        const int to = keep ? __popcll(mask & below) : kept + __popcll(~mask & below);
        u = __builtin_amdgcn_ds_permute(to * 4, u);
        float w = 1.0f;
        if constexpr (WEIGHTED) {
            if (lane < kept) {
                const int32_t k = counts[u];
                w = 1.0f / (float)(k > 1 ? k : 1);
            }
        }
        for (int j = 0; j < kept; j += G * U) {
            WordsOf<T, V> f[U][C];
            float g[U];
#pragma unroll
            for (int q = 0; q < U; ++q) {
                const int at = j + q * G + part;
                const int32_t from = __shfl(u, at & 63);
                g[q] = WEIGHTED ? __shfl(w, at & 63) : 1.0f;
                const int end = at < kept ? d : 0;
#pragma unroll
                for (int k = 0; k < C; ++k) f[q][k] = load_words<T, V, EVEN>(x + (int64_t)from * ldx, c + k * L * V, end);
            }
#pragma unroll
            for (int q = 0; q < U; ++q)
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    float v[V];
                    to_floats<T, V>(f[q][k], v);
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[k][i] += WEIGHTED ? v[i] * g[q] : v[i];
                }
        }
    }
#pragma unroll
    for (int k = 0; k < C; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int o = L; o < 64; o <<= 1) acc[k][i] += __shfl_xor(acc[k][i], o);
    return total;
}

template <class T, bool EVEN, bool WEIGHTED, int L, int C>
__global__ __launch_bounds__(kNmBlock) void k_nm_rows(const void* __restrict__ rowptr, int bits, const int32_t* __restrict__ colidx, int64_t n,
                                                      const int32_t* __restrict__ labels, const int32_t* __restrict__ counts,
                                                      const T* __restrict__ x, int64_t ldx, int d, T* __restrict__ out, int64_t ldo,
                                                      int32_t* __restrict__ counts_out, int64_t segment, uint32_t* __restrict__ found,
                                                      NmItem* __restrict__ items, NmLong* __restrict__ longs)
{
    constexpr int V = kNmV<T>;
    const int lane = threadIdx.x & 63;
    for (int64_t v = (int64_t)blockIdx.x * kNmWaves + (threadIdx.x >> 6); v < n; v += (int64_t)gridDim.x * kNmWaves) {
        const int64_t lo = nm_start(rowptr, bits, v), hi = nm_start(rowptr, bits, v + 1);
        const int32_t mine = labels ? labels[v] : 0;
        if (hi - lo > segment && mine >= 0) {
            const int32_t count = (int32_t)((hi - lo + segment - 1) / segment);
            int32_t first = 0;
            if (lane == 0) {
                first = (int32_t)atomicAdd(&found[0], (uint32_t)count);
                longs[atomicAdd(&found[1], 1u)] = NmLong{(int32_t)v, first, count, 0};
            }
            first = __shfl(first, 0);
            for (int32_t i = lane; i < count; i += 64) items[first + i] = NmItem{(int32_t)v, i};
            continue;
        }
        for (int c0 = 0; c0 < d; c0 += L * V * C) {
            float acc[C][V];
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[k][i] = 0.0f;
            const int total = nm_walk<T, EVEN, WEIGHTED, L, C>(colidx, lo, mine >= 0 ? hi : lo, labels, mine, counts, x, ldx, c0, d, acc);
            if (lane >= L) continue;
            if (c0 == 0 && lane == 0 && counts_out) counts_out[v] = total;
            const float scale = WEIGHTED ? 1.0f : 1.0f / (float)(total > 1 ? total : 1);
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const int c = c0 + (k * L + lane) * V;
#pragma unroll
                for (int i = 0; i < V; ++i) acc[k][i] *= scale;
                if (c < d) store_floats<T, V, EVEN>(out + v * ldo, c, d, acc[k]);
            }
        }
    }
}

__global__ void k_nm_clear(uint32_t* __restrict__ found)
{
    if (threadIdx.x < 2) found[threadIdx.x] = 0u;
}

// the listed segments, a wave each: sums into partial (a row of d floats an item), counts beside them
template <class T, bool EVEN, bool WEIGHTED, int L, int C>
__global__ __launch_bounds__(kNmBlock) void k_nm_segments(const void* __restrict__ rowptr, int bits, const int32_t* __restrict__ colidx,
                                                          const int32_t* __restrict__ labels, const int32_t* __restrict__ counts,
                                                          const T* __restrict__ x, int64_t ldx, int d, int64_t segment,
                                                          const uint32_t* __restrict__ found, const NmItem* __restrict__ items,
                                                          float* __restrict__ partial, int32_t* __restrict__ part_counts)
{
    constexpr int V = kNmV<T>;
    const int lane = threadIdx.x & 63;
    const uint32_t total_items = found[0];
    for (uint32_t it = blockIdx.x * kNmWaves + (threadIdx.x >> 6); it < total_items; it += gridDim.x * kNmWaves) {
        const NmItem item = items[it];
        const int64_t lo = nm_start(rowptr, bits, item.row) + item.segment * segment, end = nm_start(rowptr, bits, (int64_t)item.row + 1);
        const int64_t hi = lo + segment < end ? lo + segment : end;
        for (int c0 = 0; c0 < d; c0 += L * V * C) {
            float acc[C][V];
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[k][i] = 0.0f;
            const int total = nm_walk<T, EVEN, WEIGHTED, L, C>(colidx, lo, hi, labels, labels ? labels[item.row] : 0, counts, x, ldx, c0, d, acc);
            if (lane >= L) continue;
            if (c0 == 0 && lane == 0) part_counts[it] = total;
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const int c = c0 + (k * L + lane) * V;
                if (c < d) store_floats<float, V, EVEN>(partial + (size_t)it * (size_t)d, c, d, acc[k]);
            }
        }
    }
}

// A long row's segments added up, a workgroup a row: the columns 256/S at a time, S threads a column over every S-th segment, then
// those S in order.
template <class T, bool WEIGHTED>
__global__ __launch_bounds__(kNmBlock) void k_nm_join(int d, const uint32_t* __restrict__ found, const NmLong* __restrict__ longs,
                                                      const float* __restrict__ partial, const int32_t* __restrict__ part_counts,
                                                      T* __restrict__ out, int64_t ldo, int32_t* __restrict__ counts_out)
{
    constexpr int S = 8, W = kNmBlock / S;
    __shared__ float sums[S][W];
    __shared__ int totals[kNmBlock];
    const int q = threadIdx.x / W, i = threadIdx.x % W;
    const uint32_t rows = found[1];
    for (uint32_t l = blockIdx.x; l < rows; l += gridDim.x) {
        const NmLong r = longs[l];
        int total = 0;
        for (int s = threadIdx.x; s < r.count; s += kNmBlock) total += part_counts[r.first + s];
        totals[threadIdx.x] = total;
        __syncthreads();
        for (int o = kNmBlock / 2; o > 0; o >>= 1) {
            if (threadIdx.x < o) totals[threadIdx.x] += totals[threadIdx.x + o];
            __syncthreads();
        }
        total = totals[0];
        if (threadIdx.x == 0 && counts_out) counts_out[r.row] = total;
        const float scale = WEIGHTED ? 1.0f : 1.0f / (float)(total > 1 ? total : 1);
        for (int c0 = 0; c0 < d; c0 += W) {
            float a = 0.0f;
            if (c0 + i < d)
                for (int s = q; s < r.count; s += S) a += partial[(size_t)(r.first + s) * (size_t)d + c0 + i];
            sums[q][i] = a;
            __syncthreads();
            if (q == 0 && c0 + i < d) {
                float all = 0.0f;
#pragma unroll
                for (int s = 0; s < S; ++s) all += sums[s][i];
                out[(int64_t)r.row * ldo + c0 + i] = (T)(all * scale);
            }
            __syncthreads();
        }
    }
}

// what a call keeps in its workspace
struct NmSpace {
    int64_t segment, items;
    size_t o_items, o_longs, o_counts, o_partial, bytes;
};

NmSpace nm_space(int64_t nnz, int64_t d)
{
    NmSpace s;
    s.segment = (nnz + kNmMostSegments - 1) / kNmMostSegments;
    if (s.segment < kNmSegment) s.segment = kNmSegment;
    // a row of e > segment entries has fewer than 2e / segment segments
    s.items = nnz > s.segment ? 2 * (nnz / s.segment) + 1 : 0;
    size_t off = 256;
    auto carve = [&](size_t bytes) { const size_t at = off; off += layer_align(bytes); return at; };
    s.o_items = carve((size_t)s.items * sizeof(NmItem));
    s.o_longs = carve((size_t)s.items * sizeof(NmLong));
    s.o_counts = carve((size_t)s.items * 4);
    s.o_partial = carve((size_t)s.items * (size_t)d * 4);
    s.bytes = s.items ? off : 0;
    return s;
}

struct NmL8 { static constexpr int L = 8, C = 1; };
struct NmL16 { static constexpr int L = 16, C = 1; };
struct NmL32 { static constexpr int L = 32, C = 1; };
struct NmL64 { static constexpr int L = 64, C = 1; };
struct NmL64x2 { static constexpr int L = 64, C = 2; };

template <class T, class F> void nm_shaped(int64_t d, F f)
{
    constexpr int V = kNmV<T>;
    if (d <= 8 * V) f(NmL8{});
    else if (d <= 16 * V) f(NmL16{});
    else if (d <= 32 * V) f(NmL32{});
    else if (d <= 64 * V) f(NmL64{});
    else f(NmL64x2{});
}

int nm_run(const void* rowptr, int32_t bits, const int32_t* colidx, int64_t nnz, int64_t n, const int32_t* labels, int32_t type, int64_t d,
           const void* x, int64_t ldx, const int32_t* counts, bool weighted, void* out, int64_t ldo, int32_t* counts_out, void* workspace,
           size_t workspace_bytes, hipStream_t stream)
{
    const int size = layer_size(type);
    if (!size || n < 0 || n > kLayerMaxRows || nnz < 0 || d < 1 || d > kLayerMaxCols || (bits != 32 && bits != 64) || (n && !rowptr) ||
        (nnz && !colidx) || !layer_rows_ok(x, ldx, n, d, size) || !layer_rows_ok(out, ldo, n, d, size) || (weighted && n && !counts))
        return GREM_ERR_ARG;
    if (n == 0) return GREM_OK;
    const NmSpace s = nm_space(nnz, d);
    if (s.bytes && (!workspace || workspace_bytes < s.bytes)) return GREM_ERR_NOMEM;
    uint8_t* ws = (uint8_t*)workspace;
    uint32_t* found = (uint32_t*)ws;
    NmItem* items = s.items ? (NmItem*)(ws + s.o_items) : nullptr;
    NmLong* longs = s.items ? (NmLong*)(ws + s.o_longs) : nullptr;
    int32_t* part_counts = s.items ? (int32_t*)(ws + s.o_counts) : nullptr;
    float* partial = s.items ? (float*)(ws + s.o_partial) : nullptr;
    const int64_t groups = (n + kNmWaves - 1) / kNmWaves;
    const unsigned grid = (unsigned)(groups < (1 << 22) ? groups : 1 << 22);
    const unsigned seg_grid = (unsigned)(s.items / kNmWaves + 1 < 2048 ? s.items / kNmWaves + 1 : 2048);
    const unsigned join_grid = (unsigned)(s.items < 1024 ? s.items : 1024);
    if (s.items) hipLaunchKernelGGL(k_nm_clear, dim3(1), dim3(64), 0, stream, found);
    layer_typed(type, [&](auto t) {
        using T = decltype(t);
        nm_shaped<T>(d, [&](auto shape) {
            constexpr int L = decltype(shape)::L, C = decltype(shape)::C;
            auto run = [&](auto even, auto w) {
                constexpr bool E = decltype(even)::value, W = decltype(w)::value;
                hipLaunchKernelGGL((k_nm_rows<T, E, W, L, C>), dim3(grid), dim3(kNmBlock), 0, stream, rowptr, bits, colidx, n, labels, counts,
                                   (const T*)x, ldx, (int)d, (T*)out, ldo, counts_out, s.segment, found, items, longs);
                if (!s.items) return;
                hipLaunchKernelGGL((k_nm_segments<T, E, W, L, C>), dim3(seg_grid), dim3(kNmBlock), 0, stream, rowptr, bits, colidx, labels,
                                   counts, (const T*)x, ldx, (int)d, s.segment, found, items, partial, part_counts);
                hipLaunchKernelGGL((k_nm_join<T, W>), dim3(join_grid), dim3(kNmBlock), 0, stream, (int)d, found, longs, partial,
                                   part_counts, (T*)out, ldo, counts_out);
            };
            layer_either(d % kNmV<T> == 0, [&](auto even) { layer_either(weighted, [&](auto w) { run(even, w); }); });
        });
    });
    return layer_launched();
}

}  // namespace

extern "C" size_t grem_neighbour_mean_bytes(int64_t nnz, int64_t d)
{
    return nnz < 0 || d < 1 || d > kLayerMaxCols ? 0 : nm_space(nnz, d).bytes;
}

extern "C" int grem_neighbour_mean(const void* rowptr, int32_t rowptr_bits, const int32_t* colidx, int64_t nnz, int64_t n,
                                   const int32_t* labels, int32_t type, int64_t d, const void* x, int64_t ldx, void* out, int64_t ldo,
                                   int32_t* counts_out, void* workspace, size_t workspace_bytes, void* stream)
{
    return nm_run(rowptr, rowptr_bits, colidx, nnz, n, labels, type, d, x, ldx, nullptr, false, out, ldo, counts_out, workspace,
                  workspace_bytes, (hipStream_t)stream);
}

extern "C" int grem_neighbour_mean_backward(const void* rowptr_t, int32_t rowptr_bits, const int32_t* colidx_t, int64_t nnz, int64_t n,
                                            const int32_t* labels, const int32_t* counts, int32_t type, int64_t d, const void* dout,
                                            int64_t ldd, void* dx, int64_t lddx, void* workspace, size_t workspace_bytes, void* stream)
{
    return nm_run(rowptr_t, rowptr_bits, colidx_t, nnz, n, labels, type, d, dout, ldd, counts, true, dx, lddx, nullptr, workspace,
                  workspace_bytes, (hipStream_t)stream);
}
