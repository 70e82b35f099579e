// The mean of the neighbours' rows over a CSR graph, inside the partitions of a labelling, and its gradient, for gfx950.
//   N(v) = entries u of row v with labels[u] = labels[v] >= 0 (without labels: all entries), as stored, loops and duplicates included
//   out[v] = sum of x[u] over N(v) / |N(v)|, zero where N(v) is empty
//   dx[u]  = sum over the v that have u in N(v) of dout[v] / |N(v)|: the same walk over the transposed graph with a weight per entry
//
// The rows are gathered: an entry costs a row of d values from wherever it lies, and what bounds the kernels is how many such reads are
// under way and how many of them the caches serve.  A wave takes kNmRows vertices: it reads their entries' columns and labels, 256 at
// a time, and lists those that count in LDS (rows of other partitions are never touched).  Then L lanes read a neighbour's row, 16
// bytes each, and 64/L such groups take equal stretches of the list, whole rounds of reads under way at once, whichever vertices they
// belong to; a vertex whose entries lie in two groups' stretches is joined in LDS.  Sums are held in 32 bits.
// Where a labelling is given and x outgrows the L2s, vertices are taken in order of their partitions (k_nm_histogram, k_nm_scan, k_nm_order: one
// counting sort of the labels' low bits), an eighth of them on each chiplet: a partition's rows then meet in one L2.  The look-up of a
// neighbour's label is as much a read of a cache line as half its row is; from a copy in bytes (labels up to 254) it stays in
// the L2 too.
// Rows of more than `segment` entries are taken apart, summed by as many waves, and joined in order: no atomics on values, the
// same bytes on every run.
// 1M x 128 bfloat16, 33.5M entries, 24M of them counted: 997 us; the counted rows come from beyond the L2s at 6.9 TB/s, where a kernel that does
// nothing but read random rows reaches 7.5.
#include "grem_layers.hip.h"

namespace {

constexpr int kNmBlock = 256;
constexpr int kNmWaves = kNmBlock / 64;
constexpr int kNmRows = 8;                      // vertices a wave takes at a time
constexpr int kNmListed = 128;                  // entries of a row that goes on the list: the list holds kNmRows such rows
// entries that a long row is cut into, at least: as many as leave the few long rows of a small graph enough waves (500,000 entries x 128: 39 us,
// with 192 44), from 2^20 entries on more of them, for fewer partial sums (2M entries x 64: 73 us with 128, 60 with 192)
constexpr int64_t kNmSegmentFew = 128, kNmSegmentMany = 192, kNmManyEntries = 1 << 20;

struct NmItem {
    int32_t row, segment;
};
struct NmLong {
    int32_t row, first, count, unused;
};

// found: how many segments and long rows there are; then a histogram of the labels' low bits
constexpr int kNmBins = 256, kNmWide = 2 + kNmBins, kNmFound = kNmWide + 1;      // (kNmWide: a label beyond 254 was met)
constexpr int kNmOrderRows = 4096;              // vertices of a workgroup of the two kernels that order them

template <class T> constexpr int kNmV = 16 / (int)sizeof(T);

__device__ __forceinline__ int64_t nm_start(const void* __restrict__ rowptr, int bits, int64_t v)
{
    return bits == 64 ? ((const int64_t*)rowptr)[v] : (int64_t)((const int32_t*)rowptr)[v];
}

__device__ __forceinline__ float nm_size(int32_t count) { return (float)(count > 1 ? count : 1); }

// The sum of a row of the forward pass over its count, divided: a sum times the rounded 1/count is off by one rounding more, and falls beside
// the ties between 16-bit values (41 ones have 0.99999994 for their mean).
template <bool WEIGHTED> __device__ __forceinline__ float nm_mean(float sum, float size) { return WEIGHTED ? sum : sum / size; }

// An entry's weight in the backward pass, rounded once; its product with a value is not rounded (it is added in the same instruction), so a term
// is off by as much as the rounded quotient is.
__device__ __forceinline__ float nm_weight(const int32_t* __restrict__ counts, int32_t u) { return 1.0f / nm_size(counts[u]); }

// Adds up the counted entries of [lo, hi) for columns [c0, c0 + L*V*C); every lane ends with the sums of its columns over its own
// neighbours.  Returns how many entries counted.
template <class T, bool EVEN, bool WEIGHTED, int L, int C>
__device__ __forceinline__ int nm_walk(const int32_t* __restrict__ colidx, int64_t lo, int64_t hi, const int32_t* __restrict__ labels, int32_t mine,
                                       const int32_t* __restrict__ counts, const T* __restrict__ x, int64_t ldx, int c0, int d,
                                       float (&acc)[C][kNmV<T>])
{
    constexpr int V = kNmV<T>, G = 64 / L, U = C > 1 ? 4 : 8;
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
                w = nm_weight(counts, u);
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

// (LDS of one wave: its lanes are in step, only the compiler has to keep the order)
__device__ __forceinline__ void nm_wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <class T, bool EVEN, bool WEIGHTED, int L, int C>
__global__ __launch_bounds__(kNmBlock) void k_nm_rows(const void* __restrict__ rowptr, int bits, const int32_t* __restrict__ colidx, int64_t n,
                                                      const int32_t* __restrict__ labels, const int32_t* __restrict__ counts,
                                                      const T* __restrict__ x, int64_t ldx, int d, T* __restrict__ out, int64_t ldo,
                                                      int32_t* __restrict__ counts_out, int64_t segment, uint32_t* __restrict__ found,
                                                      NmItem* __restrict__ items, NmLong* __restrict__ longs,
                                                      const int32_t* __restrict__ order, const uint8_t* __restrict__ bytes, int take)
{
    constexpr int V = kNmV<T>, G = 64 / L, U = C > 1 ? 4 : 8, R = kNmRows, N = R * kNmListed;
    __shared__ int32_t list_of[kNmWaves][N];
    __shared__ float weight_of[WEIGHTED ? kNmWaves : 1][WEIGHTED ? N : 1];
    __shared__ int32_t off_of[kNmWaves][R + 1], vertex_of[kNmWaves][R];
    __shared__ float sizes_of[kNmWaves][R];
    __shared__ float open_of[G > 1 ? kNmWaves : 1][2][G][G > 1 ? L * V * C : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane / L, mine_c = (lane % L) * V;
    int32_t *list = list_of[wave], *off = off_of[wave], *vertices = vertex_of[wave];
    float* sizes = sizes_of[wave];
    float* weights = weight_of[WEIGHTED ? wave : 0];
    auto& open = open_of[G > 1 ? wave : 0];
    const bool narrow = bytes && found[kNmWide] == 0u;
    const uint32_t pitch = (uint32_t)ldx;
    // the vertices' order cut in eight, one for the workgroups of each chiplet (they go to the chiplets in turn)
    const int64_t share = order ? (n + 7) / 8 : n, base_at = order ? (int64_t)(blockIdx.x & 7u) * share : 0;
    const int64_t end_at = base_at + share < n ? base_at + share : n;
    const int64_t block = order ? blockIdx.x >> 3 : blockIdx.x, blocks = order ? gridDim.x >> 3 : gridDim.x;
    for (int64_t p0 = base_at + (block * kNmWaves + wave) * take; p0 < end_at; p0 += blocks * kNmWaves * take) {
        // lane r: row r's vertex, entries, label and what becomes of it
        const int rows = end_at - p0 < take ? (int)(end_at - p0) : take;
        const bool is_row = lane < rows;
        int32_t v = 0, label = 0;
        int64_t start = 0, degree = 0;
        if (is_row) {
            v = order ? order[p0 + lane] : (int32_t)(p0 + lane);
            start = nm_start(rowptr, bits, v);
            degree = nm_start(rowptr, bits, (int64_t)v + 1) - start;
            if (labels) label = labels[v];
        }
        const bool counted = is_row && label >= 0;
        const bool cut = counted && degree > segment, walked = counted && !cut && degree > kNmListed;
        if (cut) {
            const int32_t count = (int32_t)((degree + segment - 1) / segment);
            const int32_t first = (int32_t)atomicAdd(&found[0], (uint32_t)count);
            longs[atomicAdd(&found[1], 1u)] = NmLong{v, first, count, 0};
            for (int32_t i = 0; i < count; ++i) items[first + i] = NmItem{v, i};
        }

        // the entries of the rows that go on the list, one row after the other: place q is entry q + from of its row
        const int32_t length = counted && degree <= kNmListed ? (int32_t)degree : 0;
        int32_t ends = length;
#pragma unroll
        for (int o = 1; o < R; o <<= 1) {
            const int32_t y = __shfl_up(ends, o);
            if (lane >= o) ends += y;
        }
        const int32_t begins = ends - length, places = __shfl(ends, R - 1);
        const int64_t from = start - begins;
        int32_t bound[R];
#pragma unroll
        for (int k = 1; k < R; ++k) bound[k] = __shfl(begins, k);
        // the list, in that order; lane r counts what lies before its row
        int32_t kept = 0, before = 0;
        for (int32_t base = 0; base < places; base += 256) {
            int row[4];
            int32_t u[4], l[4];
            bool on[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int32_t at = base + q * 64 + lane;
                int r = 0;
#pragma unroll
                for (int k = 1; k < R; ++k) r += at >= bound[k];
                row[q] = r;
                on[q] = at < places;
                const int64_t shift = __shfl(from, r);
                u[q] = on[q] ? colidx[shift + at] : 0;
            }
            if (labels) {
#pragma unroll
                for (int q = 0; q < 4; ++q) l[q] = !on[q] ? -1 : narrow ? (int32_t)bytes[u[q]] : labels[u[q]];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int32_t own = __shfl(label, row[q]);
                    on[q] = on[q] && l[q] == own;
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const unsigned long long mask = __ballot(on[q]);
                const int to = kept + __popcll(mask & ((1ull << lane) - 1ull));
                if (on[q]) {
                    list[to] = u[q];
                    if constexpr (WEIGHTED) weights[to] = nm_weight(counts, u[q]);
                }
                const int32_t ahead = begins - (base + q * 64);
                before += __popcll(mask & (ahead >= 64 ? ~0ull : ahead <= 0 ? 0ull : (1ull << ahead) - 1ull));
                kept += __popcll(mask);
            }
        }
        if (lane <= R) off[lane] = lane < rows ? before : kept;
        if (lane < R) vertices[lane] = v;
        nm_wave_sync();
        if (is_row) {
            const int32_t here = off[lane + 1] - off[lane];
            sizes[lane] = nm_size(here);
            if (counts_out && !cut && !walked) counts_out[v] = here;
        }
        nm_wave_sync();

        for (int c0 = 0; c0 < d; c0 += L * V * C) {
            const int c = c0 + mine_c;
            auto store = [&](int32_t to, float (&acc)[C][V], float size) {
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    if (c + k * L * V >= d) continue;
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[k][i] = nm_mean<WEIGHTED>(acc[k][i], size);
                    store_floats<T, V, EVEN>(out + to * ldo, c + k * L * V, d, acc[k]);
                }
            };
            const int stretch = (kept + G - 1) / G;
            const int j0 = part * stretch < kept ? part * stretch : kept, j1 = j0 + stretch < kept ? j0 + stretch : kept;
            int r = 0;
            while (r < R && off[r + 1] <= j0) ++r;
            float acc[C][V];
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[k][i] = 0.0f;
            int end = r < R ? (off[r + 1] < j1 ? off[r + 1] : j1) : j1;
            for (int j = j0; j < j1; j += U) {
                WordsOf<T, V> f[U][C];
                float g[U];
#pragma unroll
                for (int q = 0; q < U; ++q) {
                    // (what is read for a place beyond j1 is added to sums that have been stored)
                    const int at = j + q < j1 ? j + q : j1 - 1;
                    const T* from = x + (uint64_t)(uint32_t)list[at] * pitch;
                    g[q] = WEIGHTED ? weights[at] : 1.0f;
#pragma unroll
                    for (int k = 0; k < C; ++k) {
                        const int at_c = c + k * L * V;
                        if constexpr (EVEN) f[q][k] = whole_words<T, V>(from + (at_c < d ? at_c : 0));
                        else f[q][k] = load_words<T, V, false>(from, at_c, d);
                    }
                }
#pragma unroll
                for (int q = 0; q < U; ++q) {
#pragma unroll
                    for (int k = 0; k < C; ++k) {
                        float v[V];
                        to_floats<T, V>(f[q][k], v);
#pragma unroll
                        for (int i = 0; i < V; ++i) acc[k][i] += WEIGHTED ? v[i] * g[q] : v[i];
                    }
                    if (j + q + 1 == end) {
                        // the row's last entry in this stretch
                        if (G == 1 || (off[r] >= j0 && off[r + 1] <= j1)) {
                            store(vertices[r], acc, sizes[r]);
                        } else {
                            float* to = open[off[r] >= j0 ? 1 : 0][part];
#pragma unroll
                            for (int k = 0; k < C; ++k)
#pragma unroll
                                for (int i = 0; i < V; ++i) to[k * L * V + mine_c + i] = acc[k][i];
                        }
#pragma unroll
                        for (int k = 0; k < C; ++k)
#pragma unroll
                            for (int i = 0; i < V; ++i) acc[k][i] = 0.0f;
                        while (r < R && off[r + 1] <= end) ++r;
                        end = r < R && off[r + 1] < j1 ? off[r + 1] : j1;
                    }
                }
            }
            if constexpr (G > 1) {
                nm_wave_sync();
                // a row that starts in this group's stretch and goes on in the next ones
                if (j0 < j1 && r < R && off[r] >= j0 && off[r] < j1 && off[r + 1] > j1) {
#pragma unroll
                    for (int k = 0; k < C; ++k)
#pragma unroll
                        for (int i = 0; i < V; ++i) acc[k][i] = open[1][part][k * L * V + mine_c + i];
                    for (int h = part + 1; h < G && h * stretch < off[r + 1]; ++h)
#pragma unroll
                        for (int k = 0; k < C; ++k)
#pragma unroll
                            for (int i = 0; i < V; ++i) acc[k][i] += open[0][h][k * L * V + mine_c + i];
                    store(vertices[r], acc, sizes[r]);
                }
                nm_wave_sync();
            }
            // rows without a counted entry
            const unsigned long long bare = __ballot(is_row && !cut && !walked && off[lane + 1] == off[lane]);
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[k][i] = 0.0f;
            for (int q = part; q < rows; q += G)
                if (bare >> q & 1) store(vertices[q], acc, 1.0f);
            // rows too long for the list, one after the other
            for (unsigned long long left = __ballot(walked); left; left &= left - 1) {
                const int q = __ffsll((long long)left) - 1;
                const int64_t first = __shfl(start, q), last = first + __shfl(degree, q);
#pragma unroll
                for (int k = 0; k < C; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[k][i] = 0.0f;
                const int total = nm_walk<T, EVEN, WEIGHTED, L, C>(colidx, first, last, labels, __shfl(label, q), counts, x, ldx, c0, d, acc);
                if (c0 == 0 && lane == 0 && counts_out) counts_out[vertices[q]] = total;
                if (part == 0) store(vertices[q], acc, nm_size(total));
            }
        }
        nm_wave_sync();
    }
}

__global__ void k_nm_clear(uint32_t* __restrict__ found)
{
    if (threadIdx.x < 2) found[threadIdx.x] = 0u;
}

// how many of a workgroup's vertices fall into each bin, bin by bin (hist: kNmBins rows of `blocks`; one more row says which workgroups
// met a label beyond 254), and the labels in bytes
__global__ __launch_bounds__(kNmBlock) void k_nm_histogram(const int32_t* __restrict__ labels, int64_t n, int blocks, uint32_t* __restrict__ hist,
                                                           uint8_t* __restrict__ bytes)
{
    __shared__ uint32_t bins[kNmBins];
    bins[threadIdx.x] = 0u;
    __syncthreads();
    const int64_t lo = (int64_t)blockIdx.x * kNmOrderRows, hi = lo + kNmOrderRows < n ? lo + kNmOrderRows : n;
    int wide = 0;
    for (int64_t v = lo + threadIdx.x; v < hi; v += kNmBlock) {
        const int32_t l = labels[v];
        atomicAdd(&bins[l & (kNmBins - 1)], 1u);
        bytes[v] = (uint8_t)(l < 0 ? 255 : l);
        wide |= l > 254;
    }
    wide = __syncthreads_or(wide);
    hist[(size_t)threadIdx.x * (size_t)blocks + blockIdx.x] = bins[threadIdx.x];
    if (threadIdx.x == 0) hist[(size_t)kNmBins * (size_t)blocks + blockIdx.x] = wide ? 1u : 0u;
}

// a workgroup a bin: its counts become the sums of those before; the totals and the flag go to found
__global__ __launch_bounds__(kNmBlock) void k_nm_scan(uint32_t* __restrict__ hist, int blocks, uint32_t* __restrict__ found)
{
    __shared__ uint32_t sums[2][kNmWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bin = blockIdx.x;
    uint32_t* row = hist + (size_t)bin * (size_t)blocks;
    uint32_t before = 0u;
    for (int base = 0, turn = 0; base < blocks; base += kNmBlock, turn ^= 1) {
        const int at = base + (int)threadIdx.x;
        const uint32_t mine = at < blocks ? row[at] : 0u;
        uint32_t upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t y = __shfl_up(upto, o);
            if (lane >= o) upto += y;
        }
        if (lane == 63) sums[turn][wave] = upto;
        __syncthreads();
        uint32_t all = 0u;
#pragma unroll
        for (int q = 0; q < kNmWaves; ++q) {
            if (q < wave) upto += sums[turn][q];
            all += sums[turn][q];
        }
        if (at < blocks) row[at] = before + upto - mine;
        before += all;
    }
    if (threadIdx.x == 0) found[bin < kNmBins ? 2 + bin : kNmWide] = before;
    if (bin == 0 && threadIdx.x < 2) found[threadIdx.x] = 0u;
}

// order: the vertices by the low bits of their labels, inside a bin as they come.  Which vertices share a wave decides where a row's sum is
// cut in two, so the order must be the same on every run: ranks are counted by ballots, a wave a stretch of the workgroup's vertices.
__global__ __launch_bounds__(kNmBlock) void k_nm_order(const int32_t* __restrict__ labels, int64_t n, int blocks, const uint32_t* __restrict__ found,
                                                       const uint32_t* __restrict__ hist, int32_t* __restrict__ order)
{
    __shared__ uint32_t seen[kNmWaves][kNmBins], sums[kNmWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t all = found[2 + threadIdx.x];
    uint32_t first = all;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(first, o);
        if (lane >= o) first += y;
    }
    if (lane == 63) sums[wave] = first;
#pragma unroll
    for (int q = 0; q < kNmWaves; ++q) seen[q][threadIdx.x] = 0u;
    __syncthreads();
    first -= all;
    for (int q = 0; q < wave; ++q) first += sums[q];
    first += hist[(size_t)threadIdx.x * (size_t)blocks + blockIdx.x];
    constexpr int per = kNmOrderRows / kNmBlock;
    const int64_t lo = (int64_t)blockIdx.x * kNmOrderRows + wave * (per * 64) + lane;
    uint32_t bin[per], rank[per];
#pragma unroll
    for (int i = 0; i < per; ++i) bin[i] = lo + i * 64 < n ? (uint32_t)labels[lo + i * 64] & (kNmBins - 1) : 0u;
#pragma unroll
    for (int i = 0; i < per; ++i) {
        unsigned long long same = __ballot(lo + i * 64 < n);
#pragma unroll
        for (int bit = 1; bit < kNmBins; bit <<= 1) {
            const unsigned long long set = __ballot((bin[i] & bit) != 0u);
            same &= bin[i] & bit ? set : ~set;
        }
        const int below = __popcll(same & ((1ull << lane) - 1ull));
        const uint32_t had = seen[wave][bin[i]];
        rank[i] = had + below;
        nm_wave_sync();
        if (lo + i * 64 < n && below == 0) seen[wave][bin[i]] = had + __popcll(same);
        nm_wave_sync();
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kNmWaves; ++q) {
        const uint32_t here = seen[q][threadIdx.x];
        seen[q][threadIdx.x] = first;
        first += here;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < per; ++i)
        if (lo + i * 64 < n) order[seen[wave][bin[i]] + rank[i]] = (int32_t)(lo + i * 64);
}

// the listed segments, a wave each: sums into partial (a row of d floats an item), counts beside them.  Of rows so wide that there are few segments
// gridDim.y waves take a segment's columns in turn.
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
        for (int c0 = (int)blockIdx.y * (L * V * C); c0 < d; c0 += (int)gridDim.y * (L * V * C)) {
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

// A long row's segments added up, a row's columns dealt out over gridDim.y workgroups: up to 32 segments a thread a column, more of them S
// threads a column over every S-th segment, then those S in order.  (One workgroup a row: 25 us at 7.9M entries x 256, the longest row's.)
template <class T, bool WEIGHTED>
__global__ __launch_bounds__(kNmBlock) void k_nm_join(int d, const uint32_t* __restrict__ found, const NmLong* __restrict__ longs,
                                                      const float* __restrict__ partial, const int32_t* __restrict__ part_counts,
                                                      T* __restrict__ out, int64_t ldo, int32_t* __restrict__ counts_out)
{
    constexpr int S = 8, W = kNmBlock / S;
    __shared__ float sums[S][W];
    __shared__ int total_of;
    const int q = threadIdx.x / W, i = threadIdx.x % W;
    const uint32_t rows = found[1];
    for (uint32_t l = blockIdx.x; l < rows; l += gridDim.x) {
        const NmLong r = longs[l];
        if (threadIdx.x < 64) {
            int total = 0;
            for (int s = threadIdx.x; s < r.count; s += 64) total += part_counts[r.first + s];
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
            if (threadIdx.x == 0) {
                total_of = total;
                if (counts_out && blockIdx.y == 0) counts_out[r.row] = total;
            }
        }
        __syncthreads();
        const int total = total_of;
        const float size = nm_size(total);
        const float* rowp = partial + (size_t)r.first * (size_t)d;
        if (r.count <= 32) {
            for (int c = blockIdx.y * kNmBlock + threadIdx.x; c < d; c += gridDim.y * kNmBlock) {
                float a = 0.0f;
#pragma unroll 8
                for (int s = 0; s < r.count; ++s) a += rowp[(size_t)s * (size_t)d + c];
                out[(int64_t)r.row * ldo + c] = (T)nm_mean<WEIGHTED>(a, size);
            }
            __syncthreads();
            continue;
        }
        for (int c0 = blockIdx.y * W; c0 < d; c0 += gridDim.y * W) {
            float a = 0.0f;
            if (c0 + i < d)
#pragma unroll 8
                for (int s = q; s < r.count; s += S) a += rowp[(size_t)s * (size_t)d + c0 + i];
            sums[q][i] = a;
            __syncthreads();
            if (q == 0 && c0 + i < d) {
                float all = 0.0f;
#pragma unroll
                for (int s = 0; s < S; ++s) all += sums[s][i];
                out[(int64_t)r.row * ldo + c0 + i] = (T)nm_mean<WEIGHTED>(all, size);
            }
            __syncthreads();
        }
    }
}

constexpr int64_t kNmOrderedBytes = 32 << 20;

// what a call keeps in its workspace
struct NmSpace {
    int64_t segment, items;
    int blocks;                     // workgroups of the kernels that order the vertices
    bool ordered;
    size_t o_order, o_bytes, o_hist, o_items, o_longs, o_counts, o_partial, bytes;
};

// Vertices in order of their partitions: from kNmOrderedBytes of x on
NmSpace nm_space(int64_t n, int64_t nnz, int64_t d, int size, bool labelled)
{
    NmSpace s;
    // as many segments as leave their sums in half a gigabyte, and no more than 65,536 or so: longer ones rather than more (64 at a width of 2^20)
    int64_t most = ((int64_t)1 << 26) / d;
    if (most > 65536) most = 65536;
    s.segment = (nnz + most - 1) / most;
    const int64_t least = nnz < kNmManyEntries ? kNmSegmentFew : kNmSegmentMany;
    if (s.segment < least) s.segment = least;
    // a row of e > segment entries has fewer than 2e / segment segments
    s.items = nnz > s.segment ? 2 * (nnz / s.segment) + 1 : 0;
    s.ordered = labelled && n * d * size >= kNmOrderedBytes;
    s.blocks = (int)((n + kNmOrderRows - 1) / kNmOrderRows);
    size_t off = layer_align(kNmFound * 4);
    auto carve = [&](size_t bytes) { const size_t at = off; off += layer_align(bytes); return at; };
    s.o_order = carve(s.ordered ? (size_t)n * 4 : 0);
    s.o_bytes = carve(s.ordered ? (size_t)n : 0);
    s.o_hist = carve(s.ordered ? (size_t)(kNmBins + 1) * (size_t)s.blocks * 4 : 0);
    s.o_items = carve((size_t)s.items * sizeof(NmItem));
    s.o_longs = carve((size_t)s.items * sizeof(NmLong));
    s.o_counts = carve((size_t)s.items * 4);
    s.o_partial = carve((size_t)s.items * (size_t)d * 4);
    s.bytes = s.items || s.ordered ? off : 0;
    return s;
}

// Vertices a wave takes: kNmRows where that still leaves every CU its 16 waves, fewer on smaller graphs (10,000 x 100: rows 17.5 us with 2, 19.7
// with 8).
int nm_take(int64_t n)
{
    int take = kNmRows;
    while (take > 1 && n < (int64_t)take * 4096) take /= 2;
    return take;
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
        (nnz && !colidx) || !layer_rows_ok(x, ldx, n, d, size) || ldx > (int64_t)UINT32_MAX || !layer_rows_ok(out, ldo, n, d, size) || (weighted && n && !counts) ||
        !layer_aligned(rowptr, bits / 8) || !layer_aligned(colidx, 4) || !layer_aligned(labels, 4) || !layer_aligned(counts, 4) || !layer_aligned(counts_out, 4))
        return GREM_ERR_ARG;
    if (n == 0) return GREM_OK;
    const NmSpace s = nm_space(n, nnz, d, size, labels != nullptr);
    if (const int rc = layer_space(workspace, workspace_bytes, s.bytes)) return rc;
    uint8_t* ws = (uint8_t*)workspace;
    uint32_t* found = (uint32_t*)ws;
    NmItem* items = s.items ? (NmItem*)(ws + s.o_items) : nullptr;
    NmLong* longs = s.items ? (NmLong*)(ws + s.o_longs) : nullptr;
    int32_t* part_counts = s.items ? (int32_t*)(ws + s.o_counts) : nullptr;
    float* partial = s.items ? (float*)(ws + s.o_partial) : nullptr;
    const int take = nm_take(n);
    const int64_t groups = (n + kNmWaves * take - 1) / (kNmWaves * take);
    const unsigned grid = (unsigned)(((groups < (1 << 22) ? groups : 1 << 22) + 7) / 8 * 8);
    // (a wave's columns are 512 at least)
    const unsigned seg_cols = (unsigned)(d <= 16384 ? 1 : (d + 16383) / 16384);
    const unsigned seg_grid = (unsigned)(s.items / kNmWaves + 1 < 2048 ? s.items / kNmWaves + 1 : 2048);
    const unsigned join_grid = (unsigned)(s.items < 1024 ? s.items : 1024), join_cols = (unsigned)(d < 256 ? (d + 31) / 32 : 8);
    int32_t* order = nullptr;
    uint8_t* bytes = nullptr;
    if (s.ordered) {
        uint32_t* hist = (uint32_t*)(ws + s.o_hist);
        order = (int32_t*)(ws + s.o_order);
        bytes = ws + s.o_bytes;
        hipLaunchKernelGGL(k_nm_histogram, dim3((unsigned)s.blocks), dim3(kNmBlock), 0, stream, labels, n, s.blocks, hist, bytes);
        hipLaunchKernelGGL(k_nm_scan, dim3(kNmBins + 1), dim3(kNmBlock), 0, stream, hist, s.blocks, found);
        hipLaunchKernelGGL(k_nm_order, dim3((unsigned)s.blocks), dim3(kNmBlock), 0, stream, labels, n, s.blocks, found, hist, order);
    } else if (s.items) {
        hipLaunchKernelGGL(k_nm_clear, dim3(1), dim3(64), 0, stream, found);
    }
    layer_typed(type, [&](auto t) {
        using T = decltype(t);
        nm_shaped<T>(d, [&](auto shape) {
            constexpr int L = decltype(shape)::L, C = decltype(shape)::C;
            auto run = [&](auto even, auto w) {
                constexpr bool E = decltype(even)::value, W = decltype(w)::value;
                hipLaunchKernelGGL((k_nm_rows<T, E, W, L, C>), dim3(grid), dim3(kNmBlock), 0, stream, rowptr, bits, colidx, n, labels, counts,
                                   (const T*)x, ldx, (int)d, (T*)out, ldo, counts_out, s.segment, found, items, longs, order, bytes, take);
                if (!s.items) return;
                hipLaunchKernelGGL((k_nm_segments<T, E, W, L, C>), dim3(seg_grid, seg_cols), dim3(kNmBlock), 0, stream, rowptr, bits, colidx, labels,
                                   counts, (const T*)x, ldx, (int)d, s.segment, found, items, partial, part_counts);
                hipLaunchKernelGGL((k_nm_join<T, W>), dim3(join_grid, join_cols), dim3(kNmBlock), 0, stream, (int)d, found, longs, partial,
                                   part_counts, (T*)out, ldo, counts_out);
            };
            layer_either(d % kNmV<T> == 0, [&](auto even) { layer_either(weighted, [&](auto w) { run(even, w); }); });
        });
    });
    return layer_launched();
}

}  // namespace

extern "C" size_t grem_neighbour_mean_bytes(int32_t type, int64_t n, int64_t nnz, int64_t d, int32_t labelled)
{
    const int size = layer_size(type);
    return !size || n < 0 || n > kLayerMaxRows || nnz < 0 || d < 1 || d > kLayerMaxCols ? 0 : nm_space(n, nnz, d, size, labelled != 0).bytes;
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
