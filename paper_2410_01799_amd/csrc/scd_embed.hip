// Embedding rows and their gradient (scd_embed, scd_embed_grad).
//
// Lookup: out_i = scale * E[t_i]; a copy of rows, bound by memory.
//
// Gradient: dE_v = scale * sum over the i with t_i = v of dY_i.  The rows of dE are few tokens' sums, most of them empty,
// a few of them long (tokens of a text fall off as one over their rank; padding may be half of a batch).  So (but for a few
// tokens, embed_few) the tokens are
// sorted first (embed_sort), then every row sums its own list (embed_rows), and lists that are longer than kPiece are cut
// at multiples of kPiece of the sorted order, summed piece by piece and joined in that order (embed_join).  Every sum has
// one order, the tokens' own: no atomics on floats, the same bits from run to run.
#include "scd_lm_device.h"

namespace scd {
namespace lm {
namespace {

constexpr int kCopyThreads = 256, kCopyUnroll = 4;

// A workgroup copies kCopyThreads * kCopyUnroll chunks of VN elements one after the other; cpr chunks make a row.
template <typename T, int VN>
__global__ __launch_bounds__(kCopyThreads) void embed_kernel(const T* __restrict__ E, int64_t V, int64_t D, const void* __restrict__ tokens,
                                                             int index_bytes, int64_t N, uint32_t cpr, float scale, T* __restrict__ out)
{
    typedef T VT __attribute__((ext_vector_type(VN)));
    const int64_t base = (int64_t)blockIdx.x * (kCopyThreads * kCopyUnroll);
    const int64_t row0 = base / cpr;
    const uint32_t rem0 = (uint32_t)(base - row0 * cpr);
    VT x[kCopyUnroll];
    int64_t to[kCopyUnroll];
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
        const uint64_t at = (uint64_t)rem0 + u * kCopyThreads + threadIdx.x;
        const uint32_t dr = (uint32_t)(at >> 32 ? at / cpr : (uint32_t)at / cpr);
        const int64_t row = row0 + dr;
        const int64_t col = (int64_t)(at - (uint64_t)dr * cpr) * VN;
        to[u] = row < N ? row * D + col : -1;
        const int64_t t = row < N ? index_at(tokens, index_bytes, row) : -1;
        if ((uint64_t)t < (uint64_t)V)
            x[u] = *(const VT*)(E + t * D + col);
        else
            x[u] = (VT)(T)__builtin_nanf("");
    }
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
        if (to[u] < 0) continue;
        VT y;
#pragma unroll
        for (int e = 0; e < VN; ++e) y[e] = round_to<T>(scale * to_f32(x[u][e]));
        *(VT*)(out + to[u]) = y;
    }
}

// ------------------------------------------------------------------------------------------------ gradient

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kSortRows = 64;   // vocabulary rows of a sorting workgroup
constexpr int kSortBatch = 16;  // tokens that a lane loads together
constexpr int kPiece = 16;      // tokens of a piece; longer lists are cut

// What the sort leaves in the work space.
struct Sorted {
    int32_t* start;   // [V + 1]: sorted[start[v] .. start[v + 1]) are the positions of token v, ascending
    int32_t* order;   // [N]
    int32_t* first;   // [pieces in use]: the row whose list holds the piece's first place
};

// Every workgroup reads all tokens and places those of its own kSortRows rows; how many come before them it counts itself, so
// that no workgroup waits for another (the tokens come from L2: 16384 of them are 128 KiB).  A wave takes one stretch of the
// tokens, counts it first and places it then; equal tokens among 64 lanes find each other by ballots of their six bits.
__global__ __launch_bounds__(kSortThreads) void embed_sort(const void* __restrict__ tokens, int index_bytes, int64_t N, int64_t V, int64_t pad, Sorted out)
{
    __shared__ int32_t hist[kSortWaves][kSortRows];  // counts, then where the next token of the row goes
    __shared__ int32_t lower[kSortWaves], bounds[kSortRows + 1];
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const int64_t v0 = (int64_t)blockIdx.x * kSortRows;
    const int64_t per = cdiv(cdiv(N, kSortWaves), kWave) * kWave;
    const int64_t i0 = per * wv, i1 = i0 + per < N ? i0 + per : N;

    // Rows of the next kSortBatch * 64 tokens: 0 .. kSortRows - 1 here, below 0 before, above behind (or none).
    auto rows = [&](int64_t i, int (&l)[kSortBatch]) {
        int64_t t[kSortBatch];
#pragma unroll
        for (int b = 0; b < kSortBatch; ++b) {
            const int64_t at = i + b * kWave + lane;
            t[b] = at < i1 ? index_at(tokens, index_bytes, at) : -1;
        }
#pragma unroll
        for (int b = 0; b < kSortBatch; ++b)
            l[b] = t[b] == pad || (uint64_t)t[b] >= (uint64_t)V ? kSortRows : t[b] < v0 ? -1 : t[b] - v0 < kSortRows ? (int)(t[b] - v0) : kSortRows;
    };
    // (a wave places its own tokens with its own counters: lanes read what other lanes of the wave wrote, in the order of the
    // wave's LDS instructions)
    volatile int32_t* next = hist[wv];
    next[lane] = 0;
    int32_t below = 0;
    int l[kSortBatch];
    for (int64_t i = i0; i < i1; i += kSortBatch * kWave) {
        rows(i, l);
#pragma unroll
        for (int b = 0; b < kSortBatch; ++b) {
            if (l[b] < 0) ++below;
            else if (l[b] < kSortRows) atomicAdd(&hist[wv][l[b]], 1);
        }
    }
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) below += __shfl_xor(below, off, kWave);
    if (lane == 0) lower[wv] = below;
    __syncthreads();
    if (wv == 0) {
        int32_t base = 0, mine = 0;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            base += lower[w];
            mine += hist[w][lane];
        }
        int32_t before = mine;  // inclusive sum over the rows
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const int32_t o = __shfl_up(before, off, kWave);
            if (lane >= off) before += o;
        }
        int32_t at = base + before - mine;
        bounds[lane] = at;
        if (lane == kWave - 1) bounds[kSortRows] = at + mine;
        if (v0 + lane < V) out.start[v0 + lane] = at;
        if (v0 + lane == V - 1) out.start[V] = at + mine;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const int32_t c = hist[w][lane];
            hist[w][lane] = at;
            at += c;
        }
    }
    __syncthreads();
    for (int64_t i = i0; i < i1; i += kSortBatch * kWave) {
        if (per > kSortBatch * kWave) rows(i, l);  // (else they are still there)
#pragma unroll
        for (int b = 0; b < kSortBatch; ++b) {
            const bool in = l[b] >= 0 && l[b] < kSortRows;
            uint64_t same = __ballot(in);
            if (!same) continue;
#pragma unroll
            for (int q = 0; q < 6; ++q) {
                const uint64_t set = __ballot((l[b] >> q) & 1);
                same &= (l[b] >> q) & 1 ? set : ~set;
            }
            if (in) {
                const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
                const int32_t at = next[l[b]];
                out.order[at + rank] = (int32_t)(i + b * kWave + lane);
                if (rank == 0) next[l[b]] = at + __popcll(same);  // (behind the reads of all lanes)
            }
        }
    }
    // Pieces whose first place lies here.
    const int32_t from = bounds[0], to = bounds[kSortRows];
    for (int64_t k = cdiv(from, kPiece) + threadIdx.x; k * kPiece < to; k += kSortThreads) {  // (k * kPiece passes 32 bits behind the last)
        int lo = 0, hi = kSortRows;  // bounds[lo] <= place < bounds[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (bounds[mid] <= k * kPiece) lo = mid;
            else hi = mid;
        }
        out.first[k] = (int32_t)(v0 + lo);
    }
}

constexpr int kRowThreads = 256, kRowsPerThread = 4;

// How a workgroup covers rows of cpr chunks: 1 << tsh threads a row (at most all), slices of a row.
struct RowShape {
    int tsh;
    int64_t slices;
    uint32_t cpr;
};

template <typename T, int VN>
__device__ __forceinline__ void add_rows(const T* __restrict__ dY, int64_t D, int64_t col, const int32_t* __restrict__ sorted, int32_t b, int32_t e,
                                         float (&acc)[VN])
{
    typedef T VT __attribute__((ext_vector_type(VN)));
    constexpr int U = 4;  // (8: 139 us for 132 at 16384 tokens, 32000 x 4096 bf16: fewer waves)
    for (uint32_t j = b; j < (uint32_t)e; j += U) {  // (e is up to 2^31 - 1: j + u passes that)
        VT x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = j + u < (uint32_t)e ? *(const VT*)(dY + (int64_t)sorted[j + u] * D + col) : (VT)(T)0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < VN; ++q) acc[q] += to_f32(x[u][q]);
    }
}

// PAST: past the caches.
template <typename T, int VN, bool PAST = false>
__device__ __forceinline__ void put_row(T* __restrict__ dE, int64_t D, int64_t v, int64_t col, float scale, const float (&acc)[VN])
{
    typedef T VT __attribute__((ext_vector_type(VN)));
    VT y;
#pragma unroll
    for (int q = 0; q < VN; ++q) y[q] = round_to<T>(scale * acc[q]);
    if constexpr (PAST) __builtin_nontemporal_store(y, (VT*)(dE + v * D + col));
    else *(VT*)(dE + v * D + col) = y;
}

// The first piece_groups workgroups (the longest work first): one piece of the sorted order, of which the parts that belong to
// lists longer than a piece go to parts[piece][0] (the list that holds the piece's first place) and parts[piece][1] (one that
// begins behind it; it holds the next piece's first place too).  Those behind: rows with at most kPiece tokens, written whole.
template <typename T, int VN, bool PAST>
__global__ __launch_bounds__(kRowThreads) void embed_rows(const T* __restrict__ dY, int64_t V, int64_t D, const int32_t* __restrict__ start,
                                                          const int32_t* __restrict__ sorted, const int32_t* __restrict__ first, RowShape sh,
                                                          int64_t piece_groups, float scale, T* __restrict__ dE, float* __restrict__ parts)
{
    const int64_t wg = blockIdx.x / sh.slices, slice = blockIdx.x - wg * sh.slices;
    const int tpr = 1 << sh.tsh, rows = kRowThreads >> sh.tsh;
    const int64_t chunk = slice * tpr + (threadIdx.x & (tpr - 1));
    const int64_t col = chunk * VN;
    if (chunk >= sh.cpr) return;
    if (wg >= piece_groups) {
        const int64_t r0 = (wg - piece_groups) * rows * kRowsPerThread + (threadIdx.x >> sh.tsh);
        int32_t b[kRowsPerThread], e[kRowsPerThread];
#pragma unroll
        for (int r = 0; r < kRowsPerThread; ++r) {
            const int64_t v = r0 + r * rows < V ? r0 + r * rows : V - 1;
            b[r] = start[v];
            e[r] = start[v + 1];
        }
#pragma unroll
        for (int r = 0; r < kRowsPerThread; ++r) {
            if (r0 + r * rows >= V) return;
            if (e[r] - b[r] > kPiece) continue;
            float acc[VN] = {};
            add_rows<T, VN>(dY, D, col, sorted, b[r], e[r], acc);
            put_row<T, VN, PAST>(dE, D, r0 + r * rows, col, scale, acc);
        }
        return;
    }
    const int64_t piece = wg * rows + (threadIdx.x >> sh.tsh);
    const int32_t total = start[V];
    if (piece * kPiece >= total) return;
    const int32_t j0 = (int32_t)(piece * kPiece), j1 = total - j0 < kPiece ? total : j0 + kPiece;
    const int32_t v[2] = {first[piece], first[j1 < total ? piece + 1 : piece]};
    const int32_t b[2] = {start[v[0]], start[v[1]]}, e[2] = {start[v[0] + 1], start[v[1] + 1]};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        if (e[s] - b[s] <= kPiece || (s && (b[s] <= j0 || b[s] >= j1))) continue;
        float acc[VN] = {};
        add_rows<T, VN>(dY, D, col, sorted, b[s] > j0 ? b[s] : j0, e[s] < j1 ? e[s] : j1, acc);
        float* p = parts + (piece * 2 + s) * D + col;
#pragma unroll
        for (int q = 0; q < VN; ++q) p[q] = acc[q];
    }
}

constexpr int kFewTokens = kRowThreads;

// At most kFewTokens tokens: no sort, a workgroup picks those of its own rows out of all of them, in their order, and sums them.
template <typename T, int VN>
__global__ __launch_bounds__(kRowThreads) void embed_few(const void* __restrict__ tokens, int index_bytes, int N, const T* __restrict__ dY, int64_t V, int64_t D,
                                                         int64_t pad, RowShape sh, float scale, T* __restrict__ dE)
{
    __shared__ int32_t key[kFewTokens];                 // row here and position of a token, positions ascending
    __shared__ int32_t at[kFewTokens];                  // positions by row
    __shared__ int32_t start[kRowThreads * kRowsPerThread + 1];
    __shared__ int32_t counts[kRowThreads / kWave];
    const int64_t wg = blockIdx.x / sh.slices, slice = blockIdx.x - wg * sh.slices;
    const int tpr = 1 << sh.tsh, rows = kRowThreads >> sh.tsh, all = rows * kRowsPerThread;
    const int64_t v0 = wg * all;
    const int i = threadIdx.x, lane = i & (kWave - 1), wv = i / kWave;
    const int64_t t = i < N ? index_at(tokens, index_bytes, i) : -1;
    const bool in = (uint64_t)t < (uint64_t)V && t != pad && t >= v0 && t - v0 < all;
    const uint64_t mask = __ballot(in);
    if (lane == 0) counts[wv] = __popcll(mask);
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kRowThreads / kWave; ++w) {
        before += w < wv ? counts[w] : 0;
        total += counts[w];
    }
    if (in) {
        before += __popcll(mask & (((uint64_t)1 << lane) - 1));
        key[before] = (int32_t)(t - v0) * kFewTokens + i;
    }
    __syncthreads();
    // Keys are unique: a key's place is the number of smaller ones, a row's start that of keys below its first.
    if (i < total) {
        const int32_t mine = key[i];
        int place = 0;
        for (int j = 0; j < total; ++j) place += key[j] < mine;
        at[place] = mine % kFewTokens;
    }
    for (int r = i; r <= all; r += kRowThreads) {
        int place = 0;
        for (int j = 0; j < total; ++j) place += key[j] < r * kFewTokens;
        start[r] = place;
    }
    __syncthreads();
    const int64_t chunk = slice * tpr + (i & (tpr - 1)), col = chunk * VN;
    if (chunk >= sh.cpr) return;
#pragma unroll 1
    for (int r = i >> sh.tsh; r < all && v0 + r < V; r += rows) {
        float acc[VN] = {};
        add_rows<T, VN>(dY, D, col, at, start[r], start[r + 1], acc);
        put_row<T, VN>(dE, D, v0 + r, col, scale, acc);
    }
}

constexpr int kJoinWays = 16;  // stretches that a list's parts are summed in

constexpr int kJoinThreads = kJoinWays * kWave;

// Lists longer than a piece: each is found at the first piece that it holds the first place of.  Every workgroup looks through
// all pieces and takes every gridDim.x-th of the lists' slices (64 chunks of a row): the list's parts in their order, a stretch
// of them by each wave, then the stretches in theirs.
template <typename T, int VN>
__global__ __launch_bounds__(kJoinThreads) void embed_join(int64_t V, int64_t D, const int32_t* __restrict__ start, const int32_t* __restrict__ first,
                                                           int64_t slices, float scale, T* __restrict__ dE, const float* __restrict__ parts)
{
    __shared__ float ways[kJoinWays][kWave][VN];
    __shared__ int32_t rows[kJoinThreads], counts[kJoinWays];
    const int lane = threadIdx.x & (kWave - 1), way = threadIdx.x / kWave;
    const int32_t total = start[V];
    int64_t item = 0;  // of the lists' slices before these pieces
    for (int64_t p0 = 0; p0 * kPiece < total; p0 += kJoinThreads) {
        const int64_t p = p0 + threadIdx.x;
        const int32_t row = p * kPiece < total ? first[p] : -1;
        bool in = false;
        if (row >= 0) {
            const int32_t b = start[row], e = start[row + 1];
            in = e - b > kPiece && cdiv(b, kPiece) == p;
        }
        const uint64_t mask = __ballot(in);
        __syncthreads();
        if (lane == 0) counts[way] = __popcll(mask);
        __syncthreads();
        int32_t before = 0, lists = 0;
#pragma unroll
        for (int w = 0; w < kJoinWays; ++w) {
            before += w < way ? counts[w] : 0;
            lists += counts[w];
        }
        if (in) rows[before + __popcll(mask & (((uint64_t)1 << lane) - 1))] = row;
        __syncthreads();
        const int64_t items = lists * slices;
        int64_t i = ((int64_t)blockIdx.x - item) % gridDim.x;
        for (i = i < 0 ? i + gridDim.x : i; i < items; i += gridDim.x) {
            const int64_t l = i / slices, col = ((i - l * slices) * kWave + lane) * VN;
            const int32_t v = rows[l], b = start[v], e = start[v + 1];
            const int64_t piece = b / kPiece, end = (e - 1) / kPiece + 1, per = cdiv(end - piece, kJoinWays);
            const int64_t k0 = piece + way * per, k1 = k0 + per < end ? k0 + per : end;
            float acc[VN] = {};
            if (col < D) {
                constexpr int U = 4;
                for (int64_t k = k0; k < k1; k += U) {
                    float x[U][VN];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int64_t at = k + u < k1 ? k + u : k1 - 1;
                        const float* from = parts + (at * 2 + (at * kPiece < b ? 1 : 0)) * D + col;
#pragma unroll
                        for (int q = 0; q < VN; ++q) x[u][q] = from[q];
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int q = 0; q < VN; ++q) acc[q] += k + u < k1 ? x[u][q] : 0.0f;
                }
            }
#pragma unroll
            for (int q = 0; q < VN; ++q) ways[way][lane][q] = acc[q];
            __syncthreads();
            if (way == 0 && col < D) {
                for (int w = 1; w < kJoinWays; ++w)
#pragma unroll
                    for (int q = 0; q < VN; ++q) acc[q] += ways[w][lane][q];
                put_row<T, VN>(dE, D, v, col, scale, acc);
            }
            __syncthreads();
        }
        item += items;
    }
}

int64_t pieces_of(int64_t N) { return cdiv(N, kPiece); }

template <typename T, int VN>
hipError_t embed_t(const void* E, int64_t V, int64_t D, const void* tokens, int index_bytes, int64_t N, float scale, void* out, hipStream_t st)
{
    const int64_t cpr = D / VN, grid = cdiv(N * cpr, kCopyThreads * kCopyUnroll);
    if (!grid_ok(grid, kCopyThreads)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((embed_kernel<T, VN>), dim3((unsigned)grid), dim3(kCopyThreads), 0, st, (const T*)E, V, D, tokens, index_bytes, N, (uint32_t)cpr, scale,
                       (T*)out);
    return hipGetLastError();
}

// The work space: start, order, first, parts.
size_t grad_space(int64_t V, int64_t D, int64_t N, size_t at[4])
{
    at[0] = at[1] = at[2] = at[3] = 0;
    if (N <= kFewTokens) return 0;
    at[1] = up((size_t)(V + 1) * 4, 256);
    at[2] = at[1] + up((size_t)N * 4, 256);
    at[3] = at[2] + up((size_t)pieces_of(N) * 4, 256);
    return at[3] + (size_t)pieces_of(N) * 2 * (size_t)D * 4;
}

template <typename T, int VN>
hipError_t embed_grad_t(const void* tokens, int index_bytes, int64_t N, const void* dY, int64_t V, int64_t D, int64_t pad, float scale, void* dE,
                        char* ws, hipStream_t st)
{
    size_t at[4];
    (void)grad_space(V, D, N, at);
    const Sorted so{(int32_t*)(ws + at[0]), (int32_t*)(ws + at[1]), (int32_t*)(ws + at[2])};
    float* parts = (float*)(ws + at[3]);
    RowShape sh;
    sh.cpr = (uint32_t)(D / VN);
    sh.tsh = 0;
    while ((1 << sh.tsh) < kRowThreads && (1u << sh.tsh) < sh.cpr) ++sh.tsh;
    sh.slices = cdiv(sh.cpr, (int64_t)1 << sh.tsh);
    const int64_t rows = kRowThreads >> sh.tsh;
    const int64_t row_groups = cdiv(V, rows * kRowsPerThread), piece_groups = cdiv(pieces_of(N), rows);
    if (!grid_ok((row_groups + piece_groups) * sh.slices, kRowThreads) || !grid_ok(cdiv(V, kSortRows), kSortThreads)) return hipErrorInvalidConfiguration;
    if (N <= kFewTokens) {
        hipLaunchKernelGGL((embed_few<T, VN>), dim3((unsigned)(row_groups * sh.slices)), dim3(kRowThreads), 0, st, tokens, index_bytes, (int)N, (const T*)dY, V, D,
                           pad, sh, scale, (T*)dE);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(embed_sort, dim3((unsigned)cdiv(V, kSortRows)), dim3(kSortThreads), 0, st, tokens, index_bytes, N, V, pad, so);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // Rows of dE written past the caches leave these to dY, which frequent tokens' rows and their neighbours are read from (32000 x 4096
    // bf16, a call of 16384 tokens 127 -> 113 us, of 4096 90 -> 69, of 1000 79 -> 65).  With fewer tokens to a row writing is all there is to
    // do, and a dE that is written again and again is still in the last cache (300 tokens: 48 us through the caches, 61 past; of three dE in turn
    // 66 and 58).
    auto kernel = N >= V / 32 ? embed_rows<T, VN, true> : embed_rows<T, VN, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((row_groups + piece_groups) * sh.slices)), dim3(kRowThreads), 0, st, (const T*)dY, V, D, so.start, so.order,
                       so.first, sh, piece_groups, scale, (T*)dE, parts);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t slices = cdiv(D, kWave * VN), most = pieces_of(N) * slices;
    hipLaunchKernelGGL((embed_join<T, VN>), dim3((unsigned)(most < 512 ? most : 512)), dim3(kJoinThreads), 0, st, V, D, so.start, so.first, slices, scale,
                       (T*)dE, parts);
    return hipGetLastError();
}

}  // namespace
}  // namespace lm
}  // namespace scd

using namespace scd::lm;

extern "C" {

int scd_embed(const void* E, scd_real dt, int64_t V, int64_t D, const void* tokens, int index_bytes, int64_t N, float scale, void* out,
              void* stream)
{
    if (!E || !real_ok(dt) || !dim_ok(V) || !dim_ok(D) || !index_ok(index_bytes) || !rows_ok(N) || (N > 0 && (!tokens || !out))) return SCD_EINVAL;
    if (N == 0) return SCD_OK;
    hipStream_t st = (hipStream_t)stream;
    const bool vec = aligned16(E) && aligned16(out) && D * real_bytes(dt) % 16 == 0;
    const hipError_t e = with_real(dt, [&](auto z) {
        typedef decltype(z) T;
        return vec ? embed_t<T, Vec<T>::N>(E, V, D, tokens, index_bytes, N, scale, out, st) : embed_t<T, 1>(E, V, D, tokens, index_bytes, N, scale, out, st);
    });
    return e == hipSuccess ? SCD_OK : scd::report_hip(e);
}

size_t scd_embed_grad_workspace_bytes(int64_t V, int64_t D, int64_t N)
{
    if (!dim_ok(V) || !dim_ok(D) || !rows_ok(N)) return 0;
    size_t at[4];
    return grad_space(V, D, N, at);
}

int scd_embed_grad(const void* tokens, int index_bytes, int64_t N, const void* dY, scd_real dt, int64_t V, int64_t D, int64_t pad, float scale,
                   void* dE, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!dE || !real_ok(dt) || !dim_ok(V) || !dim_ok(D) || !index_ok(index_bytes) || !rows_ok(N) || (N > 0 && (!tokens || !dY))) return SCD_EINVAL;
    const size_t need = scd_embed_grad_workspace_bytes(V, D, N);
    if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return SCD_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    const bool vec = aligned16(dY) && aligned16(dE) && D * real_bytes(dt) % 16 == 0;
    const hipError_t e = with_real(dt, [&](auto z) {
        typedef decltype(z) T;
        char* ws = (char*)workspace;
        return vec ? embed_grad_t<T, Vec<T>::N>(tokens, index_bytes, N, dY, V, D, pad, scale, dE, ws, st)
                   : embed_grad_t<T, 1>(tokens, index_bytes, N, dY, V, D, pad, scale, dE, ws, st);
    });
    return e == hipSuccess ? SCD_OK : scd::report_hip(e);
}

}  // extern "C"
