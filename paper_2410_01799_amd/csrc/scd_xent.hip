// Cross entropy of the output head and its gradients (scd_xent, scd_xent_grad).
//
//   z = scale X W^T,  lse_i = log sum_v exp z_iv,  loss_i = lse_i - z_{i,t_i}
//   dz_iv = g_i (exp(z_iv - lse_i) - [v = t_i]),  dX = scale dz W,  dW = scale dz^T X
//
// Logits live in the accumulators of a tile of the product only.  Forward: every tile leaves, for each of its tokens, the
// maximum of its logits and the sum of their exponentials below it; a second kernel joins these along the vocabulary.
// Gradient: tokens that count are listed first (xent_list), so that the others cost nothing and nothing in them spreads;
// then, for one piece of the vocabulary after the other, the logits are formed again, dz of the piece goes to the work
// space, and two products take it from there.
//
// Two forms.  The tile of scd_lm_tile.h takes 16-bit types, dz held in the type, and f32, dz in f32, on the bf16 instruction (sums of a
// few terms on the f32 instruction).  Rows that are no multiple of 16 bytes are copied to the work space first, W a piece at a time.
// tile32 below, the f32 matrix instruction from operands of any type, alignment and order with dz in f32, takes weights (in the forward:
// and hidden states) that begin at odd addresses.
#include "scd_lm_tile.h"

namespace scd {
namespace lm {
namespace {

// How many tokens count, and what lies between dz and what is held of it: dz is held relative to the largest |g| (ref), times
// 2^kLift, so that neither a small g nor a small probability meets the smallest numbers of the type, and so that with one g for
// all tokens, as in a mean, the -1 of a target is a power of two and p - 1 keeps the digits that it has there.  inv undoes both.
struct Active {
    int32_t count;
    float ref, inv;
};

template <typename T>
constexpr int kLift = 24;
template <>
constexpr int kLift<_Float16> = 15;  // f16 ends at 65504; |dz| is at most 2^15

// 2^LIFT exp(x) for x <= 0 and a little above.
template <int LIFT>
__device__ __forceinline__ float lifted_exp(float x)
{
    const float lift = (float)(1 << LIFT);
    return x > -60.0f ? expf(x) * lift : expf(x + 0.693147180559945f * LIFT);  // (there, exp(x) itself would run out of digits)
}

// ------------------------------------------------------------------------------------------------ tiles in f32

constexpr int kT = 128, kTThreads = 256, kTK = 16, kTPitch = kT + 4;

// An operand of a tile: `across` runs over the tile's 128 rows or columns, `along` over the products' terms.  along_inner:
// entries that follow one another in memory lie along the terms, else across.  idx: the rows of the array are taken from
// this list (rows are the outer index).
template <typename T>
struct Operand {
    const T* p;
    int64_t ld;
    const int32_t* idx;
    int64_t outer;  // rows of the array (of the list)
    int64_t inner;  // entries of a row
};

struct TileLds {
    float a[kTK][kTPitch], b[kTK][kTPitch];
};

// Eight entries of an operand for this thread: inner entries i0 .. i0 + 7 of row o; zero beyond the array.
template <typename T>
__device__ __forceinline__ void fetch8(const Operand<T>& op, int64_t o, int64_t i0, bool vec, float (&x)[8])
{
    typedef T V8 __attribute__((ext_vector_type(16 / sizeof(T))));
    constexpr int VN = 16 / sizeof(T);
    const bool live = o < op.outer;
    const int64_t row = live ? (op.idx ? (int64_t)op.idx[o] : o) : 0;
    const T* p = op.p + row * op.ld;
    if (vec && live && i0 + 8 <= op.inner) {
#pragma unroll
        for (int h = 0; h < 8 / VN; ++h) {
            const V8 v = *(const V8*)(p + i0 + h * VN);
#pragma unroll
            for (int e = 0; e < VN; ++e) x[h * VN + e] = to_f32(v[e]);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = live && i0 + e < op.inner ? to_f32(p[i0 + e]) : 0.0f;
}

template <typename T>
__device__ __forceinline__ bool vectors(const Operand<T>& op)
{
    return ((uintptr_t)op.p & 15u) == 0 && (op.ld * sizeof(T)) % 16 == 0;
}

// acc[a][b] (+)= sum over the terms of A's 16-blocks times B's: wave (wr, wc) of 2 x 2 holds 64 x 64 of the tile.  Lane:
// columns (B) lane mod 16, rows (A) 4 (lane / 16) + register.
template <bool A_IN, bool B_IN, typename TA, typename TB>
__device__ __forceinline__ void tile32(const Operand<TA>& A, const Operand<TB>& B, int64_t a0, int64_t b0, int64_t terms, TileLds& sh, v4f (&acc)[4][4])
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    const int li = lane & 15, kq = lane >> 4, wr = (wv >> 1) * 64, wc = (wv & 1) * 64;
    const bool va = vectors(A), vb = vectors(B);
    // inner along: two threads a row, eight terms each; inner across: sixteen threads a term, eight columns each
    const int ao = A_IN ? tid >> 1 : tid >> 4, ai = A_IN ? (tid & 1) * 8 : (tid & 15) * 8;
    const int bo = B_IN ? tid >> 1 : tid >> 4, bi = B_IN ? (tid & 1) * 8 : (tid & 15) * 8;
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[a][b] = (v4f)0.0f;
    float xa[8], xb[8];
    auto fetch = [&](int64_t k0) {
        if constexpr (A_IN) fetch8(A, a0 + ao, k0 + ai, va, xa);
        else fetch8(A, k0 + ao, a0 + ai, va, xa);
        if constexpr (B_IN) fetch8(B, b0 + bo, k0 + bi, vb, xb);
        else fetch8(B, k0 + bo, b0 + bi, vb, xb);
    };
    if (terms > 0) fetch(0);
    for (int64_t k0 = 0; k0 < terms; k0 += kTK) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (A_IN) sh.a[ai + e][ao] = xa[e];
            else sh.a[ao][ai + e] = xa[e];
            if constexpr (B_IN) sh.b[bi + e][bo] = xb[e];
            else sh.b[bo][bi + e] = xb[e];
        }
        __syncthreads();
        if (k0 + kTK < terms) fetch(k0 + kTK);
#pragma unroll
        for (int s = 0; s < kTK; s += 4) {
            float fa[4], fb[4];
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                fa[a] = sh.a[s + kq][wr + a * 16 + li];
                fb[a] = sh.b[s + kq][wc + a * 16 + li];
            }
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 4; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[a], fb[b], acc[a][b], 0, 0, 0);
        }
    }
}

// ------------------------------------------------------------------------------------------------ forward

constexpr int kStrip = kT;  // vocabulary rows behind one pair of sums of a token, in tile32

struct Sums {
    float max, sum;  // of the logits, and of exp(logit - max)
};

// Vocabulary x tokens; strips[strip][token].
template <typename T>
__global__ __launch_bounds__(kTThreads) void xent_forward32(Operand<T> W, Operand<T> X, const void* __restrict__ targets, int index_bytes, float scale,
                                                            Sums* __restrict__ strips, float* __restrict__ zt)
{
    __shared__ TileLds sh;
    __shared__ Sums lower[kT];  // of the tile's lower half
    const int64_t v0 = (int64_t)blockIdx.x * kT, n0 = (int64_t)blockIdx.y * kT;
    v4f acc[4][4];
    tile32<true, true>(W, X, v0, n0, W.inner, sh, acc);
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const int li = lane & 15, kq = lane >> 4, wr = (wv >> 1) * 64, wc = (wv & 1) * 64;
    Sums half[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const int64_t n = n0 + wc + b * 16 + li;
        const bool live = n < X.outer;
        const int64_t t = live ? index_at(targets, index_bytes, n) : -1;
        float top = -__builtin_inff();
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t v = v0 + wr + a * 16 + kq * 4 + r;
                acc[a][b][r] = v < W.outer ? acc[a][b][r] * scale : -__builtin_inff();
                if (live && v == t && v < W.outer) zt[n] = acc[a][b][r];
                top = fmaxf(top, acc[a][b][r]);
            }
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        float sum = 0.0f;
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float z = acc[a][b][r];
                sum += z == -__builtin_inff() ? 0.0f : expf(z - top);  // (a strip may hold nothing else)
            }
        sum += __shfl_xor(sum, 16, kWave);
        sum += __shfl_xor(sum, 32, kWave);
        half[b].max = top;
        half[b].sum = sum;
        if (wr && kq == 0) lower[wc + b * 16 + li] = half[b];
    }
    __syncthreads();
    if (wr || kq) return;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const int64_t n = n0 + wc + b * 16 + li;
        if (n >= X.outer) continue;
        const Sums x = half[b], y = lower[wc + b * 16 + li];
        Sums s;
        s.max = fmaxf(x.max, y.max);
        const float base = s.max == -__builtin_inff() ? 0.0f : s.max;
        s.sum = x.sum * expf(x.max - base) + y.sum * expf(y.max - base);
        strips[v0 / kStrip * X.outer + n] = s;
    }
}

// A token's loss and lse from its largest logit, the sum of exponentials below it and its target's logit.
__device__ __forceinline__ void write_loss(int64_t n, float top, double sum, float zt, int64_t target, int64_t V, int64_t ignore, float* __restrict__ loss,
                                           float* __restrict__ lse)
{
    const double l = log(sum);
    lse[n] = (float)((double)top + l);
    // (not lse - zt: lse rounded to f32 has a step of 2^-19 from 16 on, and the loss of a likely target is far below that)
    loss[n] = target == ignore ? 0.0f : (uint64_t)target < (uint64_t)V ? (float)((double)top - (double)zt + l) : __builtin_nanf("");
}

// TOKENS tokens a workgroup, the threads of a token each take every so many strips: first the largest logit, then the sum in
// f64.  (Sixteen tokens make whole lines of the strips; one token takes the whole workgroup where there are few.)
constexpr int kJoinThreads = 1024;
template <int TOKENS>
__global__ __launch_bounds__(kJoinThreads) void xent_join(const Sums* __restrict__ strips, int64_t nstrips, int64_t N, int64_t V,
                                                          const void* __restrict__ targets, int index_bytes, int64_t ignore,
                                                          const float* __restrict__ zt, float* __restrict__ loss, float* __restrict__ lse)
{
    constexpr int kWays = kJoinThreads / TOKENS, kWaves = kJoinThreads / kWave;
    __shared__ float tops[kWaves][TOKENS];
    __shared__ double sums[kWaves][TOKENS];
    const int t = threadIdx.x % TOKENS, way = threadIdx.x / TOKENS, wv = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
    const int64_t n = (int64_t)blockIdx.x * TOKENS + t, at_n = n < N ? n : N - 1;
    float top = -__builtin_inff();
#pragma unroll 4
    for (int64_t s = way; s < nstrips; s += kWays) top = fmaxf(top, strips[s * N + at_n].max);
#pragma unroll
    for (int off = TOKENS; off < kWave; off <<= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
    if (lane < TOKENS) tops[wv][t] = top;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, tops[w][t]);
    const float base = top == -__builtin_inff() ? 0.0f : top;
    double sum = 0.0;
#pragma unroll 4
    for (int64_t s = way; s < nstrips; s += kWays) {
        const Sums x = strips[s * N + at_n];
        sum += (double)(x.sum * expf(x.max - base));
    }
#pragma unroll
    for (int off = TOKENS; off < kWave; off <<= 1) sum += __shfl_xor(sum, off, kWave);
    if (lane < TOKENS) sums[wv][t] = sum;
    __syncthreads();
    if (way || n >= N) return;
    sum = 0.0;
    for (int w = 0; w < kWaves; ++w) sum += sums[w][t];
    write_loss(n, top, sum, zt[n], index_at(targets, index_bytes, n), V, ignore, loss, lse);
}

// ------------------------------------------------------------------------------------------------ gradient

constexpr int kListThreads = 1024;

__device__ __forceinline__ bool counts_for(int64_t t, int64_t V, int64_t ignore, float g) { return t != ignore && (uint64_t)t < (uint64_t)V && g != 0.0f; }

// The bits of |g| for the largest of them; a g that is not finite shows in its own token's terms and says nothing of the others.
__device__ __forceinline__ uint32_t weight_of(float g)
{
    const uint32_t m = __float_as_uint(g) & 0x7FFFFFFFu;
    return m < 0x7F800000u ? m : 0u;
}

// From the number of tokens that count and the bits of their largest |g|.
__device__ __forceinline__ Active active_of(int32_t count, uint32_t top, int lift)
{
    Active a;
    a.count = count;
    a.ref = top == 0 ? 1.0f : fmaxf(__uint_as_float(top), 0x1p-100f);  // (no finite g at all: as they are)
    a.inv = ldexpf(a.ref, -lift);
    return a;
}

// One workgroup: the tokens that count, in ascending order, then the others in descending order.
__global__ __launch_bounds__(kListThreads) void xent_list(const void* __restrict__ targets, int index_bytes, int64_t N, int64_t V, int64_t ignore,
                                                          const float* __restrict__ g, int lift, int32_t* __restrict__ list, Active* __restrict__ active)
{
    __shared__ int32_t counts[kListThreads / kWave];
    __shared__ uint32_t tops[kListThreads / kWave];
    uint32_t top = 0;
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    int64_t base = 0;
    for (int64_t i0 = 0; i0 < N; i0 += kListThreads) {
        const int64_t i = i0 + threadIdx.x;
        bool in = false;
        if (i < N) {
            const int64_t t = index_at(targets, index_bytes, i);
            const float gi = g[i];
            in = counts_for(t, V, ignore, gi);
            const uint32_t m = in ? weight_of(gi) : 0u;
            top = m > top ? m : top;
        }
        const uint64_t mask = __ballot(in);
        __syncthreads();
        if (lane == 0) counts[wv] = __popcll(mask);
        __syncthreads();
        int32_t before = 0, all = 0;
        for (int w = 0; w < kListThreads / kWave; ++w) {
            before += w < wv ? counts[w] : 0;
            all += counts[w];
        }
        const int64_t at = base + before + __popcll(mask & (((uint64_t)1 << lane) - 1));  // tokens that count before this one
        if (i < N) list[in ? at : N - 1 - (i - at)] = (int32_t)i;
        base += all;
    }
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) {
        const uint32_t o = __shfl_xor(top, off, kWave);
        top = o > top ? o : top;
    }
    if (lane == 0) tops[wv] = top;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 0; w < kListThreads / kWave; ++w) top = tops[w] > top ? tops[w] : top;
    *active = active_of((int32_t)base, top, lift);
}

// Rows of dX of tokens that do not count.
template <typename T>
__global__ __launch_bounds__(256) void xent_zero_rows(const int32_t* __restrict__ list, const Active* __restrict__ active, int64_t N, int64_t D, T* __restrict__ dX)
{
    for (int64_t i = active->count + (int64_t)blockIdx.x; i < N; i += gridDim.x) {
        T* p = dX + (int64_t)list[i] * D;
        for (int64_t d = threadIdx.x; d < D; d += blockDim.x) p[d] = (T)0.0f;
    }
}

// dz[token in the list][v - first]: vocabulary first .. first + width - 1 (ldz entries a row).
template <typename T>
__global__ __launch_bounds__(kTThreads) void xent_dz32(Operand<T> W, Operand<T> X, int64_t first, int64_t width, const void* __restrict__ targets,
                                                       int index_bytes, float scale, const float* __restrict__ lse, const float* __restrict__ g,
                                                       const Active* __restrict__ active, float* __restrict__ dz, int64_t ldz)
{
    __shared__ TileLds sh;
    const int64_t v0 = first + (int64_t)blockIdx.x * kT, n0 = (int64_t)blockIdx.y * kT;
    X.outer = active->count;
    if (n0 >= X.outer) return;
    v4f acc[4][4];
    tile32<true, true>(W, X, v0, n0, W.inner, sh, acc);
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const int li = lane & 15, kq = lane >> 4, wr = (wv >> 1) * 64, wc = (wv & 1) * 64;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const int64_t n = n0 + wc + b * 16 + li;
        if (n >= X.outer) continue;
        const int64_t row = X.idx[n];
        const int64_t t = index_at(targets, index_bytes, row);
        const float l = lse[row], gi = g[row] / active->ref;
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t v = v0 + wr + a * 16 + kq * 4 + r;
                if (v < first + width) dz[n * ldz + (v - first)] = gi * (lifted_exp<kLift<T>>(acc[a][b][r] * scale - l) - (v == t ? (float)(1 << kLift<T>) : 0.0f));
            }
    }
}

// dX += scale dz W over a piece: dims x tokens.  The sum over the pieces is kept in `sum` (list order) until the last one.
template <typename T>
__global__ __launch_bounds__(kTThreads) void xent_dx32(Operand<T> W, Operand<float> Z, const int32_t* __restrict__ list, float scale,
                                                       const Active* __restrict__ active, int first_piece, int last_piece, float* __restrict__ sum,
                                                       T* __restrict__ dX)
{
    __shared__ TileLds sh;
    const int64_t d0 = (int64_t)blockIdx.x * kT, n0 = (int64_t)blockIdx.y * kT, D = W.inner;
    Z.outer = active->count;
    if (n0 >= Z.outer) return;
    v4f acc[4][4];
    tile32<false, true>(W, Z, d0, n0, W.outer, sh, acc);
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const int li = lane & 15, kq = lane >> 4, wr = (wv >> 1) * 64, wc = (wv & 1) * 64;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const int64_t n = n0 + wc + b * 16 + li;
        if (n >= Z.outer) continue;
        const int64_t row = list[n];
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t d = d0 + wr + a * 16 + kq * 4 + r;
                if (d >= D) continue;
                float v = acc[a][b][r];
                if (!first_piece) v += sum[n * D + d];
                if (last_piece) dX[row * D + d] = round_to<T>(v * scale * active->inv);
                else sum[n * D + d] = v;
            }
    }
}

// dW of a piece: dims x vocabulary.
template <typename T>
__global__ __launch_bounds__(kTThreads) void xent_dw32(Operand<T> X, Operand<float> Z, int64_t first, float scale, const Active* __restrict__ active,
                                                       T* __restrict__ dW)
{
    __shared__ TileLds sh;
    const int64_t d0 = (int64_t)blockIdx.x * kT, v0 = (int64_t)blockIdx.y * kT, D = X.inner;
    X.outer = active->count;
    Z.outer = active->count;
    v4f acc[4][4];
    tile32<false, false>(X, Z, d0, v0, X.outer, sh, acc);
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const int li = lane & 15, kq = lane >> 4, wr = (wv >> 1) * 64, wc = (wv & 1) * 64;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const int64_t v = v0 + wc + b * 16 + li;
        if (v >= Z.inner) continue;
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t d = d0 + wr + a * 16 + kq * 4 + r;
                if (d < D) dW[(first + v) * D + d] = round_to<T>(acc[a][b][r] * scale * active->inv);
            }
    }
}

// ------------------------------------------------------------------------------------------------ the tile's form

// How values are held for the tile: P planes of In.
template <typename I, class O, int PLANES>
struct Held {
    typedef I In;
    typedef O Op;
    static constexpr int P = PLANES, kVec = 16 / (int)sizeof(I);
};
typedef Held<__bf16, OpBf16, 1> HeldBf16;
typedef Held<_Float16, OpF16, 1> HeldF16;
typedef Held<float, OpSplit, 1> HeldSplit;
typedef Held<float, OpF32, 1> HeldF32;

// How dz is held: as the operands, or in twice the digits of their 16-bit type.
template <class H>
using Twice = Held<typename H::In, typename H::Op, 2>;

// Plane by plane what is left of x.
template <class H>
__device__ __forceinline__ void planes_of(float x, typename H::In (&out)[H::P])
{
    typedef typename H::In In;
#pragma unroll
    for (int p = 0; p < H::P; ++p) {
        out[p] = (In)x;
        x -= to_f32(out[p]);
    }
}

// Eight entries from column c of a row of D, zeros behind its end.
template <typename T>
__device__ __forceinline__ void row8(const T* __restrict__ row, int64_t c, int64_t D, bool vec, float (&x)[8])
{
    typedef typename Vec<T>::V V;
    constexpr int VN = Vec<T>::N;
    if (vec && c + 8 <= D) {
#pragma unroll
        for (int h = 0; h < 8; h += VN) {
            const V v = *(const V*)(row + c + h);
#pragma unroll
            for (int e = 0; e < VN; ++e) x[h + e] = to_f32(v[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = c + e < D ? to_f32(row[c + e]) : 0.0f;
    }
}

// Eight values of In.
template <typename In>
__device__ __forceinline__ void put8(In* __restrict__ to, const In (&y)[8])
{
    typedef typename Vec<In>::V V;
    constexpr int VN = Vec<In>::N;
#pragma unroll
    for (int h = 0; h < 8; h += VN) {
        V v;
#pragma unroll
        for (int e = 0; e < VN; ++e) v[e] = y[h + e];
        *(V*)(to + h) = v;
    }
}

// Puts a row into the tile's layout: P planes of ld entries (ld >= D, a multiple of 8; zeros behind D).
template <typename T, class H>
__device__ __forceinline__ void lay_out(const T* __restrict__ row, int64_t D, bool vec, typename H::In* __restrict__ out, int64_t ld, int tid, int threads)
{
    typedef typename H::In In;
    for (int64_t c = tid * 8; c < ld; c += threads * 8) {
        float x[8];
        row8(row, c, D, vec, x);
        if constexpr (std::is_same<H, HeldSplit>::value) {  // (what would round to infinity as bf16 does not)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = fabsf(x[e]) < INFINITY ? fminf(fmaxf(x[e], -0x1.fep127f), 0x1.fep127f) : x[e];
        }
        In y[H::P][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            In one[H::P];
            planes_of<H>(x[e], one);
#pragma unroll
            for (int p = 0; p < H::P; ++p) y[p][e] = one[p];
        }
#pragma unroll
        for (int p = 0; p < H::P; ++p) put8(out + p * ld + c, y[p]);
    }
}

constexpr int kLayThreads = 256, kLayRows = 4;  // a wave a row

template <typename T, class H>
__global__ __launch_bounds__(kLayThreads) void xent_lay_out(const T* __restrict__ from, int64_t rows, int64_t D, bool vec, typename H::In* __restrict__ out,
                                                            int64_t ld)
{
    const int64_t row = (int64_t)blockIdx.x * kLayRows + threadIdx.x / kWave;
    if (row < rows) lay_out<T, H>(from + row * D, D, vec, out + row * ld * H::P, ld, threadIdx.x % kWave, kWave);
}

constexpr float kLog2e = 1.4426950408889634f;

// Vocabulary x tokens, a strip of 16 FA vocabulary rows a wave; strips[strip][token].  W is a piece of the vocabulary that begins
// at row `first`.
template <class Q>
__global__ __launch_bounds__(Q::kThreads, 2) void xent_forward_tile(TileRows W, TileRows X, int64_t first, const void* __restrict__ targets, int index_bytes,
                                                                    float scale, Sums* __restrict__ strips, float* __restrict__ zt)
{
    __shared__ __align__(128) char lds[Q::kLds];
    const int64_t V = W.rows, N = X.rows;
    int64_t tv, tn;
    tile_order(blockIdx.x, cdiv(V, Q::TA), cdiv(N, Q::TB), kTileGroup, &tv, &tn);
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const int64_t v0 = tv * Q::TA + Q::SideA::row_of(wv / Q::WB, 0, lane);  // 4 FA vocabulary rows from here
    const int64_t strip = tv * Q::WA + wv / Q::WB;
    int64_t target[Q::FB];
    auto fetch = [&] {
#pragma unroll
        for (int b = 0; b < Q::FB; ++b) {  // (all on the way at once; during the product where registers are left for it)
            const int64_t n = tn * Q::TB + Q::SideB::col_of(wv % Q::WB, b, lane);
            target[b] = index_at(targets, index_bytes, n < N ? n : N - 1);
        }
    };
    if constexpr (Q::FA <= 4) fetch();
    v4f acc[Q::FA][Q::FB];
    Q::run(W, X, tv * Q::TA, tn * Q::TB, cdiv(W.bytes, kTileStep), lds, acc, alone_begin<Q>(tv, V, N, cdiv(W.bytes, kTileStep)));
    if constexpr (Q::FA > 4) fetch();
#pragma unroll
    for (int b = 0; b < Q::FB; ++b) {
        const int64_t n = tn * Q::TB + Q::SideB::col_of(wv % Q::WB, b, lane);
        const bool live = n < N;
        const int64_t t = live ? target[b] - first - v0 : -1;
        float top = -__builtin_inff();
#pragma unroll
        for (int a = 0; a < Q::FA; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int v = a * 4 + r;
                acc[a][b][r] = v0 + v < V ? acc[a][b][r] * scale : -__builtin_inff();
                top = fmaxf(top, acc[a][b][r]);
            }
        if (t >= 0 && t < 4 * Q::FA && v0 + t < V) {
            float z = 0.0f;
#pragma unroll
            for (int v = 0; v < 4 * Q::FA; ++v) z = v == t ? acc[v / 4][b][v % 4] : z;
            zt[n] = z;
        }
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const float base = top == -__builtin_inff() ? 0.0f : top;  // (a strip may hold nothing else)
        float sum = 0.0f;
#pragma unroll
        for (int a = 0; a < Q::FA; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f((acc[a][b][r] - base) * kLog2e);
        sum += __shfl_xor(sum, 16, kWave);
        sum += __shfl_xor(sum, 32, kWave);
        if (lane < 16 && live && strip * 16 * Q::FA < V) {
            Sums s;
            s.max = top;
            s.sum = sum;
            strips[(first / (16 * Q::FA) + strip) * N + n] = s;
        }
    }
}

// Shares of an operand along k: steps s0 to s1 of rows along k, and of rows across it.
__device__ __forceinline__ void steps_along(TileRows& m, int64_t s0, int64_t s1)
{
    m.p += s0 * kTileStep;
    m.bytes = s1 * kTileStep < m.bytes ? (s1 - s0) * kTileStep : m.bytes - s0 * kTileStep;
}
__device__ __forceinline__ void steps_across(TileRows& m, int64_t s0, int64_t s1, int64_t step)
{
    m.p += s0 * step * m.pitch;
    m.rows = s1 * step < m.rows ? (s1 - s0) * step : m.rows - s0 * step;
}

// Where the logits are too few tiles for the compute units: this workgroup's share of the sums over the dims,
// z[split][token][v] (ldz entries a row, a multiple of 64).  active: tokens of a list.
template <class Q>
__global__ __launch_bounds__(Q::kThreads, 2) void xent_shares_tile(TileRows W, TileRows X, const Active* __restrict__ active, int splits,
                                                                   float* __restrict__ z, int64_t ldz)
{
    __shared__ __align__(128) char lds[Q::kLds];
    const int64_t N = X.rows, all = cdiv(W.rows, Q::TA) * cdiv(N, Q::TB), split = blockIdx.x / all;
    int64_t tv, tn;
    tile_order(blockIdx.x - split * all, cdiv(W.rows, Q::TA), cdiv(N, Q::TB), kTileGroup, &tv, &tn);
    if (active) X.rows = active->count;
    if (tn * Q::TB >= X.rows) return;
    const int64_t steps = cdiv(W.bytes, kTileStep), s0 = steps * split / splits, s1 = steps * (split + 1) / splits;
    steps_along(W, s0, s1);
    steps_along(X, s0, s1);
    v4f acc[Q::FA][Q::FB];
    Q::run(W, X, tv * Q::TA, tn * Q::TB, s1 - s0, lds, acc);
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const int64_t v0 = tv * Q::TA + Q::SideA::row_of(wv / Q::WB, 0, lane);
    z += split * N * ldz;
#pragma unroll
    for (int b = 0; b < Q::FB; ++b) {
        const int64_t n = tn * Q::TB + Q::SideB::col_of(wv % Q::WB, b, lane);
        if (n >= X.rows) continue;
#pragma unroll
        for (int a = 0; a < Q::FA; ++a)
            if (v0 + a * 4 < ldz) *(v4f*)(z + n * ldz + v0 + a * 4) = acc[a][b];
    }
}

// The sum of the shares of four logits, in their order.
__device__ __forceinline__ v4f sum_shares(const float* __restrict__ z, int64_t share, int splits)
{
    v4f x = *(const v4f*)z;
#pragma unroll 4
    for (int s = 1; s < splits; ++s) x += *(const v4f*)(z + s * share);
    return x;
}

// Losses from the shares: WAVES waves a token.
constexpr int kSharesWaves = 4;
template <int WAVES>
__global__ __launch_bounds__(kSharesWaves * kWave) void xent_join_shares(const float* __restrict__ z, int64_t ldz, int splits, int64_t N, int64_t V,
                                                                         const void* __restrict__ targets, int index_bytes, int64_t ignore, float scale,
                                                                         float* __restrict__ loss, float* __restrict__ lse)
{
    __shared__ float tops[kSharesWaves], zts[kSharesWaves];
    __shared__ double sums[kSharesWaves];
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave, own = wv / WAVES * WAVES;  // the first wave of this token's
    const int64_t n = (int64_t)blockIdx.x * (kSharesWaves / WAVES) + wv / WAVES, at_n = n < N ? n : N - 1;
    const int64_t target = index_at(targets, index_bytes, at_n);
    float top = -__builtin_inff(), sum = 0.0f, zt = 0.0f;
    for (int64_t c = ((wv - own) * kWave + lane) * 4; c < V; c += WAVES * kWave * 4) {
        v4f x = sum_shares(z + at_n * ldz + c, N * ldz, splits) * scale;
        float high = top;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            x[r] = c + r < V ? x[r] : -__builtin_inff();
            high = fmaxf(high, x[r]);
            if (c + r == target) zt = x[r];
        }
        const float base = high == -__builtin_inff() ? 0.0f : high;
        sum *= expf(top - base);
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += expf(x[r] - base);
        top = high;
    }
    float all = top;
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) {
        all = fmaxf(all, __shfl_xor(all, off, kWave));
        zt += __shfl_xor(zt, off, kWave);  // (one lane's, the others' are zero)
    }
    if (lane == 0) tops[wv] = all, zts[wv] = zt;
    __syncthreads();
    zt = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all = fmaxf(all, tops[own + w]), zt += zts[own + w];
    double s = (double)(sum * expf(top - (all == -__builtin_inff() ? 0.0f : all)));
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) s += __shfl_xor(s, off, kWave);
    if (lane == 0) sums[wv] = s;
    __syncthreads();
    if (wv != own || lane || n >= N) return;
    s = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += sums[own + w];
    write_loss(n, all, s, zt, target, V, ignore, loss, lse);
}

// What dz of a token needs beside its logits: lse, g as it is held, the target.
struct Row {
    float lse, g;
    int32_t target, pad_;
};

struct GatherArgs {
    int64_t N, D, V, ignore, ld;
    const void* targets;
    int index_bytes;
    const float *lse, *g;
    int32_t* list;
    Active* active;
    Row* rows;
    bool vec, vec_out;  // rows of X, of dX are aligned to 16 bytes
};

constexpr int64_t kScanTokens = 8192;  // up to so many tokens every workgroup of xent_gather looks through all of them itself

// The tokens that count, one after the other: rows of X in the tile's layout, and their Row; rows of dX (if wanted) of those that
// do not: zero.  A wave a token.  SCAN: there is no list yet; every workgroup finds the places of its own tokens by looking
// through all of them (a few loads a thread), and writes their part of the list.  Else xent_list has run.
template <typename T, class H, bool SCAN>
__global__ __launch_bounds__(kLayThreads) void xent_gather(const T* __restrict__ X, GatherArgs a, typename H::In* __restrict__ out, T* __restrict__ dX)
{
    typedef typename Vec<T>::V V;
    constexpr int VN = Vec<T>::N;
    const int lane = threadIdx.x % kWave, wv = threadIdx.x / kWave;
    Active act;
    int64_t place = 0;  // SCAN: of this wave's token among those that count, or the number of such tokens before it
    bool in = false;
    if constexpr (SCAN) {
        __shared__ int32_t before[kLayRows], all[kLayRows];
        __shared__ uint32_t tops[kLayRows];
        __shared__ int32_t own[kLayRows];
        const int64_t r0 = (int64_t)blockIdx.x * kLayRows;
        int32_t nb = 0, na = 0;
        uint32_t top = 0;
        for (int64_t i = threadIdx.x; i < a.N; i += kLayThreads) {
            const float g = a.g[i];
            const bool c = counts_for(index_at(a.targets, a.index_bytes, i), a.V, a.ignore, g);
            const uint32_t m = c ? weight_of(g) : 0u;
            top = m > top ? m : top;
            na += c;
            nb += c && i < r0;
            if (i >= r0 && i < r0 + kLayRows) own[i - r0] = c;
        }
#pragma unroll
        for (int off = kWave / 2; off > 0; off >>= 1) {
            const uint32_t o = __shfl_xor(top, off, kWave);
            top = o > top ? o : top;
            na += __shfl_xor(na, off, kWave);
            nb += __shfl_xor(nb, off, kWave);
        }
        if (lane == 0) before[wv] = nb, all[wv] = na, tops[wv] = top;
        __syncthreads();
        na = nb = 0;
#pragma unroll
        for (int w = 0; w < kLayRows; ++w) {
            nb += before[w];
            na += all[w];
            top = tops[w] > top ? tops[w] : top;
        }
        act = active_of(na, top, kLift<T>);
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.active = act;
        place = nb;
        for (int w = 0; w < wv; ++w) place += own[w];  // (rows of this workgroup before this wave's exist if its own does)
        in = r0 + wv < a.N && own[wv];
    } else {
        act = *a.active;
    }
    for (int64_t r = (int64_t)blockIdx.x * kLayRows + wv; r < a.N; r += SCAN ? a.N : (int64_t)gridDim.x * kLayRows) {
        int64_t row, i;  // a token, and its place in the list
        if constexpr (SCAN) {
            row = r;
            i = in ? place : a.N - 1 - (r - place);
            if (lane == 0) a.list[i] = (int32_t)row;
        } else {
            i = r;
            row = a.list[i];
            in = i < act.count;
        }
        if (in) {
            if (lane == 0) {
                Row x;
                x.lse = a.lse[row];
                x.g = a.g[row] / act.ref;
                x.target = (int32_t)index_at(a.targets, a.index_bytes, row);
                x.pad_ = 0;
                a.rows[i] = x;
            }
            lay_out<T, H>(X + row * a.D, a.D, a.vec, out + i * a.ld * H::P, a.ld, lane, kWave);
        } else if (dX && a.vec_out) {
            for (int64_t c = lane; c < a.D / VN; c += kWave) ((V*)(dX + row * a.D))[c] = (V)(T)0.0f;
        } else if (dX) {
            for (int64_t c = lane; c < a.D; c += kWave) dX[row * a.D + c] = (T)0.0f;
        }
    }
}

// dz as it is held, before it is rounded, from the sum of a logit.  (16-bit types: the lift goes into the exponent only where exp z alone
// would run out of digits; beside it, an exponent near 0 would keep 19 binary places of its own, and 1 - p of a token whose target is
// all but certain with it.)
template <typename T>
__device__ __forceinline__ float dz_of(float sum, float scale, const Row& row, bool target)
{
    constexpr float kUp = (float)(1 << kLift<T>);
    const float z = sum * scale - row.lse;
    float p;
    if constexpr (sizeof(T) == 4) {
        p = lifted_exp<kLift<T>>(z);
    } else {
        const bool low = z < -60.0f;
        p = __builtin_amdgcn_exp2f(z * kLog2e + (low ? (float)kLift<T> : 0.0f)) * (low ? 1.0f : kUp);
    }
    return row.g * (p - (target ? kUp : 0.0f));
}

// dz from shares of the logits.
template <typename T, class H>
__global__ __launch_bounds__(256) void xent_dz_shares(const float* __restrict__ z, int splits, int64_t N, int64_t V, float scale, const Row* __restrict__ rows,
                                                      const Active* __restrict__ active, typename H::In* __restrict__ dz, int64_t ldz)
{
    typedef typename H::In In;
    const int64_t cpr = ldz / 8, all = active->count * cpr;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t n = i / cpr, c = (i - n * cpr) * 8;
        const Row row = rows[n];
        In out[H::P][8];
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
            const v4f x = sum_shares(z + n * ldz + c + h, N * ldz, splits);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t v = c + h + r;
                In one[H::P];
                planes_of<H>(v < V ? dz_of<T>(x[r], scale, row, v == row.target) : 0.0f, one);
#pragma unroll
                for (int p = 0; p < H::P; ++p) out[p][h + r] = one[p];
            }
        }
#pragma unroll
        for (int p = 0; p < H::P; ++p) put8(dz + (n * H::P + p) * ldz + c, out[p]);
    }
}

// H: how dz is held.
template <typename T, class H, class Q>
__global__ __launch_bounds__(Q::kThreads, 2) void xent_dz_tile(TileRows W, TileRows X, int64_t first, float scale, const Row* __restrict__ rows,
                                                               const Active* __restrict__ active, typename H::In* __restrict__ dz, int64_t ldz)
{
    typedef typename H::In In;
    constexpr int P = H::P;
    __shared__ __align__(128) char lds[Q::kLds];
    const int64_t V = W.rows;  // of the piece
    int64_t tv, tn;
    tile_order(blockIdx.x, cdiv(V, Q::TA), cdiv(X.rows, Q::TB), kTileGroup, &tv, &tn);
    const int64_t N = X.rows;
    X.rows = active->count;
    if (tn * Q::TB >= X.rows) return;
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const int64_t v0 = tv * Q::TA + Q::SideA::row_of(wv / Q::WB, 0, lane);
    Row row[Q::FB];
    auto fetch = [&] {
#pragma unroll
        for (int b = 0; b < Q::FB; ++b) {  // (as above)
            const int64_t n = tn * Q::TB + Q::SideB::col_of(wv % Q::WB, b, lane);
            row[b] = rows[n < X.rows ? n : X.rows - 1];
        }
    };
    if constexpr (Q::FA <= 4) fetch();
    v4f acc[Q::FA][Q::FB];
    Q::run(W, X, tv * Q::TA, tn * Q::TB, cdiv(W.bytes, kTileStep), lds, acc, alone_begin<Q>(tv, V, N, cdiv(W.bytes, kTileStep)));
    if constexpr (Q::FA > 4) fetch();
#pragma unroll
    for (int b = 0; b < Q::FB; ++b) {
        const int64_t n = tn * Q::TB + Q::SideB::col_of(wv % Q::WB, b, lane);
        if (n >= X.rows) continue;
        const int64_t t = row[b].target - first - v0;
#pragma unroll
        for (int c = 0; c < 4 * Q::FA; c += 8) {
            In out[P][8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int v = c + e;
                In one[P];
                planes_of<H>(v0 + v < V ? dz_of<T>(acc[v / 4][b][v % 4], scale, row[b], v == t) : 0.0f, one);
#pragma unroll
                for (int q = 0; q < P; ++q) out[q][e] = one[q];
            }
            if (v0 + c < ldz)
#pragma unroll
                for (int q = 0; q < P; ++q) put8(dz + (n * P + q) * ldz + v0 + c, out[q]);
        }
    }
}

// Four results that follow one another in a row, as far as they lie in it.
template <typename T>
__device__ __forceinline__ void put4(T* __restrict__ row, int64_t d, int64_t D, bool vec, v4f v, float scale, float inv)
{
    typedef T V4 __attribute__((ext_vector_type(4)));
    V4 out;
#pragma unroll
    for (int r = 0; r < 4; ++r) out[r] = round_to<T>(v[r] * scale * inv);
    if (vec) {
        *(V4*)(row + d) = out;
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (d + r < D) row[d + r] = out[r];
    }
}

// dims x tokens.  splits == 1: sums over the pieces as in xent_dx32.  Else this workgroup's share of each piece goes to `sum`
// [split][token of the list][dim], and xent_join_grads makes dX of the shares.  Rows of `sum` have ld entries (a multiple of 8).
template <typename T>
struct DxArgs {
    TileRows W, Z;
    const int32_t* list;
    int first_piece, last_piece, splits;
    int64_t ld;
    float* sum;
    T* dX;
    bool vec;
};

template <typename T, class Q>
__device__ __forceinline__ void dx_tile(char* lds, int64_t block, const DxArgs<T>& a, int64_t D, float scale, const Active* __restrict__ active)
{
    TileRows W = a.W, Z = a.Z;
    const int32_t* list = a.list;
    const int first_piece = a.first_piece, last_piece = a.last_piece, splits = a.splits;
    const int64_t ld = a.ld;
    float* sum = a.sum;
    T* dX = a.dX;
    const bool vec = a.vec;
    const int64_t N = Z.rows, all = cdiv(D, Q::TA) * cdiv(N, Q::TB);
    const int64_t split = splits == 1 ? 0 : block / all;
    int64_t td, tn;
    tile_order(block - split * all, cdiv(D, Q::TA), cdiv(N, Q::TB), kTileGroup, &td, &tn);
    Z.rows = active->count;
    if (tn * Q::TB >= Z.rows) return;
    int64_t steps = cdiv(W.rows, Q::kRows);
    if (splits > 1) {  // whole steps of the vocabulary
        const int64_t s0 = steps * split / splits, s1 = steps * (split + 1) / splits;
        steps_across(W, s0, s1, Q::kRows);
        steps_along(Z, s0, s1);
        steps = s1 - s0;
        sum += split * N * ld;
    }
    v4f acc[Q::FA][Q::FB];
    Q::run(W, Z, td * Q::TA, tn * Q::TB, steps, lds, acc);
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const float inv = active->inv;
#pragma unroll
    for (int b = 0; b < Q::FB; ++b) {
        const int64_t n = tn * Q::TB + Q::SideB::col_of(wv % Q::WB, b, lane);
        if (n >= Z.rows) continue;
        const int64_t row = list[n];
#pragma unroll
        for (int a = 0; a < Q::FA; ++a) {
            const int64_t d = td * Q::TA + Q::SideA::row_of(wv / Q::WB, a, lane);
            if (d >= D) continue;
            v4f* s = (v4f*)(sum + n * ld + d);
            v4f v = acc[a][b];
            if (!first_piece) v += *s;
            if (last_piece && splits == 1) put4(dX + row * D, d, D, vec, v, scale, inv);
            else *s = v;
        }
    }
}

// Shares of a gradient, [split][row][dim], and where their sums go.  list: rows of dX, else those of dW.
template <typename T>
struct JoinArgs {
    const float* sum;
    const int32_t* list;
    int64_t rows, ld;
    int splits;
    T* out;
    bool vec;
};

// The shares of dX (`x_blocks` workgroups) and of dW, in their order.
template <typename T>
__global__ __launch_bounds__(256) void xent_join_grads(JoinArgs<T> x, JoinArgs<T> w, int x_blocks, int64_t D, float scale, const Active* __restrict__ active)
{
    const bool is_x = (int)blockIdx.x < x_blocks;
    const JoinArgs<T> a = is_x ? x : w;
    const int64_t block = is_x ? blockIdx.x : blockIdx.x - x_blocks, blocks = is_x ? x_blocks : gridDim.x - x_blocks;
    const int64_t cpr = cdiv(D, 4), all = (is_x ? active->count : a.rows) * cpr;
    const float inv = active->inv;
    for (int64_t i = block * 256 + threadIdx.x; i < all; i += blocks * 256) {
        const int64_t n = i / cpr, c = (i - n * cpr) * 4, row = is_x ? a.list[n] : n;
        put4(a.out + row * D, c, D, a.vec, sum_shares(a.sum + n * a.ld + c, a.rows * a.ld, a.splits), scale, inv);
    }
}

// dims x vocabulary of a piece.  A tile of dW in 16 bits goes through LDS, so that whole stretches of its rows are written at
// once: with few tokens writing dW is all there is to do (one token, 32000 x 4096: 104 us without, 73 with).  16-byte chunks of
// a row are permuted by an exclusive or with the row, so that neither the lanes' four dims nor the rows meet on a bank.
// Written past the caches (150 tokens, 32000 x 4096: 333 -> 293 us; 4096 of them 3214 -> 3203; small gradients as before).
// splits > 1: this workgroup's share of the tokens goes to `sum` [split][v][dim] (rows of ld entries).
template <typename T>
struct DwArgs {
    TileRows X, Z;
    int64_t width;
    int splits;
    int64_t ld;
    float* sum;
    T* dW;
    bool vec;
};

template <typename T, class Q>
__device__ __forceinline__ void dw_tile(char* lds, int64_t block, const DwArgs<T>& a, int64_t D, float scale, const Active* __restrict__ active)
{
    TileRows X = a.X, Z = a.Z;
    const int64_t width = a.width;
    T* dW = a.dW;
    const bool vec = a.vec;
    const int64_t all = cdiv(D, Q::TA) * cdiv(width, Q::TB), split = a.splits == 1 ? 0 : block / all;
    int64_t td, tv;
    tile_order(block - split * all, cdiv(D, Q::TA), cdiv(width, Q::TB), kTileGroup, &td, &tv);
    X.rows = Z.rows = active->count;
    int64_t steps = cdiv(X.rows, Q::kRows);
    if (a.splits > 1) {
        const int64_t s0 = steps * split / a.splits, s1 = steps * (split + 1) / a.splits;
        steps_across(X, s0, s1, Q::kRows);
        steps_across(Z, s0, s1, Q::kRows);
        steps = s1 - s0;
    }
    v4f acc[Q::FA][Q::FB];
    Q::run(X, Z, td * Q::TA, tv * Q::TB, steps, lds, acc);
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const float inv = active->inv;
    const int64_t v0 = tv * Q::TB, d0 = td * Q::TA;
    if (a.splits > 1) {
        float* sum = a.sum + split * width * a.ld;
#pragma unroll
        for (int b = 0; b < Q::FB; ++b) {
            const int64_t v = v0 + Q::SideB::col_of(wv % Q::WB, b, lane);
            if (v >= width) continue;
#pragma unroll
            for (int f = 0; f < Q::FA; ++f) {
                const int64_t d = d0 + Q::SideA::row_of(wv / Q::WB, f, lane);
                if (d < D) *(v4f*)(sum + v * a.ld + d) = acc[f][b];
            }
        }
        return;
    }
    if constexpr (sizeof(T) == 4) {  // 64 bytes of a row at once as it is
#pragma unroll
        for (int b = 0; b < Q::FB; ++b) {
            const int64_t v = v0 + Q::SideB::col_of(wv % Q::WB, b, lane);
            if (v >= width) continue;
#pragma unroll
            for (int a = 0; a < Q::FA; ++a) {
                const int64_t d = d0 + Q::SideA::row_of(wv / Q::WB, a, lane);
                if (d < D) put4(dW + v * D, d, D, vec, acc[a][b], scale, inv);
            }
        }
    } else {
        static_assert(Q::TA * Q::TB * 2 <= Q::kLds, "the tile fits where its operands were");
        typedef T V4 __attribute__((ext_vector_type(4)));
        typedef typename Vec<T>::V V8;
        constexpr int kRow = Q::TA * 2, kChunks = kRow / 16, kKey = kChunks < 16 ? kChunks - 1 : 15;
#pragma unroll
        for (int b = 0; b < Q::FB; ++b) {
            const int v = Q::SideB::col_of(wv % Q::WB, b, lane);
#pragma unroll
            for (int a = 0; a < Q::FA; ++a) {
                const int d = Q::SideA::row_of(wv / Q::WB, a, lane);
                V4 out;
#pragma unroll
                for (int r = 0; r < 4; ++r) out[r] = round_to<T>(acc[a][b][r] * scale * inv);
                *(V4*)(lds + v * kRow + (((d / 8) ^ (v & kKey)) * 16) + (d & 4) * 2) = out;
            }
        }
        __syncthreads();
#pragma unroll 4
        for (int i = threadIdx.x; i < Q::TB * kChunks; i += Q::kThreads) {
            const int v = i / kChunks, c = i % kChunks;
            const V8 x = *(const V8*)(lds + v * kRow + (c ^ (v & kKey)) * 16);
            if (v0 + v >= width) continue;
            T* to = dW + (v0 + v) * D + d0 + c * 8;
            if (vec) {
                if (d0 + c * 8 < D) __builtin_nontemporal_store(x, (V8*)to);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (d0 + c * 8 + e < D) to[e] = x[e];
            }
        }
    }
}

// dW of a piece from few tokens, STEPS steps of them, where writing it is all there is to do.  A workgroup keeps 128 dims of its tokens
// in registers and walks along the vocabulary, 64 rows at a time: dz of the rows two stretches ahead is on its way to LDS while the
// products of these are rounded there and written out, 256 or 512 bytes of a row at once, past the caches: they hold no gradient of
// this size for its reader, but much of W for the next product.  (32000 x 4096 bf16, two tokens: 93 us by dw_tile, whose workgroups
// each wait for their own operands, 53 here; a fill takes 38.)
template <typename T, class H, int STEPS>
struct DwFew {
    // (f32 as it is: with few tokens the f32 instruction keeps up)
    typedef typename std::conditional<sizeof(T) == 4, OpF32, typename H::Op>::type Op;
    static constexpr int ES = sizeof(typename H::In), P = H::P, FA = 4, FB = 2, WA = 2, WB = 2, WAVES = WA * WB, kThreads = WAVES * kWave;
    typedef TileSide<ES, FA, WA, WAVES, false, false, 1> SideX;
    typedef TileSide<ES, FB, WB, WAVES, false, false, P> SideZ;
    static constexpr int kStretch = SideZ::kBytes * STEPS * P, kLoads = SideZ::kLoads * STEPS * P;  // dz of 64 vocabulary rows
    static constexpr int kRow = SideX::T * (int)sizeof(T), kOut = SideZ::T * kRow, kChunks = kRow / 16, kVec = 16 / (int)sizeof(T);
    static constexpr int kFirst = kOut > SideX::kBytes ? kOut : SideX::kBytes, kLds = kFirst + 2 * kStretch;
    static constexpr int kTokens = STEPS * kTileStep / ES;
};

template <typename T, class H, int STEPS>
__global__ __launch_bounds__(256, 2) void xent_dw_few(TileRows X, TileRows Z, int64_t width, int64_t D, float scale, const Active* __restrict__ active,
                                                      T* __restrict__ dW, bool vec)
{
    typedef DwFew<T, H, STEPS> C;
    typedef T V4 __attribute__((ext_vector_type(4)));
    typedef typename Vec<T>::V V;
    constexpr int ES = C::ES, P = C::P, FA = C::FA, FB = C::FB;
    __shared__ __align__(128) char lds_[C::kLds];
    LdsChar* lds = (LdsChar*)lds_;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
    const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t nd = cdiv(D, C::SideX::T), d0 = blockIdx.x % nd * C::SideX::T, stride = gridDim.x / nd, stretches = cdiv(width, C::SideZ::T);
    X.rows = Z.rows = active->count;
    const float inv = active->inv;
    const int steps = (int)cdiv(X.rows, C::SideX::kRows), halves = (int)cdiv(X.rows, C::SideX::kRows / 2);
    v4i fx[STEPS][2][FA];
    {
        typename C::SideX side;
        side.init(X, d0, wv, lane);
        side.init_reads(wv / C::WB, lane);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            side.aim(s, steps, 0);
#pragma unroll
            for (int j = 0; j < C::SideX::kLoads; ++j) side.issue(j, lds0, wv);
            arrive<0>();
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int a = 0; a < FA; ++a) fx[s][h][a] = side.read(lds, a, h);
            arrive<0>();
        }
    }
    typename C::SideZ side;
    auto load = [&](int64_t stretch, int buffer) {
        side.init(Z, (stretch < stretches ? stretch : 0) * C::SideZ::T, wv, lane);
        const int have = stretch < stretches ? steps : 0;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int p = 0; p < P; ++p) {
                side.aim(s, have, p * (int)Z.plane);
#pragma unroll
                for (int j = 0; j < C::SideZ::kLoads; ++j) side.issue(j, lds0 + C::kFirst + buffer * C::kStretch + (s * P + p) * C::SideZ::kBytes, wv);
            }
    };
    side.init_reads(wv % C::WB, lane);
    int64_t at = blockIdx.x / nd;
    load(at, 0);
    load(at + stride, 1);
    arrive<C::kLoads>();
    int buffer = 0;
    for (; at < stretches; at += stride, buffer ^= 1) {
        v4f acc[FA][FB];
#pragma unroll
        for (int a = 0; a < FA; ++a)
#pragma unroll
            for (int b = 0; b < FB; ++b) acc[a][b] = (v4f)0.0f;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (s * 2 + h >= halves) continue;
                    v4i fz[FB];
#pragma unroll
                    for (int b = 0; b < FB; ++b) fz[b] = side.read(lds + C::kFirst + buffer * C::kStretch + (s * P + p) * C::SideZ::kBytes, b, h);
#pragma unroll
                    for (int a = 0; a < FA; ++a)
#pragma unroll
                        for (int b = 0; b < FB; ++b) acc[a][b] = C::Op::mfma(fx[s][h][a], fz[b], acc[a][b]);
                }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // every wave has read this stretch, and written out the last
        load(at + 2 * stride, buffer);
#pragma unroll
        for (int b = 0; b < FB; ++b) {
            const int v = C::SideZ::col_of(wv % C::WB, b, lane);
#pragma unroll
            for (int a = 0; a < FA; ++a) {
                const int d = C::SideX::row_of(wv / C::WB, a, lane);
                V4 out;
#pragma unroll
                for (int r = 0; r < 4; ++r) out[r] = round_to<T>(acc[a][b][r] * scale * inv);
                *(V4*)(lds_ + v * C::kRow + (((d / C::kVec) ^ (v & 15)) * 16) + (d % C::kVec) * (int)sizeof(T)) = out;
            }
        }
        arrive<C::kLoads>();  // the next stretch is there, and all of this one's results
#pragma unroll
        for (int i = threadIdx.x; i < C::SideZ::T * C::kChunks; i += C::kThreads) {
            const int v = i / C::kChunks, c = i % C::kChunks;
            const V x = *(const V*)(lds_ + v * C::kRow + (c ^ (v & 15)) * 16);
            if (at * C::SideZ::T + v >= width) continue;
            T* to = dW + (at * C::SideZ::T + v) * D + d0 + c * C::kVec;
            if (vec) {
                if (d0 + c * C::kVec < D) __builtin_nontemporal_store(x, (V*)to);
            } else {
#pragma unroll
                for (int e = 0; e < C::kVec; ++e)
                    if (d0 + c * C::kVec + e < D) to[e] = x[e];
            }
        }
    }
}

// Both gradients of a piece, the tiles of dX (which sum more) first: they need the same dz, and neither leaves compute units idle
// while the other could use them.
template <typename T, class QX, class QW>
__global__ __launch_bounds__(QX::kThreads, 2) void xent_grads_tile(DxArgs<T> x, DwArgs<T> w, int64_t x_tiles, int64_t D, float scale,
                                                                   const Active* __restrict__ active)
{
    static_assert(QX::kThreads == QW::kThreads, "one workgroup for both");
    __shared__ __align__(128) char lds[QX::kLds > QW::kLds ? QX::kLds : QW::kLds];
    if ((int64_t)blockIdx.x < x_tiles) dx_tile<T, QX>(lds, blockIdx.x, x, D, scale, active);
    else dw_tile<T, QW>(lds, blockIdx.x - x_tiles, w, D, scale, active);
}

// ------------------------------------------------------------------------------------------------ host

constexpr int64_t kFewGroups = 768;   // workgroups of xent_dw_few, three a compute unit (512 and 1536: the same)
constexpr int64_t kWaveLogits = 512;  // logits in shares: up to so many of a token are joined by one wave

// Whether the tile takes rows of this length, and operands at these addresses (one that is copied in any case: nullptr).
bool tile_reaches(const Shape& s) { return s.ld * s.bytes <= kTileMaxPitch; }
bool tile_takes(const Shape& s, const void* X, const void* W) { return tile_reaches(s) && (s.copies_w || (aligned16(X) && aligned16(W))); }

struct ForwardSpace {
    size_t zt, strips, z, x, w, bytes;
};

size_t logits_bytes(const Shape& s) { return s.z_splits > 1 ? up(s.z_splits * (size_t)s.N * up((size_t)s.V, 64) * 4, 256) : 0; }

// Vocabulary rows that the forward takes at once.
int64_t forward_piece(const Shape& s) { return s.copies_w ? s.piece : s.V; }

// One layout for whichever form runs, since addresses have a say in that: strips of the tile or of tile32, or shares of the logits.
ForwardSpace forward_space(const Shape& s)
{
    ForwardSpace f;
    auto strips = [&](int64_t rows) { return up((size_t)cdiv(s.V, rows) * (size_t)s.N * sizeof(Sums), 256); };
    size_t most = 0;
    if (tile_reaches(s)) most = s.z_splits > 1 ? logits_bytes(s) : strips(strip_rows(logits_tile(s, forward_piece(s), s.N)));
    if (!s.copies_w || !tile_reaches(s)) most = strips(kStrip) > most ? strips(kStrip) : most;
    f.zt = 0;
    f.strips = f.z = up((size_t)s.N * 4, 256);
    f.x = f.z + most;
    f.w = f.x + (s.copies_w ? up((size_t)s.N * (size_t)s.ld * s.bytes, 256) : 0);
    f.bytes = f.w + (s.copies_w ? up((size_t)s.piece * (size_t)s.ld * s.bytes, 256) : 0) + 256;
    return f;
}

// One layout for both forms, since which of them runs depends on addresses.
struct GradSpace {
    size_t list, active, rows, dz, z, sum, w_sum, x, w, bytes;
    int64_t piece32;  // vocabulary rows of a piece in tile32's form
};

GradSpace grad_space(const Shape& s)
{
    GradSpace g;
    const size_t N = (size_t)s.N;
    g.piece32 = whole_rows(kPieceBytes, (N ? N : 1) * 4, s.V);
    const size_t dz32 = N * (size_t)g.piece32 * 4, dz = N * up((size_t)s.piece, 64) * s.dz_bytes;
    g.list = 0;
    g.active = up(N * 4, 256);
    g.rows = g.active + 256;
    g.dz = g.rows + up(N * sizeof(Row), 256);
    g.z = g.dz + up(dz32 > dz ? dz32 : dz, 256);
    g.sum = g.z + logits_bytes(s);
    const bool sums = g.piece32 < s.V || s.piece < s.V || s.splits > 1;
    g.w_sum = g.sum + (sums ? up((size_t)s.splits * N * (size_t)s.ld * 4, 256) : 0);
    g.x = g.w_sum + (s.w_splits > 1 ? up((size_t)s.w_splits * (size_t)s.V * (size_t)s.ld * 4, 256) : 0);
    g.w = g.x + up(N * (size_t)s.ld * s.bytes, 256);
    g.bytes = g.w + (s.copies_w ? up((size_t)s.piece * (size_t)s.ld * s.bytes, 256) : 0);
    return g;
}

// The tiles.
template <class H, bool A, bool B>  // (H: of the operand in more planes)
using Tile256 = Tile<typename H::Op, 8, 4, 2, 4, A, B, 2, H::P>;
template <class H, bool A, bool B>
using Tile128 = Tile<typename H::Op, 4, 4, 2, 2, A, B, 2, H::P>;
template <class H, bool A, bool B>
using Tile64 = Tile<typename H::Op, 2, 2, 2, 2, A, B, 3, H::P>;
// (one tile a compute unit)
template <class H, bool A, bool B>
using Deep128 = Tile<typename H::Op, 4, 4, 2, 2, A, B, 4, H::P>;
// (of the logits, which take the compute unit for themselves; of dX, which shares it with dW, fewer buffers)
template <class H, bool A, bool B>
using Tokens64 = Tile<typename H::Op, 2, 4, 4, 1, A, B, A ? 5 : 3, H::P>;  // 128 x 64 tokens
template <class H, bool A, bool B>
using Tokens32 = Tile<typename H::Op, 2, 2, 4, 1, A, B, A ? 6 : 3, H::P>;  // 128 x 32 tokens

template <class H, bool A, bool B, typename F>
hipError_t few_tile(int64_t tokens, F&& f)
{
    return tokens <= 32 ? f(Tokens32<H, A, B>{}) : f(Tokens64<H, A, B>{});
}

// f(Tile) for the logits of na vocabulary rows and nb tokens.
template <class H, typename F>
hipError_t with_tile(const Shape& s, int64_t na, int64_t nb, F&& f)
{
    switch (logits_tile(s, na, nb)) {
        case LogitsTile::tokens32: return f(Tokens32<H, true, true>{});
        case LogitsTile::tokens64: return f(Tokens64<H, true, true>{});
        case LogitsTile::t256:
            if constexpr (sizeof(typename H::In) == 2) return f(Tile256<H, true, true>{});
            return hipErrorInvalidConfiguration;  // (16-bit types only)
        case LogitsTile::deep128: return f(Deep128<H, true, true>{});
        case LogitsTile::t128: return f(Tile128<H, true, true>{});
        default: return f(Tile64<H, true, true>{});
    }
}

// f(tile of dX, tile of dW): how the gradients are taken.
template <class HZ, typename F>
hipError_t with_grad_tiles(const Shape& s, F&& f)
{
    if (s.grads == 0) return few_tile<HZ, false, true>(s.N, [&](auto q) { return f(q, Tile128<HZ, false, false>{}); });
    if constexpr (sizeof(typename HZ::In) == 2 && HZ::P == 1)
        if (s.grads == 256) return f(Tile256<HZ, false, true>{}, Tile256<HZ, false, false>{});
    return s.grads == 128 ? f(Tile128<HZ, false, true>{}, Tile128<HZ, false, false>{}) : f(Tile64<HZ, false, true>{}, Tile64<HZ, false, false>{});
}

template <class Q, typename K, typename... Args>
hipError_t launch_tiles(K kernel, int64_t na, int64_t nb, int64_t splits, hipStream_t st, Args... args)
{
    const int64_t grid = cdiv(na, Q::TA) * cdiv(nb, Q::TB) * splits;
    if (!grid_ok(grid, Q::kThreads)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(Q::kThreads), 0, st, args...);
    return hipGetLastError();
}

template <class H>
TileRows rows_of(const void* p, int64_t rows, int64_t ld)
{
    const int64_t es = sizeof(typename H::In);
    return TileRows{(const char*)p, ld * es * H::P, rows, ld * es, H::P > 1 ? ld * es : 0};
}

template <typename T, class H>
hipError_t lay_out_rows(const T* from, int64_t rows, int64_t D, void* to, int64_t ld, hipStream_t st)
{
    const bool vec = aligned16(from) && D * sizeof(T) % 16 == 0;
    hipLaunchKernelGGL((xent_lay_out<T, H>), dim3((unsigned)cdiv(rows, kLayRows)), dim3(kLayThreads), 0, st, from, rows, D, vec, (typename H::In*)to, ld);
    return hipGetLastError();
}

// Shares of the logits of a call that makes them in shares.
template <class H>
hipError_t logits_shares(const TileRows& w, const TileRows& x, const Shape& s, const Active* active, float* z, hipStream_t st)
{
    auto launch = [&](auto q) {
        typedef decltype(q) Q;
        return launch_tiles<Q>(xent_shares_tile<Q>, s.V, s.N, s.z_splits, st, w, x, active, s.z_splits, z, (int64_t)up((size_t)s.V, 64));
    };
    if (takes_few(s.N, s.V)) return few_tile<H, true, true>(s.N, launch);
    return launch(Tile64<H, true, true>{});
}

template <typename T, class H>
hipError_t forward_t(const void* X, const void* W, const Shape& s, const void* targets, int index_bytes, int64_t ignore, float scale, float* loss, float* lse,
                     char* ws, hipStream_t st)
{
    const int64_t N = s.N, D = s.D, V = s.V;
    const ForwardSpace sp = forward_space(s);
    float* zt = (float*)(ws + sp.zt);
    Sums* strips = (Sums*)(ws + sp.strips);
    int64_t nstrips = 0;
    hipError_t e = hipSuccess;
    if (tile_takes(s, X, W)) {
        if (s.copies_w && (e = lay_out_rows<T, H>((const T*)X, N, D, ws + sp.x, s.ld, st)) != hipSuccess) return e;
        const TileRows x = rows_of<H>(s.copies_w ? ws + sp.x : X, N, s.ld);
        const int64_t piece = forward_piece(s);
        for (int64_t v0 = 0; v0 < V; v0 += piece) {
            const int64_t width = V - v0 < piece ? V - v0 : piece;
            const T* from = (const T*)W + v0 * D;
            if (s.copies_w && (e = lay_out_rows<T, H>(from, width, D, ws + sp.w, s.ld, st)) != hipSuccess) return e;
            const TileRows w = rows_of<H>(s.copies_w ? (const void*)(ws + sp.w) : from, width, s.ld);
            if (s.z_splits > 1) {
                float* z = (float*)(ws + sp.z);
                if ((e = logits_shares<H>(w, x, s, nullptr, z, st)) != hipSuccess) return e;
                const int64_t ldz = (int64_t)up((size_t)V, 64);
                if (V <= kWaveLogits)
                    hipLaunchKernelGGL((xent_join_shares<1>), dim3((unsigned)cdiv(N, kSharesWaves)), dim3(kSharesWaves * kWave), 0, st, z, ldz, s.z_splits, N, V,
                                       targets, index_bytes, ignore, scale, loss, lse);
                else
                    hipLaunchKernelGGL((xent_join_shares<kSharesWaves>), dim3((unsigned)N), dim3(kSharesWaves * kWave), 0, st, z, ldz, s.z_splits, N, V,
                                       targets, index_bytes, ignore, scale, loss, lse);
                return hipGetLastError();
            }
            e = with_tile<H>(s, piece, N, [&](auto q) {  // (the same tile for every piece: the strips are its)
                typedef decltype(q) Q;
                static_assert(256 % (16 * Q::FA) == 0, "pieces hold whole strips");
                if (strip_rows(logits_tile(s, piece, N)) != 16 * Q::FA) return hipErrorInvalidConfiguration;  // (the work space holds so many)
                nstrips = cdiv(V, 16 * Q::FA);
                return launch_tiles<Q>(xent_forward_tile<Q>, width, N, 1, st, w, x, v0, targets, index_bytes, scale, strips, zt);
            });
            if (e != hipSuccess) return e;
        }
    } else {
        const Operand<T> w{(const T*)W, D, nullptr, V, D}, x{(const T*)X, D, nullptr, N, D};
        if (cdiv(N, kT) > 65535 || !grid_ok(cdiv(V, kT), kTThreads)) return hipErrorInvalidConfiguration;
        hipLaunchKernelGGL((xent_forward32<T>), dim3((unsigned)cdiv(V, kT), (unsigned)cdiv(N, kT)), dim3(kTThreads), 0, st, w, x, targets, index_bytes, scale,
                           strips, zt);
        nstrips = cdiv(V, kStrip);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (N < 256)
        hipLaunchKernelGGL((xent_join<1>), dim3((unsigned)N), dim3(kJoinThreads), 0, st, strips, nstrips, N, V, targets, index_bytes, ignore, zt, loss, lse);
    else
        hipLaunchKernelGGL((xent_join<16>), dim3((unsigned)cdiv(N, 16)), dim3(kJoinThreads), 0, st, strips, nstrips, N, V, targets, index_bytes, ignore, zt,
                           loss, lse);
    return hipGetLastError();
}

struct GradArgs {
    const void *X, *W, *targets;
    int index_bytes;
    int64_t ignore;
    float scale;
    const float *lse, *g;
    void *dX, *dW;
    char* ws;
};

template <typename T>
hipError_t make_list(const GradArgs& a, const Shape& s, const GradSpace& sp, hipStream_t st)
{
    hipLaunchKernelGGL(xent_list, dim3(1), dim3(kListThreads), 0, st, a.targets, a.index_bytes, s.N, s.V, a.ignore, a.g, kLift<T>, (int32_t*)(a.ws + sp.list),
                       (Active*)(a.ws + sp.active));
    return hipGetLastError();
}

template <typename T, class H, class HZ>
hipError_t grad_tile_t(const GradArgs& a, const Shape& s, const GradSpace& sp, hipStream_t st)
{
    typedef typename H::In In;
    const int64_t N = s.N, D = s.D, V = s.V;
    const int32_t* list = (const int32_t*)(a.ws + sp.list);
    const Active* active = (const Active*)(a.ws + sp.active);
    Row* rows = (Row*)(a.ws + sp.rows);
    In* dz = (In*)(a.ws + sp.dz);
    float* sum = (float*)(a.ws + sp.sum);
    const bool row16 = D * sizeof(T) % 16 == 0, vec_x = row16 && aligned16(a.X), vec_dx = row16 && aligned16(a.dX), vec_dw = row16 && aligned16(a.dW);
    hipError_t e;
    GatherArgs ga;
    ga.N = N, ga.D = D, ga.V = V, ga.ignore = a.ignore, ga.ld = s.ld;
    ga.targets = a.targets, ga.index_bytes = a.index_bytes, ga.lse = a.lse, ga.g = a.g;
    ga.list = (int32_t*)(a.ws + sp.list), ga.active = (Active*)(a.ws + sp.active), ga.rows = rows;
    ga.vec = vec_x, ga.vec_out = vec_dx;
    const int64_t groups = cdiv(N, kLayRows);
    if (N > 0 && N <= kScanTokens) {
        hipLaunchKernelGGL((xent_gather<T, H, true>), dim3((unsigned)groups), dim3(kLayThreads), 0, st, (const T*)a.X, ga, (In*)(a.ws + sp.x), (T*)a.dX);
        e = hipGetLastError();
    } else {
        e = make_list<T>(a, s, sp, st);
        if (e == hipSuccess && N > 0) {
            hipLaunchKernelGGL((xent_gather<T, H, false>), dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(kLayThreads), 0, st, (const T*)a.X, ga,
                               (In*)(a.ws + sp.x), (T*)a.dX);
            e = hipGetLastError();
        }
    }
    if (e != hipSuccess) return e;
    const int64_t piece = s.piece, ldz = (int64_t)up((size_t)piece, 64);
    const int splits = s.splits, w_splits = s.w_splits;
    float* w_sum = (float*)(a.ws + sp.w_sum);
    const TileRows x = rows_of<H>(a.ws + sp.x, N, s.ld);
    for (int64_t v0 = 0; v0 < V; v0 += piece) {
        const int64_t width = V - v0 < piece ? V - v0 : piece;
        const bool first = v0 == 0, last = v0 + width == V;
        const T* from = (const T*)a.W + v0 * D;
        if (N > 0) {
            if (s.copies_w && (e = lay_out_rows<T, H>(from, width, D, a.ws + sp.w, s.ld, st)) != hipSuccess) return e;
            const TileRows w = rows_of<H>(s.copies_w ? (const void*)(a.ws + sp.w) : from, width, s.ld);
            if (s.z_splits > 1) {
                float* shared = (float*)(a.ws + sp.z);
                if ((e = logits_shares<H>(w, x, s, active, shared, st)) != hipSuccess) return e;
                const int64_t blocks = cdiv(N * (ldz / 8), 256);
                hipLaunchKernelGGL((xent_dz_shares<T, HZ>), dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, st, shared, s.z_splits, N, V, a.scale,
                                   rows, active, dz, ldz);
                e = hipGetLastError();
            } else {
                e = with_tile<H>(s, width, N, [&](auto q) {
                    typedef decltype(q) Q;
                    return launch_tiles<Q>(xent_dz_tile<T, HZ, Q>, width, N, 1, st, w, x, v0, a.scale, rows, active, dz, ldz);
                });
            }
            if (e != hipSuccess) return e;
        }
        TileRows w{}, z = rows_of<HZ>(dz, N, ldz);
        DwArgs<T> dw{x, z, width, w_splits, s.ld, w_sum, (T*)a.dW + v0 * D, vec_dw};
        if (N > 0) w = rows_of<H>(s.copies_w ? (const void*)(a.ws + sp.w) : from, width, s.ld);
        z.bytes = (int64_t)up((size_t)width, 8) * (int64_t)sizeof(In);
        const DxArgs<T> dx{w, z, list, (int)first, (int)last, splits, s.ld, sum, (T*)a.dX, vec_dx};
        bool rest = a.dW;  // dW is still to be made
        {
            typedef DwFew<T, HZ, HZ::P == 2 ? 1 : 2> F;
            static_assert(F::kTokens == (sizeof(T) == 4 || HZ::P == 2 ? 64 : 128), "as many tokens as walk_tokens says");
            if (rest && dw_walks(s, width, a.dX)) {
                const int64_t nd = cdiv(D, F::SideX::T), stretches = cdiv(width, F::SideZ::T), groups = cdiv(kFewGroups, nd);
                const int64_t grid = nd * (groups < stretches ? groups : stretches);
                if (!grid_ok(grid, F::kThreads)) return hipErrorInvalidConfiguration;
                hipLaunchKernelGGL((xent_dw_few<T, HZ, HZ::P == 2 ? 1 : 2>), dim3((unsigned)grid), dim3(F::kThreads), 0, st, x, z, width, D, a.scale, active, dw.dW,
                                   vec_dw);
                if ((e = hipGetLastError()) != hipSuccess) return e;
                rest = false;
            }
        }
        e = with_grad_tiles<HZ>(s, [&](auto qx, auto qw) {
            typedef decltype(qx) QX;
            typedef decltype(qw) QW;
            const int64_t nx = a.dX && N > 0 ? cdiv(D, QX::TA) * cdiv(N, QX::TB) * splits : 0, nw = rest ? cdiv(D, QW::TA) * cdiv(width, QW::TB) * w_splits : 0;
            if (nx + nw == 0) return hipSuccess;
            if (!grid_ok(nx + nw, QX::kThreads)) return hipErrorInvalidConfiguration;
            hipLaunchKernelGGL((xent_grads_tile<T, QX, QW>), dim3((unsigned)(nx + nw)), dim3(QX::kThreads), 0, st, dx, dw, nx, D, a.scale, active);
            return hipGetLastError();
        });
        const bool join_x = a.dX && N > 0 && splits > 1 && last, join_w = rest && w_splits > 1;
        if (e == hipSuccess && (join_x || join_w)) {
            const int64_t bx = join_x ? cdiv(N * cdiv(D, 4), 256) : 0, bw = join_w ? cdiv(V * cdiv(D, 4), 256) : 0;
            const int x_blocks = bx < 2048 ? (int)bx : 2048, w_blocks = bw < 2048 ? (int)bw : 2048;
            const JoinArgs<T> jx{sum, list, N, s.ld, splits, (T*)a.dX, vec_dx}, jw{w_sum, nullptr, V, s.ld, w_splits, (T*)a.dW, vec_dw};
            hipLaunchKernelGGL((xent_join_grads<T>), dim3((unsigned)(x_blocks + w_blocks)), dim3(256), 0, st, jx, jw, x_blocks, D, a.scale, active);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, class H>
hipError_t grad_t(const GradArgs& a, const Shape& s, hipStream_t st)
{
    const int64_t N = s.N, D = s.D, V = s.V;
    const GradSpace sp = grad_space(s);
    int32_t* list = (int32_t*)(a.ws + sp.list);
    Active* active = (Active*)(a.ws + sp.active);
    if (tile_takes(s, nullptr, a.W)) {  // (X's rows are gathered)
        if constexpr (sizeof(T) == 2)
            if (s.dz_planes == 2) return grad_tile_t<T, H, Twice<H>>(a, s, sp, st);
        return grad_tile_t<T, H, H>(a, s, sp, st);
    }
    hipError_t e = make_list<T>(a, s, sp, st);
    if (e != hipSuccess) return e;
    float *dz = (float*)(a.ws + sp.dz), *sum = (float*)(a.ws + sp.sum);
    const int64_t piece = sp.piece32, tn = cdiv(N, kT), td = cdiv(D, kT);
    if (tn > 65535 || cdiv(piece, kT) > 65535 || !grid_ok(td, kTThreads)) return hipErrorInvalidConfiguration;
    if (a.dX && N > 0) {
        hipLaunchKernelGGL((xent_zero_rows<T>), dim3((unsigned)(N < 1024 ? N : 1024)), dim3(256), 0, st, list, active, N, D, (T*)a.dX);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    for (int64_t v0 = 0; v0 < V; v0 += piece) {
        const int64_t width = V - v0 < piece ? V - v0 : piece, tv = cdiv(width, kT);
        const T *W = (const T*)a.W, *X = (const T*)a.X;
        const Operand<T> w{W, D, nullptr, V, D}, wp{W + v0 * D, D, nullptr, width, D}, x{X, D, list, N, D};
        const Operand<float> z{dz, piece, nullptr, N, width};
        if (N > 0) {
            hipLaunchKernelGGL((xent_dz32<T>), dim3((unsigned)tv, (unsigned)tn), dim3(kTThreads), 0, st, w, x, v0, width, a.targets, a.index_bytes, a.scale,
                               a.lse, a.g, active, dz, piece);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            if (a.dX) {
                hipLaunchKernelGGL((xent_dx32<T>), dim3((unsigned)td, (unsigned)tn), dim3(kTThreads), 0, st, wp, z, list, a.scale, active, v0 == 0,
                                   v0 + width == V, sum, (T*)a.dX);
                if ((e = hipGetLastError()) != hipSuccess) return e;
            }
        }
        if (a.dW) {
            hipLaunchKernelGGL((xent_dw32<T>), dim3((unsigned)td, (unsigned)tv), dim3(kTThreads), 0, st, x, z, v0, a.scale, active, (T*)a.dW);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

// f(T{}, Held{}) for a call.
template <typename F>
hipError_t with_held(int dt, const Shape& s, F&& f)
{
    if (dt == SCD_REAL_BF16) return f(__bf16{}, HeldBf16{});
    if (dt == SCD_REAL_F16) return f(_Float16{}, HeldF16{});
    return s.split ? f(float{}, HeldSplit{}) : f(float{}, HeldF32{});
}

bool sizes_ok(int dt, int64_t N, int64_t D, int64_t V) { return real_ok(dt) && rows_ok(N) && dim_ok(D) && dim_ok(V); }

}  // namespace
}  // namespace lm
}  // namespace scd

using namespace scd::lm;

extern "C" {

size_t scd_xent_workspace_bytes(scd_real dt, int64_t N, int64_t D, int64_t V)
{
    if (!sizes_ok(dt, N, D, V)) return 0;
    return forward_space(shape_of(dt, N, D, V)).bytes;
}

int scd_xent(const void* X, const void* W, scd_real dt, int64_t N, int64_t D, int64_t V, const void* targets, int index_bytes, int64_t ignore,
             float scale, float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!sizes_ok(dt, N, D, V) || !W || !index_ok(index_bytes) || (N > 0 && (!X || !targets || !loss || !lse))) return SCD_EINVAL;
    const Shape s = shape_of(dt, N, D, V);
    if (!workspace || !aligned16(workspace) || workspace_bytes < forward_space(s).bytes) return SCD_EINVAL;
    if (N == 0) return SCD_OK;
    const hipError_t e = with_held(dt, s, [&](auto z, auto h) {
        return forward_t<decltype(z), decltype(h)>(X, W, s, targets, index_bytes, ignore, scale, loss, lse, (char*)workspace, (hipStream_t)stream);
    });
    return e == hipSuccess ? SCD_OK : scd::report_hip(e);
}

size_t scd_xent_grad_workspace_bytes(scd_real dt, int64_t N, int64_t D, int64_t V)
{
    return sizes_ok(dt, N, D, V) ? grad_space(shape_of(dt, N, D, V)).bytes : 0;
}

int scd_xent_grad(const void* X, const void* W, scd_real dt, int64_t N, int64_t D, int64_t V, const void* targets, int index_bytes, int64_t ignore,
                  float scale, const float* lse, const float* g, void* dX, void* dW, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!sizes_ok(dt, N, D, V) || !W || !index_ok(index_bytes) || (!dX && !dW) || (N > 0 && (!X || !targets || !lse || !g))) return SCD_EINVAL;
    const Shape s = shape_of(dt, N, D, V);
    if (!workspace || !aligned16(workspace) || workspace_bytes < grad_space(s).bytes) return SCD_EINVAL;
    const GradArgs a{X, W, targets, index_bytes, ignore, scale, lse, g, dX, dW, (char*)workspace};
    const hipError_t e = with_held(dt, s, [&](auto z, auto h) { return grad_t<decltype(z), decltype(h)>(a, s, (hipStream_t)stream); });
    return e == hipSuccess ? SCD_OK : scd::report_hip(e);
}

}  // extern "C"
