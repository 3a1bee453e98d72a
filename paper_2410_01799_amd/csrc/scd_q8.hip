// Products in 8-bit integers (scd_q8_rows, scd_q8_linear, scd_q8_matmul).
//
//   q_ik = rint(x_ik * (127 * (1 / a_i))),  s_i = a_i / 127,  a_i = max(max_k |x_ik|, 2^-100)
//   y_ij = xs_i ws_j sum_k xq_ik wq_jk (+ bias_j)
// The sum is exact in int32: |q| <= 127 and K <= 131072 keep it below 2^31.  Both operands are rows along K, padded with
// zeros to whole 128 bytes, so no tile of a product has a tail along K.
#include "scd_lm_tile.h"

namespace scd {
namespace lm {
namespace {

// ------------------------------------------------------------------------------------------------ rows into 8 bits

constexpr int kRowThreads = 256;
constexpr int kHeld = 8;  // chunks of a row that a thread keeps in registers between the maximum and the rounding

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The multiplier and the scale of a row from the largest magnitude (its bits; NaN and infinity lie above all others).
__device__ __forceinline__ void row_scale(uint32_t top, float* mul, float* s)
{
    const bool bad = top >= 0x7F800000u;
    const float a = fmaxf(__uint_as_float(top), 0x1p-100f);
    *mul = bad ? 0.0f : 127.0f * (1.0f / a);
    *s = bad ? __builtin_nanf("") : a / 127.0f;
}

__device__ __forceinline__ int quantise(float x, float mul)
{
    return mul == 0.0f ? 0 : (int)rintf(x * mul);  // (an infinity times zero is not a number)
}

// TPR threads a row; a chunk is VN entries.  Rows of up to TPR * kHeld chunks are read once, longer ones twice.
template <typename T, int VN, int TPR>
__global__ __launch_bounds__(kRowThreads) void q8_rows_kernel(const T* __restrict__ X, int64_t M, int64_t K, int64_t stride, int8_t* __restrict__ q,
                                                              float* __restrict__ s)
{
    typedef T VT __attribute__((ext_vector_type(VN)));
    typedef int8_t VQ __attribute__((ext_vector_type(VN)));
    __shared__ uint32_t tops[kRowThreads / kWave];
    const int64_t row = (int64_t)blockIdx.x * (kRowThreads / TPR) + threadIdx.x / TPR;
    const int tid = threadIdx.x % TPR;
    const bool live = row < M;
    const T* x = X + (live ? row : 0) * K;
    const int64_t cpr = K / VN;
    VT held[kHeld];
    uint32_t top = 0;
    for (int64_t c0 = 0; c0 < cpr; c0 += TPR * kHeld) {
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            const int64_t c = c0 + h * TPR + tid;
            held[h] = c < cpr ? *(const VT*)(x + c * VN) : (VT)(T)0.0f;
        }
#pragma unroll
        for (int h = 0; h < kHeld; ++h)
#pragma unroll
            for (int e = 0; e < VN; ++e) {
                const uint32_t m = magnitude(to_f32(held[h][e]));
                top = m > top ? m : top;
            }
    }
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) {
        const uint32_t o = __shfl_xor(top, off, kWave);
        top = o > top ? o : top;
    }
    if constexpr (TPR > kWave) {
        if ((threadIdx.x & (kWave - 1)) == 0) tops[threadIdx.x / kWave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kRowThreads / kWave; ++w) top = tops[w] > top ? tops[w] : top;
    }
    if (!live) return;
    float mul, sc;
    row_scale(top, &mul, &sc);
    if (tid == 0) s[row] = sc;
    int8_t* o = q + row * stride;
    const int64_t cps = stride / VN;  // (a multiple of 128 bytes holds whole chunks)
    for (int64_t c0 = 0; c0 < cps; c0 += TPR * kHeld) {
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            const int64_t c = c0 + h * TPR + tid;
            if (c >= cps) continue;
            if (cpr > TPR * kHeld) held[h] = c < cpr ? *(const VT*)(x + c * VN) : (VT)(T)0.0f;
            VQ y;
#pragma unroll
            for (int e = 0; e < VN; ++e) y[e] = (int8_t)(c < cpr ? quantise(to_f32(held[h][e]), mul) : 0);
            *(VQ*)(o + c * VN) = y;
        }
    }
}

template <typename T, int VN>
hipError_t rows_t(const void* X, int64_t M, int64_t K, int8_t* q, float* s, hipStream_t st)
{
    // A wave for each row where that fills the chip and holds the row; else a workgroup.
    const bool narrow = M >= 1024 && K / VN <= kWave * kHeld;
    const int64_t grid = narrow ? cdiv(M, kRowThreads / kWave) : M;
    if (!grid_ok(grid, kRowThreads)) return hipErrorInvalidConfiguration;
    if (narrow)
        hipLaunchKernelGGL((q8_rows_kernel<T, VN, kWave>), dim3((unsigned)grid), dim3(kRowThreads), 0, st, (const T*)X, M, K, scd_q8_stride(K), q, s);
    else
        hipLaunchKernelGGL((q8_rows_kernel<T, VN, kRowThreads>), dim3((unsigned)grid), dim3(kRowThreads), 0, st, (const T*)X, M, K, scd_q8_stride(K), q, s);
    return hipGetLastError();
}

hipError_t rows(const void* X, int dt, int64_t M, int64_t K, int8_t* q, float* s, hipStream_t st)
{
    const bool vec = aligned16(X) && K * real_bytes(dt) % 16 == 0;
    return with_real(dt, [&](auto z) {
        typedef decltype(z) T;
        return vec ? rows_t<T, Vec<T>::N>(X, M, K, q, s, st) : rows_t<T, 1>(X, M, K, q, s, st);
    });
}

// ------------------------------------------------------------------------------------------------ product

// Channels are the tile's rows, tokens its columns: a lane ends with 4 FA channels of one token.
template <typename T, class Q>
__global__ __launch_bounds__(Q::kThreads, 2) void q8_tile_kernel(const int8_t* __restrict__ xq, const float* __restrict__ xs, int64_t M, int64_t stride,
                                                                 const int8_t* __restrict__ wq, const float* __restrict__ ws, int64_t N,
                                                                 const T* __restrict__ bias, T* __restrict__ y, bool vec)
{
    __shared__ __align__(128) char lds[Q::kLds];
    int64_t tn, tm;
    tile_order(blockIdx.x, cdiv(N, Q::TA), cdiv(M, Q::TB), kTileGroup, &tn, &tm);
    const TileRows W{(const char*)wq, stride, N, stride}, X{(const char*)xq, stride, M, stride};
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const int64_t n0 = tn * Q::TA + Q::SideA::row_of(wv / Q::WB, 0, lane);
    // What the results need besides the sums; on the way during the product where registers are left for it.
    constexpr bool kEarly = Q::FA <= 4;
    float w[4 * Q::FA], bs[4 * Q::FA], sx[Q::FB];
    auto fetch = [&] {
#pragma unroll
        for (int e = 0; e < 4 * Q::FA; ++e) {
            const int64_t n = n0 + e < N ? n0 + e : N - 1;
            w[e] = ws[n];
            bs[e] = bias ? to_f32(bias[n]) : 0.0f;
        }
#pragma unroll
        for (int b = 0; b < Q::FB; ++b) {
            const int64_t m = tm * Q::TB + Q::SideB::col_of(wv % Q::WB, b, lane);
            sx[b] = xs[m < M ? m : M - 1];
        }
    };
    if constexpr (kEarly) fetch();
    v4i acc[Q::FA][Q::FB];
    Q::run(W, X, tn * Q::TA, tm * Q::TB, stride / kTileStep, lds, acc, alone_begin<Q>(tn, N, M, stride / kTileStep));
    if constexpr (!kEarly) fetch();
    if constexpr (sizeof(T) == 2 && Q::FA == 8) {  // through LDS, so that whole stretches of a row are written at once
                                                   // (4096 tokens, 4096 -> 14336: 244 -> 227 us)
        static_assert(Q::TA * Q::TB * 2 <= Q::kLds, "the tile fits where its operands were");
        typedef T V8 __attribute__((ext_vector_type(8)));
        constexpr int kRow = Q::TA * 2, kChunks = kRow / 16;
        if (vec) {
            const int c0 = Q::SideA::row_of(wv / Q::WB, 0, lane) / 8;
#pragma unroll
            for (int b = 0; b < Q::FB; ++b) {
                const int m = Q::SideB::col_of(wv % Q::WB, b, lane);
#pragma unroll
                for (int c = 0; c < 4 * Q::FA; c += 8) {
                    V8 out;
#pragma unroll
                    for (int e = 0; e < 8; ++e) out[e] = round_to<T>((float)acc[(c + e) / 4][b][(c + e) % 4] * sx[b] * w[c + e] + bs[c + e]);
                    *(V8*)(lds + m * kRow + (((c0 + c / 8) ^ (m & 15)) * 16)) = out;
                }
            }
            __syncthreads();
#pragma unroll 4
            for (int i = threadIdx.x; i < Q::TB * kChunks; i += Q::kThreads) {
                const int m = i / kChunks, c = i % kChunks;
                const V8 x = *(const V8*)(lds + m * kRow + (c ^ (m & 15)) * 16);
                if (tm * Q::TB + m < M && tn * Q::TA + c * 8 < N) *(V8*)(y + (tm * Q::TB + m) * N + tn * Q::TA + c * 8) = x;
            }
            return;
        }
    }
    constexpr int VN = 16 / sizeof(T) < 4 * Q::FA ? 16 / sizeof(T) : 4 * Q::FA;  // channels of a store
    typedef T VT __attribute__((ext_vector_type(VN)));
#pragma unroll
    for (int b = 0; b < Q::FB; ++b) {
        const int64_t m = tm * Q::TB + Q::SideB::col_of(wv % Q::WB, b, lane);
        if (m >= M) continue;
#pragma unroll
        for (int c = 0; c < 4 * Q::FA; c += VN) {
            VT out;
#pragma unroll
            for (int e = 0; e < VN; ++e) out[e] = round_to<T>((float)acc[(c + e) / 4][b][(c + e) % 4] * sx[b] * w[c + e] + bs[c + e]);
            T* p = y + m * N + n0 + c;
            if (vec && n0 + c + VN <= N) {
                *(VT*)p = out;
            } else {
#pragma unroll
                for (int e = 0; e < VN; ++e)
                    if (n0 + c + e < N) p[e] = out[e];
            }
        }
    }
}

template <typename T, class Q>
hipError_t tile_t(const int8_t* xq, const float* xs, int64_t M, int64_t K, const int8_t* wq, const float* ws, int64_t N, const void* bias, void* y,
                  hipStream_t st)
{
    const int64_t grid = cdiv(N, Q::TA) * cdiv(M, Q::TB);
    if (!grid_ok(grid, Q::kThreads)) return hipErrorInvalidConfiguration;
    const bool vec = aligned16(y) && N * sizeof(T) % 16 == 0;
    hipLaunchKernelGGL((q8_tile_kernel<T, Q>), dim3((unsigned)grid), dim3(Q::kThreads), 0, st, xq, xs, M, scd_q8_stride(K), wq, ws, N, (const T*)bias, (T*)y,
                       vec);
    return hipGetLastError();
}

// Few tokens (at most 16, one column block of the matrix cores): bound by reading the weights, and with one matrix of a decode
// step by latency.  A workgroup takes 16 channels after the other; its waves share the rows' length between them, each with its
// own stretch of the weights on the way to its registers at once, the next channels' already while the waves' sums meet in LDS.
// OWN > 0: the tokens, at most OWN, are not yet in 8 bits; every workgroup does that for itself while its first weights are on
// the way, which takes less than a launch.  They lie in LDS then, and are read from there.
constexpr int kFewWaves = 8, kFewThreads = kFewWaves * kWave, kFewTokens = kQ8FewTokens, kFewChannels = 16;
constexpr int kFewFlight = 8;  // steps of 64 bytes that a wave has in flight
// LDS of the tokens' rows.
inline size_t few_lds(int own, int64_t M, int64_t K) { return (size_t)(own == kFewTokens ? M : own) * (size_t)(scd_q8_stride(K) + kQ8FewPad); }
constexpr int kFewGroups = 512;  // workgroups, at most: two on each compute unit

template <typename T>
struct FewTokens {
    const int8_t* xq;
    const float* xs;
    const T* x;
    bool vec;  // rows of x are aligned to 16 bytes
};

template <typename T, int OWN>
__global__ __launch_bounds__(kFewThreads) void q8_few_kernel(FewTokens<T> X, int M, int64_t K, int64_t stride, const int8_t* __restrict__ wq,
                                                             const float* __restrict__ ws, int64_t N, const T* __restrict__ bias, T* __restrict__ y)
{
    extern __shared__ __align__(16) int8_t own[];  // OWN tokens in 8 bits
    __shared__ v4i sums[2][kFewWaves][kWave];
    __shared__ uint32_t tops[kFewWaves][OWN ? OWN : 1];
    __shared__ float scales[kFewTokens];
    const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int li = lane & 15, kq = lane >> 4;
    const int steps = (int)(stride / 64), s0 = steps * wv / kFewWaves, s1 = steps * (wv + 1) / kFewWaves;
    const int m = li < M ? li : M - 1;
    v4i fw[kFewFlight];
    auto weights = [&](int64_t n0, int s) {
        const int8_t* w = wq + (n0 + li < N ? n0 + li : N - 1) * stride + kq * 16;
#pragma unroll
        for (int f = 0; f < kFewFlight; ++f) fw[f] = *(const v4i*)(w + (int64_t)(s + f < steps ? s + f : steps - 1) * 64);  // (past s1: times zero)
    };
    int64_t n0 = (int64_t)blockIdx.x * kFewChannels;
    weights(n0, s0);
    float sx = 0.0f;
    const int pitch = (int)stride + kQ8FewPad;
    if constexpr (OWN == kFewTokens) {
        constexpr int VN = 16 / sizeof(T);
        typedef typename Vec<T>::V VT;
        typedef int8_t VQ __attribute__((ext_vector_type(VN)));
        auto fetch = [&](const T* x, int c) {  // chunk c of a row, zeros behind its end
            VT v = (VT)(T)0.0f;
            if (X.vec) {
                if (c * VN < K) v = *(const VT*)(x + c * VN);
            } else {
#pragma unroll
                for (int e = 0; e < VN; ++e)
                    if (c * VN + e < K) v[e] = x[c * VN + e];
            }
            return v;
        };
        constexpr int kOnce = 4096 / VN / kWave;  // chunks of a lane between the maximum and the rounding (longer rows: read twice)
        const int chunks = (int)(stride / VN);
        for (int i = wv; i < M; i += kFewWaves) {
            const T* x = X.x + i * K;
            VT held[kOnce];
            uint32_t top = 0;
            for (int c0 = 0; c0 < chunks; c0 += kOnce * kWave) {
#pragma unroll
                for (int h = 0; h < kOnce; ++h) held[h] = fetch(x, c0 + h * kWave + lane);
#pragma unroll
                for (int h = 0; h < kOnce; ++h)
#pragma unroll
                    for (int e = 0; e < VN; ++e) {
                        const uint32_t t = magnitude(to_f32(held[h][e]));
                        top = t > top ? t : top;
                    }
            }
#pragma unroll
            for (int off = kWave / 2; off > 0; off >>= 1) {
                const uint32_t o = __shfl_xor(top, off, kWave);
                top = o > top ? o : top;
            }
            float mul, sc;
            row_scale(top, &mul, &sc);
            if (lane == 0) scales[i] = sc;
            for (int c0 = 0; c0 < chunks; c0 += kOnce * kWave) {
#pragma unroll
                for (int h = 0; h < kOnce; ++h) {
                    const int c = c0 + h * kWave + lane;
                    if (chunks > kOnce * kWave) held[h] = fetch(x, c);
                    if (c >= chunks) continue;
                    VQ q;
#pragma unroll
                    for (int e = 0; e < VN; ++e) q[e] = (int8_t)quantise(to_f32(held[h][e]), mul);
                    *(VQ*)(own + i * pitch + c * VN) = q;
                }
            }
        }
        __syncthreads();
        sx = scales[m];
    } else if constexpr (OWN > 0) {
        constexpr int VN = 16 / sizeof(T);
        typedef typename Vec<T>::V VT;
        typedef int8_t VQ __attribute__((ext_vector_type(VN)));
        constexpr int kLongest = kQ8FewLds / OWN < kQ8FewLongest ? kQ8FewLds / OWN : kQ8FewLongest;
        constexpr int kFewHeld = (kLongest / VN + kFewThreads - 1) / kFewThreads;  // chunks of a token that a thread holds
        VT held[OWN][kFewHeld];
        uint32_t top[OWN];
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const T* x = X.x + (i < M ? i : M - 1) * K;
#pragma unroll
            for (int h = 0; h < kFewHeld; ++h) {
                const int c = h * kFewThreads + threadIdx.x;
                held[i][h] = (VT)(T)0.0f;
                if (X.vec) {
                    if (c * VN < K) held[i][h] = *(const VT*)(x + c * VN);
                } else {
#pragma unroll
                    for (int e = 0; e < VN; ++e)
                        if (c * VN + e < K) held[i][h][e] = x[c * VN + e];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            top[i] = 0;
#pragma unroll
            for (int h = 0; h < kFewHeld; ++h)
#pragma unroll
                for (int e = 0; e < VN; ++e) {
                    const uint32_t t = magnitude(to_f32(held[i][h][e]));
                    top[i] = t > top[i] ? t : top[i];
                }
#pragma unroll
            for (int off = kWave / 2; off > 0; off >>= 1) {
                const uint32_t o = __shfl_xor(top[i], off, kWave);
                top[i] = o > top[i] ? o : top[i];
            }
            if (lane == 0) tops[wv][i] = top[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
#pragma unroll
            for (int u = 0; u < kFewWaves; ++u) top[i] = tops[u][i] > top[i] ? tops[u][i] : top[i];
            float mul, sc;
            row_scale(top[i], &mul, &sc);
            if (m == i) sx = sc;
#pragma unroll
            for (int h = 0; h < kFewHeld; ++h) {
                const int c = h * kFewThreads + threadIdx.x;
                if (c * VN >= stride) continue;
                VQ q;
#pragma unroll
                for (int e = 0; e < VN; ++e) q[e] = (int8_t)quantise(to_f32(held[i][h][e]), mul);
                *(VQ*)(own + i * pitch + c * VN) = q;
            }
        }
        __syncthreads();
    } else {
        sx = X.xs[m];
    }
    for (int turn = 0; n0 < N; ++turn) {
        const int64_t next = n0 + (int64_t)gridDim.x * kFewChannels;
        float wsc[4], bs[4];  // what the end needs
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t n = n0 + kq * 4 + r < N ? n0 + kq * 4 + r : N - 1;
            wsc[r] = ws[n];
            bs[r] = bias ? to_f32(bias[n]) : 0.0f;
        }
        v4i acc = (v4i)0;
        for (int s = s0; s < s1 || s == s0; s += kFewFlight) {
            v4i fx[kFewFlight];
#pragma unroll
            for (int f = 0; f < kFewFlight; ++f) {
                const int k = (s + f < steps ? s + f : steps - 1) * 64 + kq * 16;
                fx[f] = OWN > 0 ? *(const v4i*)(own + m * pitch + k) : *(const v4i*)(X.xq + m * stride + k);
                if (s + f >= s1) fx[f] = (v4i)0;
            }
#pragma unroll
            for (int f = 0; f < kFewFlight; ++f) acc = OpI8::mfma(fw[f], fx[f], acc);
            if (s + kFewFlight < s1) weights(n0, s + kFewFlight);
            else if (next < N) weights(next, s0);
        }
        v4i(*sum)[kWave] = sums[turn & 1];  // (two of them: one barrier a turn)
        sum[wv][lane] = acc;
        __syncthreads();
        if (wv == (turn & (kFewWaves - 1)) && li < M) {
            acc = sum[0][lane];
#pragma unroll
            for (int i = 1; i < kFewWaves; ++i) acc += sum[i][lane];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t n = n0 + kq * 4 + r;
                if (n < N) y[li * N + n] = round_to<T>((float)acc[r] * sx * wsc[r] + bs[r]);
            }
        }
        n0 = next;
    }
}

template <typename T, int OWN>
hipError_t few_t(const FewTokens<T>& X, int64_t M, int64_t K, const int8_t* wq, const float* ws, int64_t N, const void* bias, void* y, hipStream_t st)
{
    const size_t lds = OWN ? few_lds(OWN, M, K) : 0;
    const int64_t groups = cdiv(N, kFewChannels), most = lds > 56 * 1024 ? kFewGroups / 2 : kFewGroups, grid = groups < most ? groups : most;
    if (OWN == kFewTokens) {
        const hipError_t e = hipFuncSetAttribute((const void*)q8_few_kernel<T, OWN>, hipFuncAttributeMaxDynamicSharedMemorySize, kQ8ManyLds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((q8_few_kernel<T, OWN>), dim3((unsigned)grid), dim3(kFewThreads), (unsigned)lds, st, X, (int)M, K, scd_q8_stride(K), wq, ws, N,
                       (const T*)bias, (T*)y);
    return hipGetLastError();
}

typedef Tile<OpI8, 8, 4, 2, 4, true, true, 2> Large;  // 256 x 256
typedef Tile<OpI8, 4, 4, 2, 2, true, true, 2> Middle;  // 128 x 128
typedef Tile<OpI8, 2, 2, 2, 2, true, true, 3> Small;   // 64 x 64
typedef Tile<OpI8, 2, 1, 2, 2, true, true, 4> Narrow;  // 64 x 32

template <typename T>
hipError_t matmul_t(const int8_t* xq, const float* xs, int64_t M, int64_t K, const int8_t* wq, const float* ws, int64_t N, const void* bias, void* y,
                    hipStream_t st)
{
    switch (q8_form(M, K, N)) {
        case Q8Form::few: return few_t<T, 0>(FewTokens<T>{xq, xs, nullptr, false}, M, K, wq, ws, N, bias, y, st);
        case Q8Form::narrow: return tile_t<T, Narrow>(xq, xs, M, K, wq, ws, N, bias, y, st);
        case Q8Form::t256: return tile_t<T, Large>(xq, xs, M, K, wq, ws, N, bias, y, st);
        case Q8Form::t128: return tile_t<T, Middle>(xq, xs, M, K, wq, ws, N, bias, y, st);
        default: return tile_t<T, Small>(xq, xs, M, K, wq, ws, N, bias, y, st);
    }
}

bool product_ok(int dt, int64_t M, int64_t K, const void* wq, const void* ws, int64_t N)
{
    return real_ok(dt) && rows_ok(M) && K >= 1 && K <= SCD_Q8_MAX_K && dim_ok(N) && wq && ws && aligned16(wq);
}

}  // namespace
}  // namespace lm
}  // namespace scd

using namespace scd::lm;

extern "C" {

int64_t scd_q8_stride(int64_t K) { return K < 1 || K > SCD_Q8_MAX_K ? 0 : q8_stride(K); }

int scd_q8_rows(const void* X, scd_real dt, int64_t M, int64_t K, int8_t* q, float* s, void* stream)
{
    if (!real_ok(dt) || !rows_ok(M) || K < 1 || K > SCD_Q8_MAX_K || (M > 0 && (!X || !q || !s || !aligned16(q)))) return SCD_EINVAL;
    if (M == 0) return SCD_OK;
    const hipError_t e = rows(X, dt, M, K, q, s, (hipStream_t)stream);
    return e == hipSuccess ? SCD_OK : scd::report_hip(e);
}

int scd_q8_matmul(const int8_t* xq, const float* xs, int64_t M, int64_t K, const int8_t* wq, const float* ws, int64_t N, const void* bias,
                  scd_real dt, void* y, void* stream)
{
    if (!product_ok(dt, M, K, wq, ws, N) || (M > 0 && (!xq || !xs || !y || !aligned16(xq)))) return SCD_EINVAL;
    if (M == 0) return SCD_OK;
    const hipError_t e = with_real(dt, [&](auto z) { return matmul_t<decltype(z)>(xq, xs, M, K, wq, ws, N, bias, y, (hipStream_t)stream); });
    return e == hipSuccess ? SCD_OK : scd::report_hip(e);
}

size_t scd_q8_linear_workspace_bytes(int64_t M, int64_t K)
{
    if (!rows_ok(M) || K < 1 || K > SCD_Q8_MAX_K) return 0;
    return M <= 2 && q8_few_owns(M, K) ? 0 : up((size_t)M * (size_t)scd_q8_stride(K), 256) + up((size_t)M * 4, 256);
}

int scd_q8_linear(const void* X, scd_real dt, int64_t M, int64_t K, const int8_t* wq, const float* ws, int64_t N, const void* bias, void* y,
                  void* workspace, size_t workspace_bytes, void* stream)
{
    if (!product_ok(dt, M, K, wq, ws, N) || (M > 0 && (!X || !y))) return SCD_EINVAL;
    const size_t need = scd_q8_linear_workspace_bytes(M, K);
    if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return SCD_EINVAL;
    if (M == 0) return SCD_OK;
    int8_t* xq = (int8_t*)workspace;
    float* xs = (float*)((char*)workspace + up((size_t)M * (size_t)scd_q8_stride(K), 256));
    hipStream_t st = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    if (const int own = q8_few_takes(M, K, N) ? q8_few_owns(M, K) : 0) {
        e = with_real(dt, [&](auto z) {
            typedef decltype(z) T;
            const FewTokens<T> x{nullptr, nullptr, (const T*)X, aligned16(X) && K * sizeof(T) % 16 == 0};
            return own == 1 ? few_t<T, 1>(x, M, K, wq, ws, N, bias, y, st) : own == 2 ? few_t<T, 2>(x, M, K, wq, ws, N, bias, y, st)
                   : own == 4                                                         ? few_t<T, 4>(x, M, K, wq, ws, N, bias, y, st)
                                                                                      : few_t<T, kFewTokens>(x, M, K, wq, ws, N, bias, y, st);
        });
        return e == hipSuccess ? SCD_OK : scd::report_hip(e);
    }
    e = rows(X, dt, M, K, xq, xs, st);
    if (e == hipSuccess) e = with_real(dt, [&](auto z) { return matmul_t<decltype(z)>(xq, xs, M, K, wq, ws, N, bias, y, st); });
    return e == hipSuccess ? SCD_OK : scd::report_hip(e);
}

}  // extern "C"
