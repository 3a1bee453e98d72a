// The tile of a matrix product that scd_q8.hip and scd_xent.hip share: C[a][b] = sum_k A[a][k] B[b][k] over 16-bit floats or
// 8-bit integers or f32, TA x TB of it by a workgroup of WA x WB waves.
//
// What bounds it is feeding the matrix cores.  A step is 128 bytes along k of rows of A and B, or as many rows along
// k of arrays that lie the other way.  Steps come straight from memory into LDS (buffer loads with the LDS bit, 16 bytes a lane, nothing
// passes through registers) into a ring of NS buffers, NS - 1 to NS steps ahead of their use; what lies beyond an array reads
// as zero by the buffer's own range check, so that no product has a special tail.  A step is two halves of 64 bytes: while the
// matrix cores work on one half's operands, which are in registers, the other half's are read from LDS.  One barrier a step:
// behind it every wave has read the last of the current buffer, so it can be filled again, and every wave's share of the next
// one has arrived.
//
// LDS rows are 128 bytes (or 2 TA bytes, along a), 16-byte chunks permuted by an exclusive or with bits of the row so that
// the lanes of a read fall on different banks.  Operands along k are read with ds_read_b128; the others are transposed on the
// way into the registers (ds_read_b64_tr_b16; f32 value by value).
//
// f32 on the bf16 instruction (OpSplit): an operand x is taken apart in registers into three bf16, h = bf16(x), m = bf16(x - h),
// l = bf16(x - h - m), which leave less than 2^-24 |x| of it.  Of the nine products of two such operands the six largest are summed,
// hh hm mh hl lh mm; what is left out is below 2^-23 of the product.  Six products at the bf16 rate are 2.6 times as fast as the f32
// instruction (OpF32), and a step's f32 values are what one bf16 instruction multiplies.  198 TFLOP/s of f32 at 4096 x 4096 x 32000, 1.2
// PFLOP/s of bf16, near what a large product reaches on this card; tiles of 64 are bound by the 5.5 vector instructions that taking a
// value apart takes.  (Parts made beforehand, in memory, took 12 % less in the gradients there, loss included, 19.2 ms for 21.7, but a copy of
// both operands in one and a half times their size, which cost small products up to half of their time.)
//
// Two planes (P = 2): B is held in two parts of a 16-bit type, A in one.
//
// A lane's accumulators: column (B) 16 b + lane mod 16; rows (A): for operands along k the rows that a fragment holds are
// chosen so that a lane ends with 4 FA rows that follow one another, which makes whole 16-byte stores; else four and four.
#pragma once
#include <type_traits>

#include "scd_lm_device.h"

namespace scd {
namespace lm {

typedef __attribute__((address_space(3))) char LdsChar;

// An operand in memory: rows of `bytes` valid bytes (a multiple of 16), `pitch` bytes apart, 16-byte aligned.  plane: bytes from
// a row's first plane to its second, where it is held in two.
struct TileRows {
    const char* p;
    int64_t pitch, rows, bytes, plane = 0;
};

struct OpBf16 {
    typedef __bf16 In __attribute__((ext_vector_type(8)));
    typedef v4f Acc;
    static __device__ __forceinline__ Acc mfma(v4i a, v4i b, Acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(In, a), __builtin_bit_cast(In, b), c, 0, 0, 0);
    }
};
struct OpF16 {
    typedef _Float16 In __attribute__((ext_vector_type(8)));
    typedef v4f Acc;
    static __device__ __forceinline__ Acc mfma(v4i a, v4i b, Acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(In, a), __builtin_bit_cast(In, b), c, 0, 0, 0);
    }
};
struct OpI8 {
    typedef v4i Acc;
    static __device__ __forceinline__ Acc mfma(v4i a, v4i b, Acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};

// Four products of the f32 instruction: register j of a lane's 16 bytes is term 4 (lane / 16) + j.
struct OpF32 {
    typedef v4f Acc;
    static __device__ __forceinline__ Acc mfma(v4i a, v4i b, Acc c)
    {
        const v4f x = __builtin_bit_cast(v4f, a), y = __builtin_bit_cast(v4f, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
        return c;
    }
};

// f32 in three parts of bf16.
struct OpSplit {
    typedef v4f Acc;
    typedef __bf16 In __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ void split(v4i lo, v4i hi, In (&part)[3])
    {
        typedef float v2f __attribute__((ext_vector_type(2)));
        typedef __bf16 v2b __attribute__((ext_vector_type(2)));
        v4i out[3];
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // two values at a time: one instruction rounds both
            const v4i from = i < 2 ? lo : hi;
            v2f x = {__int_as_float(from[i * 2 % 4]), __int_as_float(from[i * 2 % 4 + 1])};
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                const uint32_t u = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, v2b));
                out[p][i] = (int)u;
                x[0] -= __uint_as_float(u << 16);
                x[1] -= __uint_as_float(u & 0xFFFF0000u);
            }
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) part[p] = __builtin_bit_cast(In, out[p]);
    }
};

// One operand's side of the tile, of PLANES planes of values of ES bytes: F fragments of 16 a wave, W waves across, T = 16 F W rows;
// WAVES waves in all.  ALONG: rows of memory run along k.  BLOCKED: the rows of a wave are dealt to its fragments four at a time, a block of 4 F for each
// quarter of the lanes.
template <int ES, int F, int W, int WAVES, bool ALONG, bool BLOCKED, int PLANES>
struct TileSide {
    static constexpr int T = 16 * F * W, kBytes = T * kTileStep;
    static constexpr int kRows = kTileStep / ES, kRow = ES * T;  // not ALONG: rows along k of a step, and bytes of one
    static constexpr int kLoads = kBytes / (WAVES * 1024);  // of a thread and step
    static_assert(kLoads * WAVES * 1024 == kBytes, "every wave loads whole KiB");
    static_assert(ALONG || T >= 64, "the swizzle needs four units of 16 columns");

    // ---- memory to LDS
    v4i rsrc;
    const char* base;
    int64_t pitch, left;  // not ALONG: bytes from base to the end of the array
    int voff[2], col[2], row_bytes;
    int jstep;

    static __device__ __forceinline__ int key(int row)
    {
        return BLOCKED ? (row & 3) | ((row / (4 * F)) & 1) << 2 : row & 7;
    }

    __device__ __forceinline__ void make_rsrc(const char* p, int64_t n)
    {
        const uint64_t u = (uint64_t)p;
        rsrc[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)u);
        rsrc[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32) & 0xFFFF);
        rsrc[2] = __builtin_amdgcn_readfirstlane((int)(n < 0 ? 0 : n > 0x7FFFFFFF ? 0x7FFFFFFF : n));
        rsrc[3] = 0x00027000;
    }

    // `first`: the tile's first row (ALONG) or column.
    __device__ __forceinline__ void init(const TileRows& m, int64_t first, int wv, int lane)
    {
        pitch = m.pitch;
        row_bytes = (int)m.bytes;
        if constexpr (ALONG) {
            const int64_t rows = m.rows - first < T ? m.rows - first : T;
            base = m.p + first * pitch;
            make_rsrc(base, rows < 1 ? 0 : (rows - 1) * pitch + (PLANES - 1) * m.plane + m.bytes);  // (below 256 * kTileMaxPitch)
#pragma unroll
            for (int par = 0; par < 2; ++par) {
                const int row = (par * WAVES + wv) * 8 + (lane >> 3);
                col[par] = ((lane & 7) ^ key(row)) * 16;
                voff[par] = (int)((wv * 8 + (lane >> 3)) * pitch) + col[par];
            }
            jstep = __builtin_amdgcn_readfirstlane((int)(8 * WAVES * pitch));
        } else {
            base = m.p + first * ES;
            left = (m.rows - 1) * pitch + (PLANES - 1) * m.plane + m.bytes - first * ES;
            constexpr int per = WAVES * 1024 / kRow;  // rows of k that the workgroup loads at once
            const int at = wv * 1024 + lane * 16, k = at / kRow, slot = (at % kRow) / 16;
#pragma unroll
            for (int par = 0; par < 2; ++par) voff[par] = (int)(k * pitch) + ((slot / ES ^ unit_key(k + par * per)) * ES + slot % ES) * 16;
            jstep = __builtin_amdgcn_readfirstlane((int)(per * pitch));
        }
    }

    // Loads of step s: aim, then issue each of kLoads into the buffer at LDS address `lds`; beyond the last step they read zeros.
    // The whole offset is the lane's own, so that the range check sees all of it; 2^31 and more lies beyond any range given here.
    uint32_t v[2];

    __device__ __forceinline__ void aim(int s, int steps, int plane)
    {
        v[0] = (uint32_t)voff[0], v[1] = (uint32_t)voff[1];
        if constexpr (ALONG) {
            const int along = s < steps ? s * kTileStep : row_bytes;
#pragma unroll
            for (int par = 0; par < 2; ++par) v[par] = along + col[par] < row_bytes ? v[par] + along + plane : 0x80000000u;
        } else {
            const int64_t at = (int64_t)s * kRows * pitch + plane;
            make_rsrc(base + at, left - at);
            if (s >= steps) v[0] = v[1] = 0x80000000u;
        }
    }

    __device__ __forceinline__ void issue(int j, uint32_t lds, int wv) const
    {
        const uint32_t to = lds + (j * WAVES + wv) * 1024;
        // (the compiler writes M0; a load with the LDS bit comes one wait state behind that at the earliest)
        asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(to), "v"(v[j & 1] + j * jstep), "s"(rsrc) : "memory");
    }

    // ---- LDS to registers
    // Exclusive or of the units of 16 columns in row k: the rows that lanes read together.
    static __device__ __forceinline__ int unit_key(int k) { return ES == 4 ? (k >> 2) & 3 : ((k & 3) | ((k >> 3) & 1) << 2) & (T / 16 - 1); }

    // Byte address in a buffer of this lane's part of fragment f, half h: along k one 16-byte read; else two 8-byte reads, 4 rows
    // apart (ES 2), or four values, a row apart (ES 4).
    int at[ALONG ? 2 : F];

    __device__ __forceinline__ void init_reads(int side, int lane)
    {
        const int li = lane & 15, kq = lane >> 4;
        if constexpr (ALONG) {
            const int row = side * 16 * F + (BLOCKED ? (li >> 2) * 4 * F + (li & 3) : li);
#pragma unroll
            for (int h = 0; h < 2; ++h) at[h] = row * kTileStep + ((h * 4 + kq) ^ key(row)) * 16;
        } else {
            const int k = ES == 4 ? kq * 4 : kq * 8 + (li >> 2);
#pragma unroll
            for (int f = 0; f < F; ++f) at[f] = k * kRow + ((side * F + f) ^ unit_key(k)) * 16 * ES + (ES == 4 ? li * 4 : (li & 3) * 8);
        }
    }

    __device__ __forceinline__ v4i read(const LdsChar* buf, int f, int h) const
    {
        if constexpr (ALONG) {
            return *(const __attribute__((address_space(3))) v4i*)(buf + at[h] + f * (BLOCKED ? 4 : 16) * kTileStep);
        } else if constexpr (ES == 4) {
            v4i x;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = *(const __attribute__((address_space(3))) int*)(buf + at[f] + (h * 16 + j) * kRow);
            return x;
        } else {
            typedef short v4s __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) v4s LdsV4s;
            LdsChar* p = (LdsChar*)buf + at[f] + h * 32 * kRow;
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsV4s*)p);
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsV4s*)(p + 4 * kRow));
            typedef short v8s __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(v4i, (v8s)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }

    // Row of the tile that register 0 of fragment f holds in this lane (A: rows), and the column (B).
    static __device__ __forceinline__ int row_of(int side, int f, int lane)
    {
        return side * 16 * F + (BLOCKED ? (lane >> 4) * 4 * F + f * 4 : f * 16 + (lane >> 4) * 4);
    }
    static __device__ __forceinline__ int col_of(int side, int f, int lane) { return side * 16 * F + f * 16 + (lane & 15); }
};

// All but this wave's last N loads have arrived, and every wave is here.
template <int N>
__device__ __forceinline__ void arrive()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <class Op_, int FA_, int FB_, int WA_, int WB_, bool A_ALONG, bool B_ALONG, int NS, int P = 1>
struct Tile {
    typedef Op_ Op;
    static constexpr int ES = std::is_same<Op, OpF32>::value || std::is_same<Op, OpSplit>::value ? 4 : std::is_same<Op, OpI8>::value ? 1 : 2;
    static_assert(ES > 1 || (A_ALONG && B_ALONG), "8-bit rows run along k");
    static constexpr int kRows = kTileStep / ES;  // terms of a step
    static constexpr bool kSplit = std::is_same<Op, OpSplit>::value;
    static constexpr int FA = FA_, FB = FB_, WA = WA_, WB = WB_;
    static constexpr int kThreads = WA * WB * kWave;
    typedef TileSide<ES, FA, WA, WA * WB, A_ALONG, A_ALONG, 1> SideA;
    typedef TileSide<ES, FB, WB, WA * WB, B_ALONG, false, P> SideB;
    static constexpr int TA = SideA::T, TB = SideB::T;
    static constexpr int kBuffer = SideA::kBytes + SideB::kBytes, kLds = kBuffer * NS;
    static constexpr int kLoads = SideA::kLoads + SideB::kLoads;
    typedef typename Op::Acc Acc;

    // All waves call it; `steps` (of a plane) is the same in all of them.  Leaves the LDS free for other use.  The steps are taken round from
    // `begin` (below `steps`): rows that lie a power of two apart would else be read at the same few memory channels by all
    // workgroups at once, where these do not share rows.
    static __device__ __forceinline__ void run(const TileRows& A, const TileRows& B, int64_t a0, int64_t b0, int64_t steps_, char* lds_, Acc (&acc)[FA][FB],
                                               int64_t begin_ = 0)
    {
        const int steps = (int)steps_, begin = (int)begin_;  // (rows of kTileMaxPitch bytes, and 2^31 rows in steps of 32 and more)
        const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        LdsChar* lds = (LdsChar*)lds_;
        const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
        SideA sa;
        SideB sb;
        sa.init(A, a0, wv, lane);
        sb.init(B, b0, wv, lane);
        sa.init_reads(wv / WB, lane);
        sb.init_reads(wv % WB, lane);
#pragma unroll
        for (int a = 0; a < FA; ++a)
#pragma unroll
            for (int b = 0; b < FB; ++b) acc[a][b] = (Acc)0;
        if (steps <= 0) return;
        const int all = steps * P;
        auto aim = [&](int t) {
            int s = P > 1 ? (int)((uint32_t)t / P) : t;
            const int plane = P > 1 ? t - s * P : 0;
            if (t < all) s = s + begin < steps ? s + begin : s + begin - steps;
            sa.aim(s, steps, 0);
            sb.aim(s, steps, plane * (int)B.plane);
        };
        auto issue = [&](int j, int slot) {
            if (j < SideA::kLoads) sa.issue(j, lds0 + slot * kBuffer, wv);
            else sb.issue(j - SideA::kLoads, lds0 + slot * kBuffer + SideA::kBytes, wv);
        };
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            aim(s);
#pragma unroll
            for (int j = 0; j < kLoads; ++j) issue(j, s);
        }
        arrive<(NS - 1) * kLoads>();
        if constexpr (kSplit) {
            split_steps(sa, sb, lds, all, aim, issue, acc);
            if constexpr (A_ALONG && B_ALONG) mend(A, B, a0, b0, acc);
        } else {
            whole_steps(sa, sb, lds, all, aim, issue, acc);
        }
    }

    // The steps with operands as they are.
    template <typename Aim, typename Issue>
    static __device__ __forceinline__ void whole_steps(const SideA& sa, const SideB& sb, const LdsChar* lds, int all, Aim& aim, Issue& issue, Acc (&acc)[FA][FB])
    {
        v4i fa[2][FA], fb[2][FB];
        // Fragment i of FB + FA of half h.
        auto read = [&](int slot, int h, int i) {
            const LdsChar* buf = lds + slot * kBuffer;
            if (i < FB) fb[h][i] = sb.read(buf + SideA::kBytes, i, h);
            else fa[h][i - FB] = sa.read(buf, i - FB, h);
        };
        // The products of half h, a row of fragments after the other, and before each row its share of what else there is to issue:
        // the other half's reads and, in the second half, the loads.  Issued all at once these would hold up the products behind them.
        auto multiply = [&](auto half, int from, int into) {
            constexpr int h = decltype(half)::value;
#pragma unroll
            for (int a = 0; a < FA; ++a) {
#pragma unroll
                for (int j = 0; j < kLoads; ++j)
                    if (h == 1 && j * FA / kLoads == a) issue(j, into);
#pragma unroll
                for (int i = 0; i < FA + FB; ++i)
                    if (i * FA / (FA + FB) == a) read(from, 1 - h, i);
#pragma unroll
                for (int b = 0; b < FB; ++b) acc[a][b] = Op::mfma(fa[h][a], fb[h][b], acc[a][b]);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
#pragma unroll
        for (int i = 0; i < FA + FB; ++i) read(0, 0, i);
        int slot = 0;
        for (int s = 0; s < all; ++s) {
            multiply(std::integral_constant<int, 0>{}, slot, 0);
            arrive<(NS - 2) * kLoads>();
            aim(s + NS);
            const int next = slot + 1 == NS ? 0 : slot + 1;
            multiply(std::integral_constant<int, 1>{}, next, slot);
            slot = next;
        }
        arrive<0>();
    }

    // The steps with operands taken apart: behind a step's barrier its values are in registers, and as each is taken apart the next
    // step's takes its place.
    template <typename Aim, typename Issue>
    static __device__ __forceinline__ void split_steps(const SideA& sa, const SideB& sb, const LdsChar* lds, int all, Aim& aim, Issue& issue, Acc (&acc)[FA][FB])
    {
        typedef OpSplit::In In;
        v4i ra[FA][2], rb[FB][2];
        auto read_a = [&](int slot, int a) {
#pragma unroll
            for (int h = 0; h < 2; ++h) ra[a][h] = sa.read(lds + slot * kBuffer, a, h);
        };
        auto read_b = [&](int slot, int b) {
#pragma unroll
            for (int h = 0; h < 2; ++h) rb[b][h] = sb.read(lds + slot * kBuffer + SideA::kBytes, b, h);
        };
#pragma unroll
        for (int a = 0; a < FA; ++a) read_a(0, a);
#pragma unroll
        for (int b = 0; b < FB; ++b) read_b(0, b);
        int slot = 0;
        for (int s = 0; s < all; ++s) {
            arrive<(NS - 2) * kLoads>();
            aim(s + NS);
            const int next = slot + 1 == NS ? 0 : slot + 1;
            In pb[FB][3];
#pragma unroll
            for (int b = 0; b < FB; ++b) {
                OpSplit::split(rb[b][0], rb[b][1], pb[b]);
                read_b(next, b);
            }
#pragma unroll
            for (int a = 0; a < FA; ++a) {
#pragma unroll
                for (int j = 0; j < kLoads; ++j)
                    if (j * FA / kLoads == a) issue(j, slot);
                In pa[3];
                OpSplit::split(ra[a][0], ra[a][1], pa);
                read_a(next, a);
                constexpr int kA[6] = {2, 1, 0, 1, 0, 0}, kB[6] = {0, 1, 2, 0, 1, 0};  // small ones first
#pragma unroll
                for (int p = 0; p < 6; ++p)
#pragma unroll
                    for (int b = 0; b < FB; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa[kA[p]], pb[b][kB[p]], acc[a][b], 0, 0, 0);
            }
            slot = next;
        }
        arrive<0>();
    }

    // Taken apart, an infinity (and what rounds to one as bf16) meets others' zero parts and gives NaN.  So a result that comes out as
    // NaN is summed again here, value by value, until it is NaN for good.  (Logits; where the sums run across rows, as in gradients, one
    // NaN among the terms makes all of an array's results NaN, and looking for it in each would take seconds.  512 tokens, 32000 x 4096 with
    // the weights' last column NaN, the longest way to it: 39 ms.)
    static __device__ __forceinline__ void mend(const TileRows& A, const TileRows& B, int64_t a0, int64_t b0, Acc (&acc)[FA][FB])
    {
        const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int64_t chunks = A.bytes / 16;
#pragma unroll
        for (int b = 0; b < FB; ++b) {
            const int64_t col = b0 + SideB::col_of(wv % WB, b, lane);
            uint32_t bad = 0;
#pragma unroll
            for (int i = 0; i < 4 * FA; ++i) bad |= acc[i / 4][b][i % 4] != acc[i / 4][b][i % 4] ? 1u << i : 0u;
            while (bad) {
                const int i = __ffs(bad) - 1;
                bad &= bad - 1;
                const int64_t row = a0 + SideA::row_of(wv / WB, i / 4, lane) + i % 4;
                if (row >= A.rows || col >= B.rows) continue;
                const v4f *x = (const v4f*)(A.p + row * A.pitch), *y = (const v4f*)(B.p + col * B.pitch);
                float sum = 0.0f;
                for (int64_t k = 0; k < chunks && sum == sum; ++k) {
                    const v4f p = x[k] * y[k];
                    sum += (p[0] + p[1]) + (p[2] + p[3]);
                }
#pragma unroll
                for (int e = 0; e < 4 * FA; ++e) acc[e / 4][b][e % 4] = e == i ? sum : acc[e / 4][b][e % 4];
            }
        }
    }
};

constexpr int64_t kTileGroup = 4;

// Tiles in the order that keeps each XCD (every eighth workgroup) on neighbouring tiles: its share of the tiles is one stretch
// of an order that walks `group` tiles along b before the next along a.
__device__ __forceinline__ void tile_order(int64_t index, int64_t na, int64_t nb, int64_t group, int64_t* ta, int64_t* tb)
{
    const int64_t all = na * nb, share = all / 8, more = all % 8, xcd = index % 8, i = index / 8;
    const int64_t t = xcd * share + (xcd < more ? xcd : more) + i;
    const int64_t strip = t / (group * na), first = strip * group;
    const int64_t width = nb - first < group ? nb - first : group, r = t - strip * group * na;
    *ta = r / width;
    *tb = first + r % width;
}

// Where tile ta of na begins its steps if it has its rows of A to itself (one tile holds all of b): spread evenly.
template <class Q>
__device__ __forceinline__ int64_t alone_begin(int64_t ta, int64_t a, int64_t b, int64_t steps)
{
    return b <= Q::TB ? ta * steps / cdiv(a, Q::TA) : 0;
}

}  // namespace lm
}  // namespace scd
