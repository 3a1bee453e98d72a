// Which form of the operators of scd_lm.h takes a call: rules on sizes, host arithmetic only.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "scd_lm.h"

namespace scd {
namespace lm {

constexpr size_t up(size_t x, size_t unit) { return (x + unit - 1) / unit * unit; }
constexpr int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ------------------------------------------------------------------------------------------------ the product tile

constexpr int kTileStep = 128;  // bytes along k of a step
constexpr int64_t kTileMaxPitch = (int64_t)1 << 22;  // 256 rows of it keep a 32-bit offset

// Which of the square tiles of 256, 128 and 64 a product of na x nb entries takes: the one that the compute
// units are done with first, each with its share of the tiles one after the other.  A smaller tile takes more time for its
// entries (less is multiplied between two reads), relative to that of 256: rate128, rate64; largest: 128 leaves out that of 256.
inline int pick_tile(int64_t na, int64_t nb, double rate128, double rate64, int largest = 256)
{
    int best = 0;
    double least = 0;
    for (int t = largest; t >= 64; t /= 2) {
        const double turns = (double)cdiv(cdiv(na, t) * cdiv(nb, t), 256), cost = turns * t * t / (t == 256 ? 1.0 : t == 128 ? rate128 : rate64);
        if (best == 0 || cost < least) best = t, least = cost;
    }
    return best;
}

// ------------------------------------------------------------------------------------------------ products in 8-bit integers

constexpr int64_t q8_stride(int64_t K) { return cdiv(K, 128) * 128; }

constexpr int kQ8FewTokens = 16;  // one column block of the matrix cores
constexpr int kQ8FewPad = 64;     // bytes between the tokens' rows in LDS
constexpr int kQ8FewLds = 48 * 1024;    // for the rows of up to four tokens, which all threads round together
constexpr int kQ8FewLongest = 16384;    // bytes of a row there, at most
constexpr int kQ8ManyLds = 112 * 1024;  // for the rows of more, which the waves round one by one

// How the workgroups put the tokens into 8 bits themselves: 1, 2 or 4: all threads, so many tokens at once; kQ8FewTokens: a token a
// wave; 0: not at all.
inline int q8_few_owns(int64_t M, int64_t K)
{
    const int64_t row = q8_stride(K) + kQ8FewPad;
    const int together = M <= 1 ? 1 : M == 2 ? 2 : 4;
    if (M <= 4 && row <= kQ8FewLongest + kQ8FewPad && together * row <= kQ8FewLds) return together;
    return M <= kQ8FewTokens && M * row <= kQ8ManyLds ? kQ8FewTokens : 0;
}

// Whether q8_few_kernel takes so many tokens at all.  It has the least latency and reads long rows by many waves each; its channels come in
// turns of 8192, which cost 4 us each however short the rows, and from three tokens on putting them into 8 bits is on its way, too.  The
// tile takes 5 us and the larger of 2.1 us for 1000 entries of a row and reading the weights at 5.6 TB/s.  Measured, us, here / tile, weights from
// memory (bf16; K -> N at 3, 8 and 16 tokens):
//     1024 ->  4096    7.9 /  7.7    7.2 /  7.9    9.2 /  8.0       8192 ->  4096   14.0 / 22.3   17.4 / 22.4   16.0 / 22.7
//     1024 ->  6144   11.1 /  8.5   10.4 /  8.7   13.1 /  8.8       8192 ->  8192   19.4 / 23.2   23.0 / 23.5   24.6 / 23.8
//     4096 ->  1024    8.3 / 12.3    8.3 / 12.6   11.4 / 12.6       8192 -> 14336   27.5 / 26.8   32.9 / 26.9   40.0 / 27.2
//     4096 ->  4096   10.1 / 14.1   10.0 / 14.4   13.4 / 14.5      14336 ->  4096   26.5 / 34.6   22.1 / 34.9   24.9 / 35.3
//     4096 ->  7168   13.7 / 14.6   14.4 / 14.8   16.7 / 15.1      14336 ->  6144   33.8 / 36.0   33.7 / 36.2   39.1 / 36.9
//     4096 ->  8192   14.2 / 14.8   15.1 / 14.9   17.2 / 15.3      14336 ->  8192   36.4 / 37.5   35.3 / 37.8   40.6 / 38.5
//     4096 -> 14336   17.5 / 16.8   18.9 / 16.8   23.7 / 17.0      14336 -> 14336   54.5 / 43.8   60.1 / 44.1   71.3 / 44.5
//     2048 ->  8192   11.4 / 10.6   11.5 / 10.8   15.0 / 10.9      32768 ->  4096   62.2 / 69.6   50.5 / 69.8   53.4 / 70.8
// One or two tokens stay here always, since they need no work space (mostly faster too: 4096 -> 4096 7.6 / 14.0, 14336 -> 14336 42.6 / 43.7; slower
// where short rows are many: 2048 -> 64000 40 / 28).
inline bool q8_few_takes(int64_t M, int64_t K, int64_t N)
{
    return M <= 2 || (M <= kQ8FewTokens && N < 8192 && (N <= 4096 || K > 2048));
}

enum class Q8Form { few, narrow, t256, t128, t64 };  // narrow: tiles of 64 channels and 32 tokens
inline Q8Form q8_form(int64_t M, int64_t K, int64_t N)
{
    if (q8_few_takes(M, K, N)) return Q8Form::few;
    if (M <= 64) return Q8Form::narrow;
    const int t = pick_tile(N, M, 0.8, 0.45);
    return t == 256 ? Q8Form::t256 : t == 128 ? Q8Form::t128 : Q8Form::t64;
}

// ------------------------------------------------------------------------------------------------ cross entropy

constexpr size_t kPieceBytes = (size_t)128 << 20;  // dz of a piece in 16 bits, at most (or of 256 rows)
constexpr int64_t kTwiceTokens = 64;               // 16-bit types: up to so many tokens, which are bound by memory, dz has twice the
                                                   // type's digits, so that a gradient is not off by two roundings of one number
constexpr size_t kCopyBytes = (size_t)1 << 30;     // the copy of a piece of W, at most (or of 256 rows)
// dW of few tokens from so many bytes on pays for a launch of its own: alone, and beside dX, whose launch it would else share (bf16,
// 30 tokens, 20000 x 1024: 33 -> 26 us alone, 48 -> 48 with dX; 2 tokens, 32000 x 4096: 171 -> 103, 217 -> 152).
// (f32: one limit for both, since the f32 instruction gives other bits than the tile's.)
constexpr int64_t kFewBytes = (int64_t)16 << 20, kFewBesideBytes = (int64_t)128 << 20;
constexpr int64_t kLeastShare = 8;    // steps

// How the tile takes a call of these sizes; the same for the forward and for the gradients.
struct Shape {
    int64_t N, D, V;
    bool f32, split;    // split: f32 on the bf16 instruction
    int64_t ld;         // entries of a row of the copies
    int bytes;          // of an entry
    int dz_planes, dz_bytes;

    bool copies_w;      // W is copied a piece at a time (X always is for the gradients)
    int64_t piece;      // vocabulary rows of a piece
    int grads;          // the gradients' tile: 256, 128 or 64, or 0 for the tiles of few tokens
    int splits;         // shares of the vocabulary that dX is summed in
    int w_splits;       // shares of the tokens that dW is summed in
    int z_splits;       // shares of the dims that the logits are summed in
};

// Whether products of `rows` rows with so many tokens take all tokens in one tile, of 128 rows.
inline bool takes_few(int64_t N, int64_t rows) { return N <= 64 && rows > 2048; }

inline int64_t whole_rows(size_t bytes, size_t bytes_a_row, int64_t V)
{
    int64_t rows = (int64_t)(bytes / bytes_a_row) / 256 * 256;
    if (rows < 256) rows = 256;
    return rows < V ? rows : V;
}

// The gradients' tile and the shares that dX is summed in along the vocabulary and dW along the tokens.
//
// Few tokens: as many shares of dX as give every compute unit two tiles, of 8 steps at least.  Else both products are one launch, tiles
// of dX first: it ends, in us, with these or with the work of all on all compute units and half a tile of dW, a step taking about what is
// measured of it.  Shares are three quarters of that work at most, and cost a launch and their sums' way
// through memory.  (4000 tokens, 4096 x 200, where dW is few tiles and long: f32 490 us without shares, 115 with them.)
inline void choose_grads(Shape& s, int64_t room)
{
    const int64_t N = s.N, D = s.D, K = s.piece, row = s.f32 ? 32 : 64;  // entries along k of a step
    s.splits = s.w_splits = 1;
    s.grads = 64;
    if (N <= 0) return;
    const int64_t x_room = room / (N * s.ld), w_room = K == s.V ? room / (K * s.ld) : 1;
    auto within = [](int64_t k, int64_t most, int64_t also) {
        k = k < most ? k : most;
        k = k < also ? k : also;
        return k < 1 ? 1 : k;
    };
    if (takes_few(N, D)) {
        s.grads = 0;
        s.splits = (int)within(512 / cdiv(D, 128), cdiv(K, 64 * kLeastShare), x_room);
        return;
    }
    const int64_t kx = cdiv(K, row), kw = cdiv(N, row);
    double best = 0;
    for (int t = row == 32 || s.dz_planes == 2 ? 128 : 256; t >= 64; t /= 2) {
        const double step = s.split ? (t == 128 ? 0.9 : 0.35) : s.f32 ? (t == 128 ? 1.75 : 0.48) : (t == 256 ? 1.6 : t == 128 ? 0.5 : 0.24) * s.dz_planes;
        const int64_t nx = cdiv(D, t) * cdiv(N, t), nw = cdiv(D, t) * cdiv(K, t), each = cdiv(nx * kx + nw * kw, 256);
        const int64_t aim = each * 3 / 4 > kLeastShare ? each * 3 / 4 : kLeastShare;
        const int64_t sx = within(cdiv(kx, aim), kx / kLeastShare, x_room), sw = within(cdiv(kw, aim), kw / kLeastShare, w_room);
        for (int shared = 0; shared < 2; ++shared) {
            if (shared && sx == 1 && sw == 1) break;
            const int64_t x = shared ? cdiv(kx, sx) : kx, w = shared ? cdiv(kw, sw) : kw, both = each + w / 2;
            const int64_t sums = shared ? (sx > 1 ? sx * N : 0) + (sw > 1 ? sw * K : 0) : 0;
            const double cost = (double)(x > both ? x : both) * step + (shared ? 4.0 + 2e-6 * (double)(sums * s.ld) : 0.0);
            if (best == 0 || cost < best) best = cost, s.grads = t, s.splits = shared ? (int)sx : 1, s.w_splits = shared ? (int)sw : 1;
        }
    }
}

// Shares of the dims for the logits: where a tile a compute unit leaves units without one, and long sums in the others, these take as
// many shares as end first, in us: whole turns of a tile of 64 (a step takes 0.28 in 16 bits, 0.58 in f32), and with
// shares one more launch and their sums' way through memory.  (40 tokens, 4096 x 200 in f32: gradients 172 us in one, 52 in 16.)
inline int logits_shares_of(const Shape& s, int64_t room)
{
    const int64_t ldz = (int64_t)up((size_t)s.V, 64), tiles = takes_few(s.N, s.V) ? cdiv(s.V, 128) : cdiv(s.V, 64) * cdiv(s.N, 64);
    if (tiles >= 512) return 1;
    const int64_t steps = cdiv(s.ld * s.bytes, kTileStep);
    const double step = s.f32 ? 0.58 : 0.28, sums = 8e-6 * (double)(s.N * ldz) / 4;
    int best = 1;
    double least = 0;
    for (int k = 1; k <= 16 && (k == 1 || (k * kLeastShare <= steps && k <= room / (s.N * ldz))); ++k) {
        const double cost = (double)cdiv(tiles * k, 256) * (double)cdiv(steps, k) * step + (k > 1 ? 5.0 + k * sums : 0.0);
        if (k == 1 || cost < least) best = k, least = cost;
    }
    return best;
}

inline Shape shape_of(int dt, int64_t N, int64_t D, int64_t V)
{
    Shape s;
    s.N = N, s.D = D, s.V = V;
    s.f32 = dt == SCD_REAL_F32;
    s.split = s.f32 && D >= 64 && V >= 64;  // (sums of a few terms keep all of f32 without)
    s.ld = (int64_t)up((size_t)D, 8);
    s.bytes = s.f32 ? 4 : 2;
    s.copies_w = s.ld != D;
    s.dz_planes = !s.f32 && N <= kTwiceTokens ? 2 : 1;
    s.dz_bytes = s.dz_planes == 2 ? 4 : s.bytes;
    s.piece = whole_rows(kPieceBytes * (s.dz_bytes / 2), (size_t)(N > 0 ? N : 1) * s.dz_bytes, V);
    if (s.copies_w) {
        const int64_t w = whole_rows(kCopyBytes, (size_t)s.ld * s.bytes, V);
        s.piece = w < s.piece ? w : s.piece;
    }
    const int64_t room = (int64_t)(kPieceBytes / 4);  // of the sums of shares: no more than a piece
    choose_grads(s, room);
    s.z_splits = N > 0 && s.piece == V ? logits_shares_of(s, room) : 1;
    return s;
}

// Whether dW of a piece of so many rows is made by the workgroups that walk along the vocabulary (tokens: as many as they hold in
// registers).
inline int64_t walk_tokens(const Shape& s) { return s.f32 || s.dz_planes == 2 ? 64 : 128; }
inline bool dw_walks(const Shape& s, int64_t width, bool dX)
{
    return s.N > 0 && s.N <= walk_tokens(s) && width * s.D * s.bytes >= (dX || s.f32 ? kFewBesideBytes : kFewBytes);
}

// The tile of the logits of na vocabulary rows and nb tokens.  256 x 256 keeps the matrix cores fed best, and needs a few hundred of
// them; smaller ones where there are fewer; few tokens take all of them in one tile, deep in flight, and are bound by reading the other
// operand.
enum class LogitsTile { t256, t128, deep128, t64, tokens64, tokens32 };
inline LogitsTile logits_tile(const Shape& s, int64_t na, int64_t nb)
{
    if (takes_few(nb, na)) return nb <= 32 ? LogitsTile::tokens32 : LogitsTile::tokens64;
    // (f32 as it is: its instruction is slow enough to be fed from any tile; taken apart, the parts leave no registers for a tile of 256)
    const int t = s.f32 && !s.split ? pick_tile(na, nb, 1.0, 0.9, 128) : pick_tile(na, nb, 0.8, s.f32 ? 0.5 : 0.45, s.f32 ? 128 : 256);
    // (where a compute unit has one tile at most: its LDS all for that one, steps further ahead; logits of 128 tokens 67 -> 54 us)
    if (t == 128 && cdiv(na, t) * cdiv(nb, t) <= 256) return LogitsTile::deep128;
    return t == 256 ? LogitsTile::t256 : t == 128 ? LogitsTile::t128 : LogitsTile::t64;
}
// Vocabulary rows behind one pair of sums of a token.
inline int64_t strip_rows(LogitsTile t) { return t == LogitsTile::t256 ? 128 : t == LogitsTile::t128 || t == LogitsTile::deep128 ? 64 : 32; }

}  // namespace lm
}  // namespace scd
