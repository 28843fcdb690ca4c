// The forms of the attention over the 8-bit cache (attn8.cu): what a block of each takes of an SM.  Plain C++.
#pragma once

namespace osp {

constexpr int A8_CH = 32;            // tail keys of a step
constexpr int A8_PG = 2048;          // bytes of 16 weight columns of a tile
constexpr int A8_SM = 228 * 1024;    // shared memory of an SM; a block takes 1 KB beside its own
constexpr int A8_OPT = 227 * 1024;   // of one block, at most, 3 KB of static arrays among it

// QT queries a block, QW of them a warpgroup's (4 warps); QP and PP planes of a query and
// of a weight; BPS blocks an SM, of NS slots of K and V each.
template <int HD_, int QT_, int QW_, int QP_, int PP_, int BPS_, int NS_>
struct A8 {
    static constexpr int HD = HD_, QT = QT_, QW = QW_, QP = QP_, PP = PP_, BPS = BPS_, NS = NS_ * 128 / HD;
    static constexpr int NWG = QT / QW, CT = NWG * 128;   // warpgroups that compute, their threads
    static constexpr int THREADS = CT + 96;               // and three warps: products, K copies, V copies
    static constexpr int KB = 16 * HD, TB = 8 * KB;       // bytes of a page, of a tile's slot
    static constexpr int SC = (QP * QT + 15) / 16 * 16, OC = (PP * QT + 15) / 16 * 16;   // TMEM columns of scores, output
    static constexpr int TM = 512 / BPS;                  // columns a block may take
    static constexpr int USED = 2 * SC + OC;               // two tiles' scores, one's output
    static constexpr int COLS = USED <= 32 ? 32 : USED <= 64 ? 64 : USED <= 128 ? 128 : USED <= 256 ? 256 : 512;
    static constexpr int QB = SC * HD;                    // bytes of q's planes
    static constexpr int PW = A8_PG * (OC / 16);          // bytes of the weights' planes
    static constexpr int PB = PW > QT * HD * 4 ? PW : QT * HD * 4;   // their place, q's for the tail
    static constexpr int NEED = 2 * NS * TB + QB + PB + QT * A8_CH * 4;
    // A block waits for its TMEM columns without a limit, and its cluster waits for it: were
    // there more blocks on an SM than its columns serve, of one call or of two, each could
    // hold what the other's cluster waits for.  So a block asks for at least a third of the
    // SM's shared memory, with the SM to itself two thirds: whatever the forms, either two
    // blocks of 256 columns fit or one of 512, and no other beside it.
    static constexpr int SHARE = A8_SM / 3 * (BPS == 2 ? 1 : 2);
    static constexpr int SMEM = NEED > SHARE ? NEED : SHARE;
    static_assert((BPS == 1 || BPS == 2) && SMEM + 3 * 1024 <= A8_OPT, "shares are thirds");
    static_assert((QW == 4 || QW == 8) && COLS <= TM && QB + PB >= KB && QT % QW == 0, "operands");
    static_assert(QT * HD * 4 <= NS * TB, "the merge's outputs take the K slots");
};

// By the queries that a block takes; F: float32 queries, R: rotated bf16 ones.
template <int HD> using A8_4F = A8<HD, 4, 4, 6, 6, 2, 3>;
template <int HD> using A8_8F = A8<HD, 8, 8, 6, 6, 2, 2>;
template <int HD> using A8_4 = A8<HD, 4, 4, 4, 4, 2, 3>;
template <int HD> using A8_8 = A8<HD, 8, 8, 4, 4, 2, 3>;
template <int HD> using A8_16R = A8<HD, 16, 8, 4, 4, 2, 2>;
template <int HD> using A8_16 = A8<HD, 16, 8, 2, 4, 2, 3>;
template <int HD> using A8_32R = A8<HD, 32, 8, 4, 4, 1, 4>;
template <int HD> using A8_32 = A8<HD, 32, 8, 2, 4, 1, 4>;

}  // namespace osp
