// The forms of the attention over the 8-bit cache (attn8.cu): what a block of each takes of an SM.  Plain C++.
#pragma once

namespace osp {

constexpr int A8_CH = 32;            // tail keys of a step
constexpr int A8_PG = 2048;          // bytes of 16 weight columns of a tile
constexpr int A8_SM = 228 * 1024;    // shared memory of an SM,
constexpr int A8_OPT = 227 * 1024;   // of one block at most,
constexpr int A8_OWN = 1024;         // of a block beside what it asks for,
constexpr int A8_STATIC = 3 * 1024;  // of its static arrays, at most

// Columns of an allocation: a power of two, 32 or more.
constexpr int a8_columns(int n) { return n <= 32 ? 32 : 2 * a8_columns((n + 1) / 2); }

// QT queries a block, QW of them a warpgroup's (4 warps); QP and PP planes of a query and
// of a weight; BPS blocks an SM, of NS slots of K and V each.
template <int HD_, int QT_, int QW_, int QP_, int PP_, int BPS_, int NS_>
struct A8 {
    static constexpr int HD = HD_, QT = QT_, QW = QW_, QP = QP_, PP = PP_, BPS = BPS_, NS = NS_ * 128 / HD;
    static constexpr int NWG = QT / QW, CT = NWG * 128;   // warpgroups that compute, their threads
    static constexpr int THREADS = CT + 96;               // and three warps: products, K copies, V copies
    static constexpr int KB = 16 * HD, TB = 8 * KB;       // bytes of a page, of a tile's slot
    static constexpr int SC = (QP * QT + 15) / 16 * 16, OC = (PP * QT + 15) / 16 * 16;   // TMEM columns of scores, output
    // TMEM, in two pieces: two tiles' scores, one's output
    static constexpr int SCOLS = a8_columns(2 * SC), OCOLS = a8_columns(OC);
    static constexpr int QB = SC * HD;                    // bytes of q's planes
    static constexpr int PW = A8_PG * (OC / 16);          // bytes of the weights' planes
    static constexpr int PB = PW > QT * HD * 4 ? PW : QT * HD * 4;   // their place, q's for the tail
    static constexpr int NEED = 2 * NS * TB + QB + PB + QT * A8_CH * 4;
    // A block waits for its TMEM without a limit, and its cluster waits for it, so it may never
    // wait for a block that a cluster of this kernel, of this call or of another stream's, waits
    // with.  Two things see to that, whatever the compiler's register counts are:
    // - Two blocks of these forms (one, where BPS is 1) take all of an SM's shared memory: beside
    //   them is no third, and no other kernel's block that holds or queues for TMEM.
    // - Two blocks' pieces fit wherever the first ones lie.  Nothing says that an allocation is
    //   aligned, and a block that has left may have pushed one to any column: of 16 units of 32
    //   columns, pieces of 4 and 2 leave 10 in three gaps, one of them of 4 at least, and then 6
    //   in four gaps, one of them of 2.  (One piece of 8 units in the middle would leave two gaps of 4.)
    // What else a block may meet on its SM ends by itself: it holds its TMEM before it lets a
    // dependent start, and waits for none of these blocks unless all of those hold theirs.
    static constexpr int SHARE = (A8_SM / BPS < A8_OPT + A8_OWN ? A8_SM / BPS : A8_OPT + A8_OWN) - A8_OWN - A8_STATIC;
    static constexpr int SMEM = NEED > SHARE ? NEED : SHARE;
    static_assert(SMEM + A8_STATIC <= A8_OPT && BPS * (SMEM + A8_STATIC + A8_OWN) <= A8_SM, "shared memory");
    static_assert(BPS == 1 ? SCOLS + OCOLS <= 512 : BPS == 2 && SCOLS <= 128 && OCOLS <= 64, "TMEM");
    static_assert((QW == 4 || QW == 8) && QB + PB >= KB && QT % QW == 0, "operands");
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
