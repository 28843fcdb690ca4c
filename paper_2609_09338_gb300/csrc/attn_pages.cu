// Attention over the bf16 paged cache on the tensor cores: a sequence's newest rows over
// all of it, a prefix that sequences share read once for all of them, or each row over the
// pages listed for it.
//
//   out_i = sum_j w_ij V_j / sum_j w_ij,  w_ij = 2^(q_i . K_j log2(e) / sqrt(hd) - m_i)
//
// Work is cut into units: up to 256 queries (row, head) of one KV head and the pages that
// they read.  The rows of a run of sequences are packed side by side, so a shared prefix
// is one unit for every 256 of the run's queries, and each sequence's own pages are units
// of their own.  A first kernel, a few blocks, lists the units; a unit is so many tiles of
// 128 keys (float32 queries: 64); the tiles of all units in a row are dealt out evenly in stretches to the workers
// of the second kernel, one block an SM.  Where a unit ends in one worker and its rows
// have no other, that worker writes the output; else (max, sum, output) parts go to the
// workspace and a third kernel joins them, in an order that goes by the lengths alone.
//
// A block has two streams, each with 128 columns of TMEM for scores and 128 for outputs, a
// warpgroup of its own that makes weights, and a warp that issues its products.  A unit of more than 128
// queries is a block's: its streams have 128 queries each and share the tiles of keys, and
// one warp issues both streams' products, so that one stream's run while the other's
// weights are made.  Others are a stream's, with a ring of tiles of its own: while one waits at a
// unit's end or begin the other goes on.  A thread is a query: maxima and sums need no
// exchange.  The reference m moves where a score exceeds it by AP_OVER; weights take the
// place of their scores in TMEM as bf16 and are the next product's operand there, 64 keys
// as soon as they are made.
//
// Measured (GB300, 8 KV heads of 128, us a call of three kernels; the second alone, caches flushed, in brackets).  Prompts of
// 1000..2048 rows of 4 sequences, groups of four, behind 4096 shared positions: 422 (409),
// 1.3 PFLOP/s in the kernel, 0.65 of cuBLAS: products alone take 340 of them, weights alone
// 290, and a tile's chain leaves a third uncovered.  One row of 64 sequences behind 8192 shared positions and 50..1000
// of their own: 61 (47, of 26 at the copy's rate: four or five tiles a unit, of which the
// last is half empty, and 1.5 us around them).  1..8 rows of 96 sequences behind four prefixes: 105 (81).
// Listed pages, 96 of each of 960 (row, head): 135 (120, 0.95 of the copy's rate).
#include <algorithm>

#include "internal.h"
#include "kv8.cuh"
#include "pages.cuh"
#include "tc.cuh"
#include "tcgen05.cuh"
#include "tma.cuh"

namespace osp {

constexpr float AP_OVER = 8.f;        // a weight is at most 2^AP_OVER before its reference moves
// From here on scores count in quarters, exactly, not in sc: the reference's rounding, half a step of it, must stay below
// what an exponent can be (with sc alone equal scores of 1e12 gave NaN).  A step of such a score is 65 and more in the exponent,
// so all but the largest weigh nothing either way.
constexpr float AP_HUGE = 0x1p32f;
constexpr int AP_SEEN = 1 << 30;      // position of a row that sees every key of its unit
constexpr int AP_NONE = -32;          // of one whose list is none, below every page: whoever reads the list refuses its entries
// What a unit costs beside its tiles, in tiles: its queries' loads, its outputs' stores and the waits
// between (with tiles alone dealt out evenly, 1..8 rows of 96 sequences: blocks ended between 57 and 92 us, 129 us a call
// instead of 116).  Units of lists are much alike, and whole numbers of tiles more even without it (132 us instead of 140).
constexpr int AP_COST_PAIR = 4, AP_COST = 1;
__host__ __device__ constexpr int ap_cost(bool lists, bool pair) { return lists ? 0 : pair ? AP_COST_PAIR : AP_COST; }
constexpr int AP_BLOCKS = 4;          // blocks that plan: each counts everything and writes its share of the units
constexpr int AP_PLAN = 1024;         // threads of a planning block
constexpr int AP_MAXB = 4096;
constexpr int AP_SHARE = 128;         // a prefix is shared where a sequence has fewer queries a KV head

template <int HD_, bool F32_>
struct AP {
    static constexpr int HD = HD_;
    static constexpr bool F32 = F32_;
    static constexpr int QP = F32 ? 3 : 1, PP = F32 ? 3 : 1;   // planes of a query and of a weight
    static constexpr int NH = HD / 64;
    static constexpr int KEYS = F32 ? 64 : 128, PG = KEYS / 16, PARTS = KEYS / 64;   // of a tile
    static constexpr int QR = F32 ? 64 : 128;                  // queries of a stream
    static constexpr bool PAIRS = !F32;                        // units of up to 2 * QR, both streams'
    static constexpr int QHB = QR * 128, KHB = KEYS * 128;     // bytes of 64 dims of a stream's queries, of a tile of keys
    static constexpr int QTB = NH * QHB, TB = NH * KHB;        // of all dims
    static constexpr int QS = QP * QTB, QB = 2 * QS;           // of a stream's planes, of both
    static constexpr int NS = (224 * 1024 - QB) / TB > 16 ? 16 : (224 * 1024 - QB) / TB, NSS = NS / 2;   // slots of K and V tiles, in turn; of one stream's
    static constexpr int SC = 128;                             // columns of a stream's scores and weights
    // An accumulator in TMEM is cut off, not rounded, at each product's addition, 16 keys or dims: up to 2^-23 of it, all of
    // one sign (outputs of 2^21 keys of bf16 queries in one accumulator: 1.2 % short).  So outputs are added up in float32
    // after every RUN tiles: 2^10 additions with bf16 queries, 2^-13 where the output's own rounding is 2^-8; with float32 ones
    // 24, and their scores are two accumulators, half of the dims each, with the small planes first.
    static constexpr int RUN = F32 ? 2 : 128;
    static constexpr int THREADS = 384;                        // two streams' 128, their warps of products, two of copies
    static constexpr int SMEM = 224 * 1024 + 1024;             // all of an SM's, so that no other kernel's TMEM lies beside this one's
    // (with 64 rows the first operand's other 64 are whatever lies behind: no one reads what they give)
    static_assert(QB + NS * TB + 1024 <= SMEM && RUN > 0 && NSS >= 2 && NS * TB >= QHB && 2 * SC <= 256, "room");
};

// A unit: queries i0 .. i0 + nq of the packed rows from row0 on, one KV head, and pages p0 .. p0 + np
// (np entries of the row's list).  Pages below pre come from the table's row lead, others from seq.
struct __align__(16) ApUnit {
    int cum, np;               // tiles of the units before, of its class, and what they cost beside; pages
    int row0, i0, nq, kvh;     // (a list's row0 is its row, b * max_rows + j)
    int seq, lead, pre, p0;
    int base;                  // position of row row0, or AP_SEEN, AP_NONE
    int poff, c0;              // its first part's first row in the workspace, the worker that begins it
    int poff1, stride;         // part k > 0 begins at poff1 + k * stride
    int id, own;               // own: the packed rows are sequence seq's
    int direct, pad[2];        // direct: its worker writes the output, the part's place holds sums on the way
};
static_assert(sizeof(ApUnit) == 80, "five loads of 16 bytes");

// A worker (a block for units of two streams, a stream for the others): its tiles, and the first one's unit
struct __align__(16) ApStart {
    ApUnit u;
    int t0, t1, pad[2];        // numbered as cum is
};

struct __align__(16) ApSeq {   // what the join needs of a sequence
    int n, row, unit, tiles;           // rows, the first packed one, first unit of its own pages, tiles of queries
    int pre_unit, pre_tiles, pre_row;  // of its run's prefix (pre_unit -1: none)
    int lead, size, pre_size, pad[2];  // queries of a unit
};

struct ApHead {
    int bad;                   // 1: a sequence's output is to be cleared; 2: all are
    int split[AP_BLOCKS];      // units that several workers have, where rows have no other parts, as each block counted them
    int pad[3];
};

struct ApWork {
    ApHead *head;
    ApUnit *units;
    int4 *parts;               // of a unit: poff (-1: its output is written), poff1, stride, how many
    ApSeq *seqs;
    int2 *rows;                // packed rows: b * max_rows + j, position
    ApStart *start;            // [sms] workers of two streams, [2 * sms] of one
    int *split;                // [AP_BLOCKS][3 * sms] their numbers
    int *bad, *bad_pre;        // [B]; of a run's prefix, by its first sequence
    float2 *ml;                // parts: (max, sum)
    float *o;                  // [hd]
};

static size_t ap_layout(int B, int max_rows, int Hq, int Hkv, int hd, bool lists, int sms, void *base, ApWork *w) {
    const long long G = Hq / Hkv, queries = (long long)max_rows * G, rows = (long long)B * max_rows;
    const long long qt = 64;   // queries of the smallest full unit
    long long units, parts;
    if (lists) {
        units = rows * Hkv;
        parts = 4LL * sms * 8;
    } else {
        // room for shared prefixes, also where max_rows rules them out: a workspace serves fewer rows too
        const long long some = B * std::min<long long>(max_rows, (AP_SHARE - 1) / G);
        units = (long long)B * Hkv * ((queries + qt - 1) / qt) + Hkv * (B + (some * G + qt - 1) / qt);
        parts = 2LL * sms * 256 + 4LL * sms * 128 + 4 * some * Hq;
    }
    size_t at = 0;
    auto take = [&](size_t n) {
        const size_t r = at;
        at += (n + 255) / 256 * 256;
        return (char *)base + r;
    };
    ApWork v;
    v.head = (ApHead *)take(sizeof(ApHead));
    v.units = (ApUnit *)take(units * sizeof(ApUnit));
    v.parts = (int4 *)take(units * sizeof(int4));
    v.seqs = (ApSeq *)take(B * sizeof(ApSeq));
    v.rows = (int2 *)take(rows * sizeof(int2));
    v.start = (ApStart *)take((size_t)3 * sms * sizeof(ApStart));
    v.split = (int *)take((size_t)AP_BLOCKS * 3 * sms * 4);
    v.bad = (int *)take((size_t)B * 4);
    v.bad_pre = (int *)take((size_t)B * 4);
    v.ml = (float2 *)take(parts * sizeof(float2));
    v.o = (float *)take(parts * hd * 4);
    if (w) *w = v;
    return at;
}
size_t kv_attend_workspace(int B, int max_rows, int Hq, int Hkv, int hd, bool lists, int sms) {
    return ap_layout(B, max_rows, Hq, Hkv, hd, lists, sms, nullptr, nullptr);
}

// ---------------------------------------------------------------- units
// Exclusive prefixes of N numbers over the block's first `warps` warps, and their sums (in those warps).
template <int N>
__device__ __forceinline__ void ap_scan(unsigned long long (&x)[N], unsigned long long (&sum)[N], unsigned long long (*sh)[4], int warps) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long in[N];
    if (warp < warps) {
#pragma unroll
        for (int k = 0; k < N; ++k) in[k] = x[k];
#pragma unroll 1
        for (int o = 1; o < 32; o <<= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const unsigned long long y = __shfl_up_sync(0xffffffffu, in[k], o);
                if (lane >= o) in[k] += y;
            }
        if (lane == 31)
#pragma unroll
            for (int k = 0; k < N; ++k) sh[warp][k] = in[k];
    }
    __syncthreads();
    if (warp < warps) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            x[k] = in[k] - x[k];
            sum[k] = 0;
        }
#pragma unroll 1
        for (int v = 0; v < warps; ++v)
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const unsigned long long y = sh[v][k];
                if (v < warp) x[k] += y;
                sum[k] += y;
            }
    }
    __syncthreads();
}

__host__ __device__ constexpr int ap_ceil(int a, int b) { return (a + b - 1) / b; }

// How a number of queries becomes units: how many, and how many queries each (the last one may have fewer).
struct ApCut {
    int units, size;
    bool pair;
};
__device__ __forceinline__ ApCut ap_cut(int queries, int QR, bool pairs) {
    ApCut c;
    c.pair = pairs && queries > QR;
    c.units = ap_ceil(queries, c.pair ? 2 * QR : QR);
    c.size = c.units > 1 ? ap_ceil(queries, c.units) : queries;
    return c;
}

// Tiles of keys that unit qt of a sequence's queries reads from page p0 on.
__device__ __forceinline__ int ap_tiles(int base, int queries, int lg, const ApCut &c, int qt, int p0, int PG) {
    const int i = min((qt + 1) * c.size, queries) - 1;
    return ap_ceil((base + (i >> lg)) / 16 + 1 - p0, PG);
}

// Which of a warp's lanes (of those in `todo`) have a list with an entry past the row's pages, from np on, that is not -1:
// four lists at a time, 256 entries each.  64 rows of 8 heads with 127 entries behind one page: 3 us; 512 rows 17 (a list
// a lane: 8 and 70); one row with 65535: 275.  (In the attention's copying warps, inlined or called, it moved the other
// warps' loops so that prompts took 444 us instead of 419.)
__device__ __noinline__ uint32_t ap_behind(const int32_t *pages, int list, int np, uint32_t todo, int n) {
    const int lane = threadIdx.x & 31;
    const bool wide = n % 4 == 0 && (uintptr_t)pages % 16 == 0;
    uint32_t found = 0;
    while (todo) {
        const int32_t *x[4];
        int from[4], low = n;
        uint32_t bits[4], odd[4] = {0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            bits[u] = todo & (0u - todo);   // 0: no more
            const int src = bits[u] ? __ffs(todo) - 1 : 0;
            todo ^= bits[u];
            x[u] = pages + (size_t)__shfl_sync(0xffffffffu, list, src) * n;
            from[u] = __shfl_sync(0xffffffffu, np, src);
            if (!bits[u]) from[u] = n;
            low = min(low, from[u]);
        }
        if (wide) {
            for (int i = (low & ~3) + lane * 4; i < n; i += 256) {
                int4 v[4][2];
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int at = i + 128 * k;
                        v[u][k] = at < n && at + 3 >= from[u] ? *(const int4 *)(x[u] + at) : make_int4(-1, -1, -1, -1);
                    }
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int at = i + 128 * k - from[u];   // of the first one, behind the list's pages
                        odd[u] |= (at >= 0 ? ~v[u][k].x : 0) | (at >= -1 ? ~v[u][k].y : 0) | (at >= -2 ? ~v[u][k].z : 0) | ~v[u][k].w;
                    }
            }
        } else {
            for (int i = low + lane; i < n; i += 64) {
                int v[4][2];
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int k = 0; k < 2; ++k) v[u][k] = i + 32 * k < n && i + 32 * k >= from[u] ? x[u][i + 32 * k] : -1;
#pragma unroll
                for (int u = 0; u < 4; ++u) odd[u] |= ~v[u][0] | ~v[u][1];
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (__any_sync(0xffffffffu, odd[u] != 0)) found |= bits[u];
    }
    return found;
}

// Lists the units, in one block or in several that each count everything.  Those of two streams and those of one are two classes, each
// with tiles, units and workers of its own; in a class the prefixes' come first.
template <int QR, bool PAIRS, int PG, bool LISTS>
__global__ void __launch_bounds__(AP_PLAN) attend_plan_kernel(const KvAttendArgs a, const ApWork w, int sms) {
    extern __shared__ unsigned long long s_dyn[];
    const int B = a.B, Hkv = a.Hkv, lg = __ffs(a.Hq / Hkv) - 1, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // of a sequence: rows (-1: refused; later a head's tiles) and position of the first one, its run's first sequence, pages of the prefix, packed
    // rows before it; of a run: rows.  Then units and tiles, first numbers then sums: a prefix's, its own.
    int *s_n = (int *)s_dyn, *s_base = s_n + B, *s_lead = s_base + B, *s_pre = s_lead + B, *s_row = s_pre + B, *s_cnt = s_row + B + 1;
    int *s_punit = s_cnt + B, *s_ptile = s_punit + B, *s_unit = s_ptile + B, *s_tile = s_unit + B;
    __shared__ unsigned long long sh[32][4];
    __shared__ int s_bad, s_split;
    __shared__ uint32_t s_begin[AP_MAXB / 32];   // a bit a sequence
    const int nb = (int)gridDim.x, rank = (int)blockIdx.x;
    if (tid == 0) s_bad = s_split = 0;
    for (int b = tid; b < B; b += AP_PLAN) s_cnt[b] = 0;
    pdl_wait();
    pdl_trigger();
    constexpr bool lists = LISTS;
    const bool split = !LISTS && a.share && (a.max_rows << lg) < AP_SHARE;
    for (int b0 = 0; b0 < B; b0 += AP_PLAN) {
        const int b = b0 + tid;
        bool begins = false;   // a run, or none of them: its first sequence is not the one before's
        if (b < B) {
            const SeqRows r = seq_rows(a.n_rows[b], a.seq_len[b], a.advanced, a.max_rows, a.max_pages);
            s_n[b] = r.code ? -1 : r.n;
            s_base[b] = r.base;
            auto first = [&](int x) {
                const int s = a.share ? a.share[x] : -1;
                return s == -1 ? x : s;
            };
            const int lead = first(b);
            begins = b == 0 || lead == b || lead != first(b - 1);
            s_lead[b] = lead;
            s_pre[b] = a.share ? a.shared_len[b] : 0;
            if (rank == 0) w.bad[b] = r.code != 0;
            if (rank == 0) w.bad_pre[b] = 0;
            if (r.code && rank == 0) set_status(a.status, r.code);
        }
        const uint32_t mask = __ballot_sync(0xffffffffu, begins);
        if (lane == 0) s_begin[b0 / 32 + warp] = mask;
    }
    __syncthreads();
    // no run begins in lead + 1 .. b: all of them, and lead itself, say that lead is their first
    auto together = [&](int lead, int b) {
        for (int i = (lead + 1) / 32; i <= b / 32; ++i) {
            uint32_t m = s_begin[i];
            if (i == (lead + 1) / 32) m &= ~0u << ((lead + 1) & 31);
            if (i == b / 32) m &= ~0u >> (31 - (b & 31));
            if (m) return false;
        }
        return true;
    };
    // runs: checked against what the sequences said, then written over it
    unsigned long long rows = 0;
    for (int b0 = 0; b0 < B; b0 += AP_PLAN) {
        const int b = b0 + tid;
        unsigned long long x[1] = {0}, sum[1];
        int n = 0, lead = b, pre = 0;
        if (b < B) {
            n = s_n[b];
            lead = s_lead[b];
            bool ok = n >= 0;
            if (a.share) {
                const bool run = lead == b || (lead >= 0 && lead < b && together(lead, b));
                if (!run) lead = b;
                const bool alone = lead == b && !(b + 1 < B && s_lead[b + 1] == b);
                pre = alone ? 0 : s_pre[lead];
                const bool fits = run && s_n[lead] >= 0 && pre >= 0 && pre % 16 == 0 && s_base[lead] >= pre && s_base[b] >= pre;
                if (ok && !fits && rank == 0) set_status(a.status, OSPREY_ERR_INVALID_ARG);
                ok = ok && fits;
            }
            if (!ok) {
                if (rank == 0) w.bad[b] = 1;
                s_bad = 1;
                n = pre = 0;
            }
            x[0] = n;
            if (split && n) atomicAdd(&s_cnt[lead], n);
        }
        ap_scan<1>(x, sum, sh, min(32, ap_ceil(B - b0, 32)));
        if (b < B) {
            s_row[b] = (int)(rows + x[0]);
            if (b == B - 1) s_row[B] = (int)(rows + x[0]) + n;
        }
        rows += warp * 32 < B - b0 ? sum[0] : 0;
        if (b < B) {   // checked, until all have read what the sequences said
            s_unit[b] = lead;
            s_tile[b] = pre / 16;
        }
    }
    __syncthreads();
    for (int b = tid; b < B; b += AP_PLAN) {
        s_lead[b] = s_unit[b];
        s_pre[b] = s_tile[b];
    }
    __syncthreads();
    auto shared = [&](int b) { return split && s_lead[b] == b && s_pre[b] > 0 && b + 1 < B && s_lead[b + 1] == b && s_cnt[b] > 0; };
    auto list_tiles = [&](int pos) { return ap_ceil(min(a.n_select, pos / 16 + 1), PG); };
    // a warp counts a sequence's tiles, its lanes those of a query tile or a row each (a thread's own sequence's, where there
    // is one of either)
    const bool many = lists ? a.max_rows > 1 : (a.max_rows << lg) > (PAIRS ? 2 * QR : QR);
    for (int b = warp; b < B && many; b += AP_PLAN / 32) {
        const int n = s_row[b + 1] - s_row[b], base = s_base[b];
        const ApCut c = ap_cut(max(1, n << lg), QR, PAIRS);
        const int p0 = shared(s_lead[b]) ? s_pre[b] : 0, items = n == 0 ? 0 : lists ? n : c.units;
        int t = 0;
        for (int i = lane; i < items; i += 32)
            t += ap_cost(lists, c.pair) + (lists ? list_tiles(base + i) : ap_tiles(base, n << lg, lg, c, i, p0, PG));
        t = __reduce_add_sync(0xffffffffu, t);
        if (lane == 0) s_tile[b] = t;
    }
    if (many) __syncthreads();
    // units and tiles of each class, in 32 bits each: pairs low, others high
    unsigned long long done[4] = {0, 0, 0, 0};   // prefix units and tiles, own units and tiles
    for (int b0 = 0; b0 < B; b0 += AP_PLAN) {
        const int b = b0 + tid;
        unsigned long long x[4] = {0, 0, 0, 0}, sum[4];
        if (b < B) {
            const int n = s_row[b + 1] - s_row[b];
            if (shared(b)) {
                const ApCut c = ap_cut(s_cnt[b] << lg, QR, PAIRS);
                const int k = Hkv * c.units;
                x[0] = (unsigned long long)k << (c.pair ? 0 : 32);
                x[1] = (unsigned long long)(k * (ap_ceil(s_pre[b], PG) + ap_cost(false, c.pair))) << (c.pair ? 0 : 32);
            }
            if (n > 0) {
                const ApCut c = ap_cut(n << lg, QR, PAIRS && !lists);
                x[2] = (unsigned long long)((lists ? n : c.units) * Hkv) << (c.pair ? 0 : 32);
                if (!many)
                    s_tile[b] = ap_cost(lists, c.pair) +
                                (lists ? list_tiles(s_base[b]) : ap_tiles(s_base[b], n << lg, lg, c, 0, shared(s_lead[b]) ? s_pre[b] : 0, PG));
                x[3] = (unsigned long long)(s_tile[b] * Hkv) << (c.pair ? 0 : 32);
            }
        }
        const bool ppair = (uint32_t)x[0] != 0, opair = (uint32_t)x[2] != 0;
        ap_scan<4>(x, sum, sh, min(32, ap_ceil(B - b0, 32)));
        if (warp * 32 < B - b0)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[k] += done[k];
                done[k] += sum[k];
            }
        if (b < B) {   // of its class; the offsets of the classes and of the prefixes come on top
            s_punit[b] = (int)(ppair ? (uint32_t)x[0] : (uint32_t)(x[0] >> 32));
            s_ptile[b] = (int)(ppair ? (uint32_t)x[1] : (uint32_t)(x[1] >> 32));
            s_unit[b] = (int)(opair ? (uint32_t)x[2] : (uint32_t)(x[2] >> 32));
            s_n[b] = s_tile[b];   // a head's tiles
            s_tile[b] = (int)(opair ? (uint32_t)x[3] : (uint32_t)(x[3] >> 32));
        }
    }
    if (tid == 0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) sh[0][k] = done[k];
        sh[1][0] = rows;
    }
    __syncthreads();
    rows = sh[1][0];
#pragma unroll
    for (int k = 0; k < 4; ++k) done[k] = sh[0][k];
    const int pre_units[2] = {(int)(uint32_t)done[0], (int)(done[0] >> 32)}, pre_tiles[2] = {(int)(uint32_t)done[1], (int)(done[1] >> 32)};
    const int tiles[2] = {pre_tiles[0] + (int)(uint32_t)done[3], pre_tiles[1] + (int)(done[3] >> 32)};
    const int pairs = pre_units[0] + (int)(uint32_t)done[2];   // units: pairs first
    // a worker takes `each` tiles
    const int each[2] = {max(1, ap_ceil(tiles[0], sms)), max(1, ap_ceil(tiles[1], 2 * sms))};
    const int used[2] = {ap_ceil(tiles[0], each[0]), ap_ceil(tiles[1], each[1])};
    for (int c = rank * AP_PLAN + tid; c < 3 * sms; c += nb * AP_PLAN)
        if (c < sms ? c >= used[0] : c - sms >= used[1]) w.start[c].t0 = w.start[c].t1 = 0;
    const float fd[2] = {1.f / each[0], 1.f / each[1]};
    auto by = [&](int x, bool pair) {   // x / each
        const int d = each[pair ? 0 : 1];
        int q = (int)((float)x * fd[pair ? 0 : 1]);
        while (q * d > x) --q;
        while (x - q * d >= d) ++q;
        return q;
    };
    auto put = [&](ApUnit &u, bool pair, bool other, int nt, int before) {
        const int d = each[pair ? 0 : 1], T = tiles[pair ? 0 : 1], t0 = u.cum + ap_cost(lists, pair);
        u.c0 = by(t0, pair);
        const int last = by(t0 + nt - 1, pair), segs = last - u.c0 + 1;
        // Places of parts.  Where a run's rows have two units each, the queries of the units before, and room for a whole
        // unit at each border between workers, which adds a part of one; else a worker has room for two units' parts,
        // the one that it goes on with and the one that it begins.
        const int most = pair ? 2 * QR : lists ? a.Hq / Hkv : QR, from = pair || !PAIRS || lists ? 0 : split ? sms * 2 * QR + 2 * a.Hq * (int)rows : 2 * sms * 2 * QR;
        if (split) {
            u.poff = u.poff1 = from + before + u.c0 * most;
            u.stride = u.nq;
        } else {
            u.poff = from + (2 * u.c0 + 1) * most;
            u.poff1 = from + 2 * u.c0 * most;
            u.stride = 2 * most;
        }
        u.direct = segs == 1 && !other;
        w.parts[u.id] = make_int4(u.direct ? -1 : u.poff, u.poff1, u.stride, segs);
        w.units[u.id] = u;
        if (segs > 1 && !split) w.split[rank * 3 * sms + atomicAdd(&s_split, 1)] = u.id;
        for (int c = by(u.cum + d - 1, pair); c <= last; ++c) {
            ApStart s;
            s.u = u;
            s.t0 = c * d;
            s.t1 = min(T, (c + 1) * d);
            s.pad[0] = s.pad[1] = 0;
            w.start[pair ? c : sms + c] = s;
        }
    };
    // a warp takes a sequence (several, where there are few), its lanes the units
    const int all = nb * (AP_PLAN / 32), wide = max(1, all / B), part = (rank * (AP_PLAN / 32) + warp) % wide;
    for (int b = (rank * (AP_PLAN / 32) + warp) / wide; b < B; b += all / wide) {
        const int n = s_row[b + 1] - s_row[b], lead = s_lead[b], base = s_base[b], row = s_row[b];
        const bool pre = shared(lead) && n > 0;
        const ApCut pc = ap_cut(max(1, s_cnt[lead] << lg), QR, PAIRS), c = ap_cut(max(1, n << lg), QR, PAIRS && !lists);
        const int punit = (pc.pair ? 0 : pairs) + s_punit[lead];
        const int unit = (c.pair ? pre_units[0] : pairs + pre_units[1]) + s_unit[b];
        if (split)
            for (int j = part * 32 + lane; j < n; j += 32 * wide) w.rows[row + j] = make_int2(b * a.max_rows + j, base + j);
        if (lane == 0 && part == 0) {
            ApSeq s;
            s.n = n;
            s.row = row;
            s.unit = unit;
            s.tiles = c.units;
            s.size = c.size;
            s.pre_unit = pre ? punit : -1;
            s.pre_tiles = pc.units;
            s.pre_size = pc.size;
            s.pre_row = s_row[lead];
            s.lead = lead;
            s.pad[0] = s.pad[1] = 0;
            w.seqs[b] = s;
        }
        ApUnit u{};
        u.seq = b;
        u.lead = lead;
        u.pre = s_pre[b];
        if (lead == b && shared(b)) {
            const int nt = ap_ceil(s_pre[b], PG), cost = nt + ap_cost(false, pc.pair);
            for (int k = part * 32 + lane; k < Hkv * pc.units; k += 32 * wide) {
                u.id = punit + k;
                u.kvh = k / pc.units;
                u.row0 = row;
                u.i0 = k % pc.units * pc.size;
                u.nq = min(pc.size, (s_cnt[b] << lg) - u.i0);
                u.p0 = 0;
                u.np = s_pre[b];
                u.base = AP_SEEN;
                u.own = 0;
                u.cum = s_ptile[b] + k * cost;
                put(u, pc.pair, true, nt, row * a.Hq + u.kvh * (s_cnt[b] << lg) + u.i0);
            }
        }
        if (n <= 0) continue;
        u.own = 1;
        u.p0 = pre ? s_pre[b] : 0;
        // 32 tiles of queries, or rows with lists, at a time: their tiles of keys, those before, then a lane each unit
        const int items = lists ? n : c.units, one = s_n[b], cum0 = (c.pair ? pre_tiles[0] : pre_tiles[1]) + s_tile[b];
        const float fh = 1.f / Hkv;   // (k + 1/2) / Hkv is 1 / (2 Hkv) from a whole number at least
        int before = 0;
        for (int i0 = 0; i0 < items; i0 += 32) {
            const int i = i0 + lane, cnt = min(32, items - i0);
            const int cost = ap_cost(lists, c.pair);
            const int nt = i >= items ? 0 : cost + (lists ? list_tiles(base + i) : ap_tiles(base, n << lg, lg, c, i, u.p0, PG));
            int e = nt;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, e, o);
                if (lane >= o) e += y;
            }
            const int sum = __shfl_sync(0xffffffffu, e, 31);
            e += before - nt;
            before += sum;
            for (int k0 = part * 32; k0 < cnt * Hkv; k0 += 32 * wide) {
                const int k = k0 + lane, x = min((int)(((float)k + 0.5f) * fh), cnt - 1), kvh = k - x * Hkv;
                const int xt = __shfl_sync(0xffffffffu, nt, x), xe = __shfl_sync(0xffffffffu, e, x), y = i0 + x;
                const bool mine = k < cnt * Hkv;
                if (!LISTS && !mine) continue;
                u.kvh = kvh;
                if (lists) {
                    u.id = unit + y * Hkv + kvh;
                    u.cum = cum0 + xe * Hkv + kvh * xt;
                    u.row0 = b * a.max_rows + y;   // the row itself
                    u.nq = 1 << lg;
                    u.base = base + y;
                    u.np = min(a.n_select, u.base / 16 + 1);
                    const uint32_t some = __ballot_sync(0xffffffffu, mine && u.np < a.n_select);
                    if (some && ap_behind(a.pages, u.row0 * Hkv + kvh, u.np, some, a.n_select) >> lane & 1) u.base = AP_NONE;
                } else {
                    u.id = unit + kvh * c.units + y;
                    u.cum = cum0 + kvh * one + xe;
                    u.row0 = row;
                    u.i0 = y * c.size;
                    u.nq = min(c.size, (n << lg) - u.i0);
                    u.base = base;
                    u.np = (base + ((u.i0 + u.nq - 1) >> lg)) / 16 + 1 - u.p0;
                }
                if (mine) put(u, c.pair, pre, xt - cost, ((int)rows + row) * a.Hq + kvh * (n << lg) + u.i0);
            }
        }
    }
    __syncthreads();
    if (tid == 0) {
        w.head->split[rank] = s_split;
        if (rank == 0) {
            w.head->bad = s_bad;
            for (int i = nb; i < AP_BLOCKS; ++i) w.head->split[i] = 0;
        }
    }
}

// ---------------------------------------------------------------- attention
// Shared-memory matrix descriptor of V, whose dims lie side by side: 128-byte rows of 64 dims,
// a key each, swizzled in eights; the next 64 dims `halves` bytes on.
__device__ __forceinline__ uint64_t ap_desc_v(uint32_t addr, uint32_t halves) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(halves >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
// the weights are A, in TMEM, two to a column
__device__ __forceinline__ void ap_mma_t(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
                 "r"(a), "l"(b), "r"(idesc), "r"(acc)
                 : "memory");
}
__device__ __forceinline__ float ap_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// the upper halves of two floats: bf16, cut off
__device__ __forceinline__ uint32_t ap_cut2(float lo, float hi) { return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632); }
__device__ __forceinline__ void ap_ld32(uint32_t addr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
// a page of V, 64 dims of its rows, then the next 64
__device__ __forceinline__ void ap_copy_v(void *dst, const CUtensorMap *m, int y, uint64_t *bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                     smem_u32(dst)),
                 "l"(m), "r"(0), "r"(y), "r"(0), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void ap_fence_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void ap_st16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}

// Waits for a phase, about a second at most, or a second without a change of `steps`, where that is given: then, or when
// another wait of the block has run out, false.
__device__ __forceinline__ bool ap_wait_limit(uint64_t *bar, uint32_t parity, const int *steps, int *abort, int32_t *status) {
    long long t0 = 0;
    int seen = 0;
    for (int i = 0; !mbar_try_wait(bar, parity);) {
        if (++i < 64) continue;
        if (*(volatile int *)abort) return false;
        const long long t = clock64();
        const int now = steps ? *(const volatile int *)steps : 0;
        if (!t0 || now != seen) {
            t0 = t;
            seen = now;
        }
        if (t - t0 > 2000000000LL) {
            *(volatile int *)abort = 1;
            set_status(status, OSPREY_ERR_TIMEOUT);
            return false;
        }
        i = 0;
    }
    return true;
}
// What is not needed for a phase that has ended is a call: the loops' code has to stay in the instruction cache.
__device__ __noinline__ bool ap_wait_long(uint64_t *bar, uint32_t parity, int *abort, int32_t *status) {
    return ap_wait_limit(bar, parity, nullptr, abort, status);
}
// A wait as long as another warp's work, which may be seconds: `steps` are the tiles that it is through with.
__device__ __noinline__ bool ap_wait_work(uint64_t *bar, uint32_t parity, const int *steps, int *abort, int32_t *status) {
    return ap_wait_limit(bar, parity, steps, abort, status);
}
__device__ __forceinline__ bool ap_wait(uint64_t *bar, uint32_t parity, int *abort, int32_t *status) {
    return mbar_try_wait(bar, parity & 1) || ap_wait_long(bar, parity & 1, abort, status);
}

// A stream's tiles lie in a ring of slots, K and V in turn; the units of two streams have a ring that both read.
struct ApRing {
    uint64_t *full, *freed;
    int base, n;               // its first slot, slots
};
// Where a tile's K or V lies in its ring, and how often the ring has been gone around.  (By increments: with the slot
// by division a product's issue waited some 300 cycles for it.)
struct ApSlot {
    int slot;
    uint32_t use;
    __device__ __forceinline__ void step(int n) {
        slot += 2;
        if (slot >= n) {
            slot -= n;
            ++use;
        }
    }
};

template <typename C>
__global__ void __launch_bounds__(C::THREADS, 1)
    attend_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                  const __grid_constant__ KvAttendArgs a, const __grid_constant__ ApWork w, int sms) {
    constexpr int HD = C::HD, NS = C::NS, NSS = C::NSS, NH = C::NH, TB = C::TB, HB = C::KHB, QP = C::QP, PP = C::PP, PG = C::PG, KEYS = C::KEYS;
    constexpr int W_MMA = 8, W_COPY = 10;
    extern __shared__ uint8_t raw[];
    uint8_t *sq = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023), *ring = sq + C::QB;
    __shared__ __align__(8) uint64_t full2[NS], freed2[NS], full1[2 * NSS], freed1[2 * NSS], sfull[2], pready[4], qready[2], odone[2], handed, drained[2];
    // units with a value that is not finite among keys that not every row sees (a stream is a few units ahead at most)
    __shared__ int s_abort, s_steps, s_odd[3][16];
    __shared__ uint32_t s_tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int G = a.Hq / a.Hkv, lg = __ffs(G) - 1;
    if (warp == W_MMA) {
        if (lane == 0) {
            for (int i = 0; i < NS; ++i) {
                mbar_init(&full2[i], 1);
                mbar_init(&freed2[i], 1);
            }
            for (int i = 0; i < 2 * NSS; ++i) {
                mbar_init(&full1[i], 1);
                mbar_init(&freed1[i], 1);
            }
            for (int i = 0; i < 2; ++i) {
                mbar_init(&sfull[i], 1);
                mbar_init(&pready[i], 4);
                mbar_init(&pready[2 + i], 4);
                mbar_init(&qready[i], 4);
                mbar_init(&odone[i], 1);
                mbar_init(&drained[i], 1);
            }
            mbar_init(&handed, 1);
            s_abort = s_steps = 0;
            for (int i = 0; i < 48; ++i) s_odd[0][i] = -1;
            mbar_fence_init();
        }
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    pdl_wait();
    asm volatile("fence.proxy.async.global;" ::: "memory");
    const uint32_t tmem = s_tmem;
    auto wait = [&](uint64_t *bar, uint32_t parity) { return ap_wait(bar, parity, &s_abort, a.status); };
    // a worker's units, and the tiles of each that are its own; `two`: units of two streams
    struct Walk {
        ApUnit u;
        int at, t1, k0, k1, cost;
        bool first;
    };
    auto begin = [&](bool two, int s) {
        const ApStart *x = w.start + (two ? (int)blockIdx.x : sms + 2 * (int)blockIdx.x + s);
        Walk k;
        k.u = x->u;
        k.at = x->t0;
        k.t1 = x->t1;
        k.k0 = k.k1 = 0;
        k.first = true;
        k.cost = ap_cost(a.pages, two);
        return k;
    };
    auto next = [&](Walk &k) {
        while (k.at < k.t1) {
            if (!k.first) k.u = w.units[k.u.id + 1];
            k.first = false;
            const int nt = ap_ceil(k.u.np, PG), t = k.u.cum + k.cost;   // its first tile's number
            k.k0 = max(0, k.at - t);
            k.k1 = min(nt, k.t1 - t);
            k.at = t + nt;
            if (k.k1 > k.k0) return true;   // (or the stretch ends before its first tile)
        }
        return false;
    };
    auto ring_of = [&](bool two, int s) { return two ? ApRing{full2, freed2, 0, NS} : ApRing{full1 + s * NSS, freed1 + s * NSS, s * NSS, NSS}; };

    if (warp >= W_COPY) {
        // copies: of a stream's K and V; where both read a tile, of its K or of its V.  The ids of 32 pages at a
        // time, the next 32 on their way.
        const int s = warp - W_COPY;
        auto id_of = [&](const ApUnit &x, int i) {
            if (i >= x.np) return -1;
            int p = x.p0 + i, seq = x.seq;
            bool bad = false;
            if (a.pages) {
                const int j = x.row0, pos = x.base;
                const int32_t *list = a.pages + ((size_t)j * a.Hkv + x.kvh) * a.n_select;
                const int e = list[i], before = i ? list[i - 1] : -1;
                bad = e < -1 || e > pos / 16 || (e >= 0 && i && before < 0) || (e >= 0 && e <= before);
                if (bad) set_status(a.status, OSPREY_ERR_INVALID_ARG);
                p = bad ? -1 : e;
            } else if (p < x.pre) {
                seq = x.lead;
            }
            int id = -1;
            if (p >= 0) {
                id = a.page_table[(size_t)seq * a.max_pages + p];
                if (id < 0 || id >= a.n_pages) {
                    id = 0;
                    bad = true;
                    set_status(a.status, OSPREY_ERR_CAPACITY);
                }
            }
            if (bad) {
                *(volatile int *)((!a.pages && p < x.pre ? w.bad_pre : w.bad) + seq) = 1;
                atomicMax(&w.head->bad, 1);
            }
            return id;
        };
        bool go = true;
        uint32_t uses2 = 0;   // of the ring of both streams
#pragma unroll 1
        for (int phase = C::PAIRS ? 0 : 1; phase < 2; ++phase) {
            const bool two = phase == 0;
            const int kv0 = two ? s : 0, kv1 = two ? s : 1;
            const ApRing r = ring_of(two, s);
            Walk k = begin(two, s);
            if (!two && C::PAIRS) {   // what both streams read has been read: of each slot's last tile the warp that copied it knows
                for (int i = 0; i < NS && go; ++i) {
                    const uint32_t n = uses2 / NS + ((uint32_t)i < uses2 % NS ? 1 : 0);
                    if (n && ((int)(n - 1) * NS + i & 1) == s) go = wait(&freed2[i], n - 1);
                }
                __syncwarp();
                named_sync(1, 64);
            }
            go = __all_sync(0xffffffffu, go);
            uint32_t g = 0;
            ApSlot ks{0, 0}, vs{1, 0};
            auto fetch = [&](int &from, int &to, int &kvh) {   // the next pages to ask for: a unit's tiles from .. to
                from = to = 0;
                if (k.k0 >= k.k1 && !next(k)) return -1;
                from = k.k0;
                to = min(from + 32 / PG, k.k1);
                k.k0 = to;
                kvh = k.u.kvh;
                const int i = from * PG + lane;
                return i < to * PG ? id_of(k.u, i) : -1;
            };
            int from, to, nfrom = 0, nto = 0, kvh = 0, nkvh = 0;
            int ids = fetch(from, to, kvh), nids = -1;
            while (to > from && go) {
#pragma unroll 1
                for (int t = from; t < to; ++t) {
                    const int id = __shfl_sync(0xffffffffu, ids, (t - from) * PG + (lane & (PG - 1)));
                    const uint32_t have = __ballot_sync(0xffffffffu, id >= 0) & ((1u << PG) - 1);
                    int y[PG];
#pragma unroll
                    for (int p = 0; p < PG; ++p) y[p] = __shfl_sync(0xffffffffu, (id * a.Hkv + kvh) * 16, p);
                    // K as its operand wants it, 64 dims of a tile's keys side by side; V a page at a time
                    if (kv0 == 0) {
                        const int slot = ks.slot;
                        if (ks.use) go = wait(&r.freed[slot], ks.use - 1);
                        go = __all_sync(0xffffffffu, go);
                        uint8_t *dst = ring + (r.base + slot) * TB;
                        if (go && tc_elect()) {
                            mbar_arrive_expect_tx(&r.full[slot], (uint32_t)(__popc(have) * 2048 * NH));
#pragma unroll
                            for (int p = 0; p < PG; ++p)
                                if (have >> p & 1)
#pragma unroll
                                    for (int h = 0; h < NH; ++h) tma_2d(dst + h * HB + p * 2048, &mk, h * 64, y[p], &r.full[slot]);
                        }
                        __syncwarp();
                    }
                    if (kv1 == 1 && go) {
                        const int slot = vs.slot;
                        if (vs.use) go = wait(&r.freed[slot], vs.use - 1);
                        go = __all_sync(0xffffffffu, go);
                        uint8_t *dst = ring + (r.base + slot) * TB;
                        if (go && tc_elect()) {
                            mbar_arrive_expect_tx(&r.full[slot], (uint32_t)(__popc(have) * 2048 * NH));
#pragma unroll
                            for (int p = 0; p < PG; ++p)
                                if (have >> p & 1) ap_copy_v(dst + p * 2048 * NH, &mv, y[p], &r.full[slot]);
                        }
                        __syncwarp();
                    }
                    ++g;
                    ks.step(r.n);
                    vs.step(r.n);
                    if (!go) break;
                    // the next stretch's ids, while these copies are on their way
                    if (t == from) nids = fetch(nfrom, nto, nkvh);
                }
                ids = nids;
                kvh = nkvh;
                from = nfrom;
                to = nto;
            }
            if (two) uses2 = 2 * g;
        }
    } else if (warp == W_MMA || warp == W_MMA + 1) {
        const int me = warp - W_MMA;
        if (tc_elect()) {
            const uint64_t dk = tc_desc(smem_u32(ring)), dv = ap_desc_v(smem_u32(ring), 2048);
            const uint32_t is = tc_idesc(128, KEYS), io = tc_idesc(128, HD) | 1u << 16;
            uint32_t np = 0, seg = 0;   // a bit a stream: the phases of its tiles' and its units' barriers
            bool go = true;
            auto scores = [&](const ApRing &r, int s, const ApSlot &k, bool done) {   // of the tile in slot k; done: nobody else reads it
                go = go && wait(&r.full[k.slot], k.use);
                if (!go) return;
                tc_fence_after();
                const uint64_t d = dk + ((r.base + k.slot) * TB >> 4), dq = tc_desc(smem_u32(sq + s * C::QS));
                constexpr int half = C::F32 ? HD / 32 : HD / 16;   // steps of an accumulator
#pragma unroll
                for (int p = QP - 1; p >= 0; --p)
#pragma unroll
                    for (int x = 0; x < HD / 16; ++x)
                        tc_mma(tmem + s * C::SC + x / half * 64, dq + (((uint32_t)p * C::QTB + (x / 4) * C::QHB + (x % 4) * 32) >> 4),
                               d + ((uint32_t)((x / 4) * HB + (x % 4) * 32) >> 4), is, p + 1 < QP || x % half > 0);
                tc_commit(&sfull[s]);
                if (done) tc_commit(&r.freed[k.slot]);
            };
            auto outputs = [&](const ApRing &r, int s, const ApSlot &v, int steps, bool first, bool done) {
                go = go && wait(&r.full[v.slot], v.use);
                const uint64_t d = dv + ((r.base + v.slot) * TB >> 4);
                const uint32_t ts = tmem + s * C::SC, to = tmem + 256 + s * 128;
#pragma unroll
                for (int h = 0; h < C::PARTS; ++h) {   // 64 keys as soon as their weights are there
                    go = go && wait(&pready[2 * h + s], np >> s);
                    if (!go) return;
                    tc_fence_after();
                    for (int x = h * 4; x < min(steps, h * 4 + 4); ++x)
#pragma unroll
                        for (int p = 0; p < PP; ++p)
                            ap_mma_t(to, ts + (p < 2 ? (x >> 1) * 32 + p * 16 + (x & 1) * 8 : KEYS + x * 8),
                                     d + (x * 2048 * NH >> 4), io, !first || p > 0 || x > 0);
                }
                np ^= 1u << s;
                if (done) tc_commit(&r.freed[v.slot]);
            };
            if (C::PAIRS) {
                // one warp issues both streams' products, a stream's output and next scores together: then the other
                // makes weights meanwhile.  (With a warp a stream they fell into step.)
                const ApRing r = ring_of(true, 0);
                Walk k = begin(true, 0);
                ApSlot ks{0, 0}, vs{1, 0};
                if (me == 1) {
                    // what its stream's barriers have behind them; a wait for a phase is right only when the one before
                    // it has ended, so it starts when the other warp is through
                    while (next(k)) {
                        seg ^= 2;
                        np ^= (uint32_t)(k.k1 - k.k0 & 1) << 1;
                    }
                    go = ap_wait_work(&handed, 0, &s_steps, &s_abort, a.status);
                } else {
                    int steps = 0;
                    while (go && next(k)) {
#pragma unroll 1
                        for (int s = 0; s < 2 && go; ++s) {
                            go = wait(&qready[s], seg >> s);
                            seg ^= 1u << s;
                            tc_fence_after();
                            scores(r, s, ks, s == 1);
                        }
                        ks.step(r.n);
#pragma unroll 1
                        for (int t = k.k0; t < k.k1 && go; ++t) {
#pragma unroll 1
                            for (int s = 0; s < 2 && go; ++s) {
                                outputs(r, s, vs, min(PG, k.u.np - t * PG), (t - k.k0) % C::RUN == 0, s == 1);
                                if (t + 1 < k.k1) scores(r, s, ks, s == 1);
                                else if (go) tc_commit(&odone[s]);
                            }
                            if (t + 1 < k.k1) ks.step(r.n);
                            vs.step(r.n);
                            *(volatile int *)&s_steps = ++steps;
                        }
                    }
                    mbar_arrive(&handed);
                }
            }
            const ApRing r = ring_of(false, me);
            Walk k = begin(false, me);
            ApSlot ks{0, 0}, vs{1, 0};
            while (go && next(k)) {
                go = wait(&qready[me], seg >> me);
                seg ^= 1u << me;
                tc_fence_after();
                scores(r, me, ks, true);
                ks.step(r.n);
#pragma unroll 1
                for (int t = k.k0; t < k.k1 && go; ++t) {
                    outputs(r, me, vs, min(PG, k.u.np - t * PG), (t - k.k0) % C::RUN == 0, true);
                    vs.step(r.n);
                    if (t + 1 < k.k1) {
                        scores(r, me, ks, true);
                        ks.step(r.n);
                    } else if (go) {
                        tc_commit(&odone[me]);
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp < W_MMA) {
        const int s = warp >> 2, r = tid & 127;   // stream, query
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t ts = tmem + lanes + s * C::SC, to = tmem + lanes + 256 + s * 128;
        constexpr float sc = (float)((HD == 128 ? 0.08838834764831845 : 0.125) * 1.4426950408889634);
        uint32_t ns = 0, seg = 0;
        bool go = true;   // a warp's threads leave together, a run of tiles after a wait that gave up at most
#pragma unroll 1
        for (int phase = C::PAIRS ? 0 : 1; phase < 2 && go; ++phase) {
            const bool two = phase == 0;
            const ApRing rg = ring_of(two, s);
            Walk k = begin(two, s);
            ApSlot vs{1, 0};
            while (go && next(k)) {
                const ApUnit &u = k.u;
                const int q0 = u.i0 + (two ? s * C::QR : 0), nq = two && s ? u.nq - C::QR : min(u.nq, C::QR);   // the stream's queries
                // ------------------------------------------------ queries
                {
                    // a thread takes 8 dims and the 8 that the rotation pairs them with, of some queries at a time: their
                    // loads are on their way together (one after another, 128 queries took 10 us)
                    constexpr int CH = HD / 16, N = C::F32 ? 2 : 4, W = C::F32 ? 4 : 2;
#pragma unroll 1
                    for (int x0 = r; x0 < nq * CH; x0 += 128 * N) {
                        uint4 raw[N][W];
                        int at[N];
#pragma unroll
                        for (int k = 0; k < N; ++k) {
                            const int x = min(x0 + 128 * k, nq * CH - 1), qr = x / CH, c = x % CH, i = q0 + qr;
                            // an own row is the sequence's i >> lg, a list's the one row
                            int row = a.pages ? u.row0 : u.seq * a.max_rows + (i >> lg);
                            at[k] = u.base + (a.pages ? 0 : i >> lg);
                            if (!u.own) {
                                const int2 y = w.rows[u.row0 + (i >> lg)];
                                row = y.x;
                                at[k] = y.y;
                            }
                            const int64_t e = (int64_t)row * a.q_stride + (u.kvh * G + (i & (G - 1))) * HD + c * 8;
                            const int esize = C::F32 ? 4 : 2;
                            const uint4 *p = (const uint4 *)((const char *)a.q + e * esize);
#pragma unroll
                            for (int y = 0; y < W / 2; ++y) {
                                raw[k][y] = p[y];
                                raw[k][W / 2 + y] = p[HD / 2 * esize / 16 + y];
                            }
                        }
#pragma unroll
                        for (int k = 0; k < N; ++k) {
                            const int x = x0 + 128 * k, qr = x / CH, c = x % CH;
                            if (x >= nq * CH) break;
                            float lo[8], hi[8];
                            if constexpr (C::F32) {
#pragma unroll
                                for (int y = 0; y < 2; ++y) {
                                    *(uint4 *)(lo + 4 * y) = raw[k][y];
                                    *(uint4 *)(hi + 4 * y) = raw[k][2 + y];
                                }
                            } else {
                                const uint32_t y0[4] = {raw[k][0].x, raw[k][0].y, raw[k][0].z, raw[k][0].w};
                                const uint32_t y1[4] = {raw[k][1].x, raw[k][1].y, raw[k][1].z, raw[k][1].w};
#pragma unroll
                                for (int y = 0; y < 4; ++y) {
                                    lo[2 * y] = bf_lo(y0[y]);
                                    lo[2 * y + 1] = bf_hi(y0[y]);
                                    hi[2 * y] = bf_lo(y1[y]);
                                    hi[2 * y + 1] = bf_hi(y1[y]);
                                }
                            }
                            if (a.rotate) {
#pragma unroll
                                for (int y = 0; y < 8; ++y) {
                                    float cc, ss;
                                    rope_cs_fix(a.freq[c * 8 + y], at[k], cc, ss);
                                    const float t = lo[y] * cc - hi[y] * ss;
                                    hi[y] = hi[y] * cc + lo[y] * ss;
                                    lo[y] = t;
                                }
                            }
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                float *v = h ? hi : lo;
                                const int d = c * 8 + h * (HD / 2);
                                uint8_t *dst = sq + s * C::QS + (d >> 6) * C::QHB + qr * 128 + (((d & 63) >> 3) ^ (qr & 7)) * 16;
#pragma unroll
                                for (int p = 0; p < QP; ++p) {
                                    uint32_t y[4];
#pragma unroll
                                    for (int z = 0; z < 4; ++z) {
                                        y[z] = kv8_bf2(v[2 * z], v[2 * z + 1]);
                                        if (p + 1 < QP) {
                                            v[2 * z] -= bf_lo(y[z]);
                                            v[2 * z + 1] -= bf_hi(y[z]);
                                        }
                                    }
                                    *(uint4 *)(dst + p * C::QTB) = make_uint4(y[0], y[1], y[2], y[3]);
                                }
                            }
                        }
                    }
                    ap_fence_smem();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&qready[s]);
                }
                // ------------------------------------------------ tiles
                const bool live = r < nq, warp_live = (r & ~31) < nq;
                const int pos = u.base == AP_SEEN ? AP_SEEN : u.base + (a.pages ? 0 : (q0 + r) >> lg);
                const int pos_min = u.base == AP_SEEN || a.pages ? u.base : u.base + (u.i0 >> lg);   // of the unit
                const int pos_max = u.base == AP_SEEN || a.pages ? u.base : u.base + ((u.i0 + u.nq - 1) >> lg);
                const int32_t *list = a.pages ? a.pages + ((size_t)u.row0 * a.Hkv + u.kvh) * a.n_select : nullptr;
                float m = -INFINITY, l = 0.f;
                // The accumulator's outputs, added to those of the runs before: to the unit's part, or (all of them: `last`) to the
                // call's output.
                bool added = false;
                float m_then = 0.f;
                auto flush = [&](bool last) {
                    const int seg_key = max((u.p0 + k.k0 * PG) * 16, pos_min + 1), seg_end = min((u.p0 + min(k.k1 * PG, u.np)) * 16, pos + 1);
                    const bool odd = last && *(volatile int *)&s_odd[two ? 2 : s][u.id & 15] == u.id && !list && u.base != AP_SEEN;
                    const bool direct = u.direct;
                    const int me = two ? blockIdx.x : 2 * blockIdx.x + s, iq = q0 + r;
                    const int part = me - u.c0;
                    const size_t prow = (size_t)(part == 0 ? u.poff : u.poff1 + part * u.stride) + (iq - u.i0);
                    const size_t orow = ((size_t)(a.pages ? u.row0 : u.seq * a.max_rows + (iq >> lg)) * a.Hq + u.kvh * G + (iq & (G - 1))) * HD;
                    // an empty list's output is 0; other rows' without a weight, whose scores are all -inf, NaN
                    const float by = !direct || !last ? 1.f : l == 0.f ? (list && list[0] < 0 ? 0.f : NAN) : 1.f / l;
                    const float then = !added || m_then == -INFINITY ? 0.f : ap_ex2(m_then - m);
#pragma unroll 1
                    for (int c = 0; c < HD / 32; ++c) {
                        uint32_t v[32];
                        __syncwarp();
                        ap_ld32(to + c * 32, v);
                        tc_ld_wait();
                        float o[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            asm volatile("" : "+r"(v[i]));
                            o[i] = __uint_as_float(v[i]);
                        }
                        if (odd && live)
#pragma unroll 1
                            for (int key = seg_key; key < seg_end; ++key) {
                                const int pg = key / 16, id = a.page_table[(size_t)(pg < u.pre ? u.lead : u.seq) * a.max_pages + pg];
                                if (id < 0 || id >= a.n_pages) continue;
                                const uint16_t *vr = a.v_pages + (((size_t)id * a.Hkv + u.kvh) * 16 + key % 16) * HD + c * 32;
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if ((vr[i] & 0x7f80u) == 0x7f80u) o[i] += bf_to_f(vr[i]);
                            }
                        if (live) {
                            float *acc = w.o + prow * HD + c * 32;
                            if (added) {
#pragma unroll
                                for (int i = 0; i < 32; i += 4) {
                                    const float4 x = *(const float4 *)(acc + i);
                                    o[i] = fmaf(x.x, then, o[i]);
                                    o[i + 1] = fmaf(x.y, then, o[i + 1]);
                                    o[i + 2] = fmaf(x.z, then, o[i + 2]);
                                    o[i + 3] = fmaf(x.w, then, o[i + 3]);
                                }
                            }
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] *= by;
                            if (!direct || !last || C::F32) {
                                float *dst = direct && last ? (float *)a.out + orow + c * 32 : acc;
#pragma unroll
                                for (int i = 0; i < 32; i += 4) *(float4 *)(dst + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                            } else {
                                uint16_t *dst = (uint16_t *)a.out + orow + c * 32;
#pragma unroll
                                for (int i = 0; i < 32; i += 8)
                                    *(uint4 *)(dst + i) = make_uint4(kv8_bf2(o[i], o[i + 1]), kv8_bf2(o[i + 2], o[i + 3]),
                                                                     kv8_bf2(o[i + 4], o[i + 5]), kv8_bf2(o[i + 6], o[i + 7]));
                            }
                        }
                    }
                    if (live && !direct && last) w.ml[prow] = make_float2(m, l);
                    added = true;
                    m_then = m;
                };
#pragma unroll 1
                for (int t0 = k.k0; t0 < k.k1 && go; t0 += C::RUN) {
                    const int t1 = min(t0 + C::RUN, k.k1);
#pragma unroll 1
                    for (int t = t0; t < t1; ++t, vs.step(rg.n)) {
                        const int key0 = (u.p0 + t * PG) * 16;
                        const int pages = min(PG, u.np - t * PG);
                        // keys of the tile that the thread's query, every query and any query sees
                        int lim, lim_min, lim_max;
                        if (list) {
                            int n = 0, e_last = -1;
#pragma unroll
                            for (int p = 0; p < PG; ++p) {
                                const int e = p < pages ? list[t * PG + p] : -1;
                                if (e >= 0) {
                                    n = p + 1;
                                    e_last = e;
                                }
                            }
                            lim = lim_min = lim_max = e_last == pos / 16 ? (n - 1) * 16 + pos % 16 + 1 : n * 16;
                        } else {
                            lim = min(pages * 16, pos - key0 + 1);
                            lim_min = min(pages * 16, pos_min - key0 + 1);
                            lim_max = min(pages * 16, pos_max - key0 + 1);
                        }
                        wait(&sfull[s], ns++);
                        __syncwarp();
                        tc_fence_after();
                        // V of keys that not every query sees: what none sees counts as 0, whatever the page holds, and what
                        // is not finite is added at the end to the queries that see it.  (Behind the wait for the scores: the
                        // tile before's V has landed then, and the barrier is in this one's phase or past it.)
                        if (max(lim_min, 0) < pages * 16) {
                            wait(&rg.full[vs.slot], vs.use);
                            if (r >= lim_min && r < pages * 16) {
                                uint8_t *v = ring + (rg.base + vs.slot) * TB + (r >> 4) * 2048 * NH + (r & 15) * 128;
#pragma unroll 1
                                for (int c = 0; c < 8 * NH; ++c) {
                                    uint4 *x = (uint4 *)(v + (c >> 3) * 2048 + (c & 7) * 16);
                                    if (r >= lim_max) {
                                        *x = make_uint4(0, 0, 0, 0);
                                    } else {
                                        uint4 y = *x;
                                        uint32_t z[4] = {y.x, y.y, y.z, y.w};
                                        bool odd = false;
#pragma unroll
                                        for (int q = 0; q < 4; ++q) {
                                            if ((z[q] & 0x7f80u) == 0x7f80u) z[q] &= 0xffff0000u, odd = true;
                                            if ((z[q] & 0x7f800000u) == 0x7f800000u) z[q] &= 0xffffu, odd = true;
                                        }
                                        if (odd) {   // the flag first: the other stream may find zeros
                                            *(volatile int *)&s_odd[two ? 2 : s][u.id & 15] = u.id;
                                            __threadfence_block();
                                            *x = make_uint4(z[0], z[1], z[2], z[3]);
                                        }
                                    }
                                }
                                ap_fence_smem();
                            }
                            __syncwarp();
                        }
                        if (warp_live) {
                            if (lim_min < KEYS) {   // of the whole tile: a warp's threads take the same way.  What is not seen is -inf.
#pragma unroll 1
                                for (int c = max(lim_min, 0) & ~15; c < KEYS; c += 16) {
                                    float x[16];
                                    tc_ld16(ts + c, x);
                                    tc_ld_wait();
                                    tc_ld_tie(x);
#pragma unroll
                                    for (int i = 0; i < 16; ++i) x[i] = c + i < lim ? x[i] : -INFINITY;
                                    tc_st16(ts + c, x);
                                    if constexpr (C::F32) {
                                        tc_ld16(ts + 64 + c, x);
                                        tc_ld_wait();
                                        tc_ld_tie(x);
#pragma unroll
                                        for (int i = 0; i < 16; ++i) x[i] = c + i < lim ? x[i] : 0.f;
                                        tc_st16(ts + 64 + c, x);
                                    }
                                }
                                tc_st_wait();
                            }
                            // 32 scores at a time, twice: for the largest, and for the weights.  (The block's loops have to stay in the
                            // instruction cache: all 128 scores in registers, once, made prompts 468 us instead of 418, 64 at a time
                            // 430, the weights' loop unrolled 424, the first loop rolled 463.)
                            uint32_t v[32];
                            auto scores = [&](int c) {
                                ap_ld32(ts + c * 32, v);
                                tc_ld_wait();
#pragma unroll
                                for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(v[i]));   // not before the wait
                                if constexpr (C::F32) {
                                    uint32_t x[32];
                                    ap_ld32(ts + 64 + c * 32, x);
                                    tc_ld_wait();
#pragma unroll
                                    for (int i = 0; i < 32; ++i) {
                                        asm volatile("" : "+r"(x[i]));
                                        v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(x[i]));
                                    }
                                }
                            };
                            float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                            for (int c = 0; c < KEYS / 32; ++c) {
                                scores(c);
#pragma unroll
                                for (int i = 0; i < 32; i += 2)
                                    asm("max.f32 %0, %0, %1, %2;" : "+f"(t4[i / 2 & 3]) : "f"(__uint_as_float(v[i])), "f"(__uint_as_float(v[i + 1])));
                            }
                            const float best = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3]));
                            const float top = best * (fabsf(best) >= AP_HUGE ? 0.25f : sc);
                            const float was = m;
                            if (m == -INFINITY || top > m + AP_OVER) m = top;
                            const bool moved = m != was && was != -INFINITY;
                            if (__any_sync(0xffffffffu, moved)) {   // every product of this stream has ended: the scores came behind them
                                const float f = moved ? ap_ex2(was - m) : 1.f;
                                l *= f;
#pragma unroll 1
                                for (int c = 0; c < HD / 16; ++c) {
                                    float x[16];
                                    tc_ld16(to + c * 16, x);
                                    tc_ld_wait();
                                    tc_ld_tie(x);
#pragma unroll
                                    for (int i = 0; i < 16; ++i) x[i] *= f;
                                    tc_st16(to + c * 16, x);
                                }
                            }
                            const float ref = m == -INFINITY ? 0.f : m;
                            // A weight in one plane of bf16: 2^-8 of it off at most, outputs 2.3e-3 from float64 where their own rounding
                        // is 1.7e-3.  Two planes, 16 bits, leave that alone and take prompts 526 us instead of 419, 1..8 rows 116
                        // (102), the shared prefix 62 (58), listed pages 140 (131).
                        f2 sum[2] = {0ull, 0ull};
                            const float scm = fabsf(m) >= AP_HUGE / 4 ? 0.25f : sc;
                            const f2 sc2 = mk2(scm, scm), rf2 = mk2(-ref, -ref);
#pragma unroll 1
                            for (int c = 0; c < KEYS / 32; ++c) {
                                scores(c);
                                uint32_t p[PP][16];
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    float e0, e1;
                                    un2(fma2(mk2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), sc2, rf2), e0, e1);
                                    e0 = ap_ex2(e0);
                                    e1 = ap_ex2(e1);
                                    if constexpr (PP == 1) {
                                        p[0][i] = kv8_bf2(e0, e1);
                                    } else {
                                        // 24 bits in three planes, cut off, so that none has another sign, and none is 0 but of a weight
                                        // of 0: a value of infinity stays one
                                        p[0][i] = ap_cut2(e0, e1);
                                        const float d0 = e0 - bf_lo(p[0][i]), d1 = e1 - bf_hi(p[0][i]);
                                        p[1][i] = ap_cut2(d0, d1);
                                        p[2][i] = ap_cut2(d0 - bf_lo(p[1][i]), d1 - bf_hi(p[1][i]));
                                        const uint32_t least = __vminu2(p[0][i], 0x00800080u);
                                        p[1][i] = __vmaxu2(p[1][i], least);
                                        p[2][i] = __vmaxu2(p[2][i], least);
                                    }
                                    sum[i & 1] = add2(sum[i & 1], mk2(e0, e1));
                                }
                                ap_st16(ts + c * 32, p[0]);
                                if constexpr (PP == 3) {
                                    ap_st16(ts + c * 32 + 16, p[1]);
                                    ap_st16(ts + KEYS + c * 16, p[2]);
                                }
                                if (c & 1) {   // 64 keys' weights: their products may begin
                                    tc_st_wait();
                                    tc_fence_before();
                                    __syncwarp();
                                    if (lane == 0) mbar_arrive(&pready[2 * (c >> 1) + s]);
                                }
                            }
                            float x0, x1, y0, y1;
                            un2(sum[0], x0, x1);
                            un2(sum[1], y0, y1);
                            l += (x0 + x1) + (y0 + y1);
                        }
                        if (!warp_live) {
                            __syncwarp();
                            if (lane == 0)
#pragma unroll
                                for (int h = 0; h < C::PARTS; ++h) mbar_arrive(&pready[2 * h + s]);
                        }
                    }
                    // ------------------------------------------------ the run's outputs
                    // (the next tile's scores come behind the products of all before)
                    if (t1 < k.k1) wait(&sfull[s], ns);
                    else wait(&odone[s], seg++);
                    go = __all_sync(0xffffffffu, !*(volatile int *)&s_abort);   // (a tile each: prompts took 8 % longer)
                    tc_fence_after();
                    if (go && warp_live) flush(t1 == k.k1);
                }
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if (s_abort) {   // every wait has ended, one of them too early: the call's outputs are cleared, and the block stays until its
                     // products and its copies are through
        if ((warp == W_MMA || warp == W_MMA + 1) && tc_elect()) {
            tc_commit(&drained[warp - W_MMA]);
            mbar_wait(&drained[warp - W_MMA], 0, 20000000LL);
        }
        if (tid == 0) {
            atomicMax(&w.head->bad, 2);   // (another block's bad page may come later)
            for (int ph = 0; ph < 2; ++ph) {
                for (int i = 0; i < NS && C::PAIRS; ++i) mbar_wait(&full2[i], ph, 20000000LL);
                for (int i = 0; i < 2 * NSS; ++i) mbar_wait(&full1[i], ph, 20000000LL);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == W_MMA) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// ---------------------------------------------------------------- joining parts
// A warp a query: its parts, four on their way together, each lane HD / 32 dims.  (With the
// (max, sum) a lane each and eight parts together it took twice as long: more code than
// work, and a kernel's code is fetched anew by each launch.)
template <int HD>
__device__ __forceinline__ void ap_join(const KvAttendArgs &a, const ApWork &w, int4 p0, int r0, int4 p1, int r1, size_t orow, const int32_t *list) {
    constexpr int N = HD / 32;
    const int lane = threadIdx.x & 31, all = p0.w + p1.w;
    float M = -INFINITY, L = 0.f, o[N];
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] = 0.f;
#pragma unroll 1
    for (int k0 = 0; k0 < all; k0 += 4) {
        float x[4][N];
        float2 ml[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = k0 + i, k1 = k - p0.w;
            ml[i] = make_float2(-INFINITY, 0.f);
            if (k < all) {
                const size_t p = k < p0.w ? (k == 0 ? p0.x : p0.y + k * p0.z) + r0 : (k1 == 0 ? p1.x : p1.y + k1 * p1.z) + r1;
                ml[i] = w.ml[p];
                if constexpr (N == 4) *(float4 *)x[i] = *(const float4 *)(w.o + p * HD + lane * 4);
                else *(float2 *)x[i] = *(const float2 *)(w.o + p * HD + lane * 2);
            }
        }
        const float top = fmaxf(M, fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)));
        const float f = M == -INFINITY ? 0.f : ap_ex2(M - top);
        L *= f;
#pragma unroll
        for (int d = 0; d < N; ++d) o[d] *= f;
        M = top;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k0 + i < all) {
                // a part without a key that its row sees holds a sum of products with 0
                const float g = ml[i].x == -INFINITY ? 0.f : ap_ex2(ml[i].x - M);
                L = fmaf(g, ml[i].y, L);
#pragma unroll
                for (int d = 0; d < N; ++d) o[d] = fmaf(g, x[i][d], o[d]);
            }
    }
    const float by = L == 0.f ? (list && list[0] < 0 ? 0.f : NAN) : 1.f / L;
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] *= by;
    if (a.q_f32) {
        float *dst = (float *)a.out + orow + lane * N;
        if constexpr (N == 4) *(float4 *)dst = make_float4(o[0], o[1], o[2], o[3]);
        else *(float2 *)dst = make_float2(o[0], o[1]);
    } else {
        uint16_t *dst = (uint16_t *)a.out + orow + lane * N;
        if constexpr (N == 4) *(uint2 *)dst = make_uint2(kv8_bf2(o[0], o[1]), kv8_bf2(o[2], o[3]));
        else *(uint32_t *)dst = kv8_bf2(o[0], o[1]);
    }
}

// by row: rows have parts of a shared prefix and of their own pages; else by unit that several workers have, AP_JOIN blocks each
constexpr int AP_JOIN = 8;
template <int HD>
__global__ void __launch_bounds__(512, 2) attend_join_kernel(const KvAttendArgs a, const ApWork w, int by_row, int sms) {
    const int warp = threadIdx.x >> 5, G = a.Hq / a.Hkv, lg = __ffs(G) - 1;
    pdl_wait();
    pdl_trigger();
    const int bad = w.head->bad;
    auto cleared = [&](int b) { return bad == 2 || w.bad[b] || w.bad_pre[w.seqs[b].lead]; };
    const int4 none = make_int4(0, 0, 0, 0);
    if (by_row) {
        // a block a row, a warp its heads
        const int to = blockIdx.x, b = to / a.max_rows, j = to - b * a.max_rows;
        const ApSeq s = w.seqs[b];
        if (j < s.n && !(bad && cleared(b)))
#pragma unroll 1
            for (int h = warp; h < a.Hq; h += blockDim.x / 32) {
                const int kvh = h >> lg, g = h & (G - 1);
                const int i1 = (j << lg) + g, i0 = ((s.row + j - s.pre_row) << lg) + g;
                const int q1 = s.tiles == 1 ? 0 : i1 / s.size, q0 = s.pre_tiles == 1 ? 0 : i0 / s.pre_size;
                const int4 p1 = w.parts[s.unit + kvh * s.tiles + q1];
                const int4 p0 = s.pre_unit < 0 ? none : w.parts[s.pre_unit + kvh * s.pre_tiles + q0];
                if (p1.x >= 0) ap_join<HD>(a, w, p0, i0 - q0 * s.pre_size, p1, i1 - q1 * s.size, ((size_t)to * a.Hq + h) * HD, nullptr);
            }
    } else {
        int first = 0;
        for (int k = 0; k < AP_BLOCKS; ++k) {
            const int items = w.head->split[k] * AP_JOIN;
            for (int x = (int)((blockIdx.x + gridDim.x - first % gridDim.x) % gridDim.x); x < items; x += gridDim.x) {
                const ApUnit u = w.units[w.split[k * 3 * sms + x / AP_JOIN]];
                const int4 p = w.parts[u.id];
                for (int r = x % AP_JOIN * 8 + warp; r < u.nq; r += 8 * AP_JOIN) {
                    const int iq = u.i0 + r, to = a.pages ? u.row0 : u.seq * a.max_rows + (iq >> lg);
                    if (bad && cleared(u.seq)) continue;
                    ap_join<HD>(a, w, none, 0, p, r, ((size_t)to * a.Hq + u.kvh * G + (iq & (G - 1))) * HD,
                                a.pages ? a.pages + ((size_t)u.row0 * a.Hkv + u.kvh) * a.n_select : nullptr);
                }
            }
            first += items;
        }
    }
    if (!bad) return;
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        if (!cleared(b)) continue;
        const SeqRows r = seq_rows(a.n_rows[b], a.seq_len[b], a.advanced, a.max_rows, a.max_pages);
        const size_t n = (size_t)r.n * a.Hq * HD, at = (size_t)b * a.max_rows * a.Hq * HD;
        for (size_t i = threadIdx.x; i < n; i += blockDim.x) {
            if (a.q_f32) ((float *)a.out)[at + i] = 0.f;
            else ((uint16_t *)a.out)[at + i] = 0;
        }
    }
}

template <typename... P, typename... A>
static cudaError_t ap_launch(void (*k)(P...), int grid, int threads, size_t smem, cudaStream_t s, const A &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k, args...);
    count_launch();
    return e;
}

template <typename C>
static cudaError_t launch_attend_t(const KvAttendArgs &a, const ApWork &w, int sms, cudaStream_t s) {
    static std::atomic<int> done[kMaxDevices];
    auto *rows = attend_plan_kernel<C::QR, C::PAIRS, C::PG, false>, *lists = attend_plan_kernel<C::QR, C::PAIRS, C::PG, true>;
    cudaError_t e = once_per_device(done, [rows, lists] {
        cudaError_t x = cudaFuncSetAttribute(rows, cudaFuncAttributeMaxDynamicSharedMemorySize, (10 * AP_MAXB + 1) * 4);
        if (x == cudaSuccess) x = cudaFuncSetAttribute(lists, cudaFuncAttributeMaxDynamicSharedMemorySize, (10 * AP_MAXB + 1) * 4);
        return x != cudaSuccess ? x : cudaFuncSetAttribute(attend_kernel<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    });
    if (e != cudaSuccess) return e;
    CUtensorMap mk, mv;
    const int keys = a.n_pages * a.Hkv * 16;
    if (!tc_encode_rows(&mk, a.k_pages, keys, 16, C::HD) || !tc_encode_pages(&mv, a.v_pages, keys, C::HD)) return cudaErrorInvalidValue;
    if ((e = ap_launch(a.pages ? lists : rows, (long long)a.B * a.max_rows * a.Hq > 128 ? AP_BLOCKS : 1, AP_PLAN, (size_t)(10 * a.B + 1) * 4, s, a, w, sms)) != cudaSuccess) return e;
    if ((e = ap_launch(attend_kernel<C>, sms, C::THREADS, C::SMEM, s, mk, mv, a, w, sms)) != cudaSuccess) return e;
    const int by_row = a.share && a.max_rows * (a.Hq / a.Hkv) < AP_SHARE;
    const int grid = by_row ? a.B * a.max_rows : 4 * sms;
    // by row a warp a head, up to 16: one after another they wait for their parts
    return ap_launch(attend_join_kernel<C::HD>, grid, by_row ? 32 * std::min(a.Hq, 16) : 256, 0, s, a, w, by_row, sms);
}

cudaError_t launch_kv_attend(const KvAttendArgs &a, void *workspace, int sms, cudaStream_t s) {
    ApWork w;
    ap_layout(a.B, a.max_rows, a.Hq, a.Hkv, a.hd, a.pages != nullptr, sms, workspace, &w);
    if (a.hd == 128) return a.q_f32 ? launch_attend_t<AP<128, true>>(a, w, sms, s) : launch_attend_t<AP<128, false>>(a, w, sms, s);
    return a.q_f32 ? launch_attend_t<AP<64, true>>(a, w, sms, s) : launch_attend_t<AP<64, false>>(a, w, sms, s);
}

}  // namespace osp
