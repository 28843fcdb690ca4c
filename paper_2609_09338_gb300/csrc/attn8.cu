// Causal attention of a sequence's newest rows over the 8-bit paged cache.
//
//   out_i = sum_j w_ij V_j / sum_j w_ij,  w_ij = exp(q_i . K_j / sqrt(hd)),  j <= position of i
//
// A cluster of blocks takes up to QT (row, head) queries of one KV head, each block a
// range of the finished pages, the last one the tail's bf16 rows too (on the CUDA
// cores, while its first pages are on their way).  The blocks' (max, sum, output) are
// merged through distributed shared memory: a call is one launch without a workspace.
//
// The pages are operands as they lie (kv8.cuh): bulk copies bring 8 of them, 128 keys,
// to shared memory and tcgen05.mma kind::f8f6f4 reads them there, K as 128 rows of the
// scores' product, V transposed as head_dim rows of the output's.  What is not 8 bits
// wide comes as e4m3 planes, the operand's other side: x 2^e = x0 + x1/16 + x2/256 ...,
// each plane the nearest e4m3 (4 significant bits) of 16 times what the one before it
// left.  Planes have columns of their own (N = planes x queries) and are put together in
// float32, so no product of unlike sizes shares an accumulator.  A bf16 query, scaled to
// a magnitude of 128 to 256, is two planes: exactly where an element is 2^-13 of its row's
// largest or more, within 2^-21 of the largest elsewhere (two planes end at 2^-13).
//
// Per tile of 128 keys a thread is a key: it reads its scores from TMEM and writes its
// weights' planes; then it is a dim, and adds the output of the tile before from TMEM to
// registers in float32.  Weights are 2^(s - m) with a reference m that stays while no
// score exceeds it by more than A8_OVER: then a tile needs one vote, and no maxima.
// The planes have a last step of their own, 2^-25 of the reference for four, 2^-33 for
// six, so the reference has to come down too: behind a key that takes nearly all of the
// weight the others' are 2^-20 of it and less, and their sum may be the whole output (16 k
// keys behind one of 0.99 and value 0: an output off by 1.5e-1 of itself with three planes
// and no such step, 9e-3 with four).  In the third tile, every A8_RENEW from there, and in
// the one behind a tile that raised it, the reference becomes the tile's maximum, however
// low, down to 2^-A8_DROP of the largest: float32 holds sums that much larger than the
// reference.  References are whole but the tail's, so sums are scaled by powers of two.
// (One thread a query finds the new references, all read what it left: with each thread
// finding all of them, which takes its registers, the many-row calls below took 187 and 229 us.)
// The V block's scale goes into the weight, w' = 2^(s + log2(vs) - m); the sum adds
// w' / vs.
//
// Measured (GB300, keys of 8 KV heads of 128).  One row of 64 sequences of 1024..16384
// keys: 174 us, 6.55 TB/s, bound by memory (0.97 of a plain copy's rate).  Groups of four,
// 1..8 rows of 96 sequences of 1024..4096 keys: 172 us; 50..64 rows of 8 sequences of
// 2000..8192 keys: 206 us (160 and 190 with three planes of the weights, 12 bits instead of
// 16).  Both wait for a tile's chain, scores to weights to outputs: half of the issue slots
// are used, 375 instructions a warp and tile, 15 % of the tensor pipe.
// float32 queries, groups of four, 16 sequences of 2048..8192 keys of 4 heads: 26 us.  A
// call of one sequence takes 6.3 us.  Taking sequences longest first (a ranking in each
// block) made the first 183 us, and with three planes the second 163, the third, which was
// 187 to 207 with the sequences' order, 189: sequences are taken as they come.
#include <cooperative_groups.h>

#include <algorithm>

#include "attn8.cuh"
#include "attn8_forms.h"
#include "internal.h"
#include "tcgen05.cuh"
#include "tma.cuh"

namespace osp {

namespace cg = cooperative_groups;

// Smallest log2 of a V scale that moves the reference.  Lower, and the sum of the weights (up to
// 2^(A8_OVER - A8_LO + A8_DROP) a key) or a weight beside one of V scale 2^40 would leave
// float32's range; the values of such a block have steps of 2^(A8_LO - 25) in the output.
constexpr float A8_LO = -60.f;
constexpr float A8_OVER = 4.f;       // a weight is at most 2^A8_OVER, times A8_UP an e4m3 number
constexpr float A8_DROP = 40.f;      // a reference is at least 2^-A8_DROP of the largest one so far
constexpr int A8_RENEW = 16;         // tiles a reference stays at most
constexpr float A8_UP = 16.f;

// Shared-memory matrix descriptor of an operand without swizzle.  K-major: core matrices
// of 8 rows x 16 bytes, lbo bytes apart along the reduction, sbo along the rows.  The
// weights lie the other way round, 8 keys x 16 columns (lbo still along the reduction), so
// that a thread, which is a key, writes its queries' weights side by side.
__device__ __forceinline__ uint64_t a8_desc(uint32_t addr, uint32_t lbo, uint32_t sbo) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(sbo >> 4) << 32 | (uint64_t)1 << 46;
}
// kind::f8f6f4, e4m3 operands, A K-major, B K-major or columns side by side, float32 accumulator, M 128
__host__ __device__ constexpr uint32_t a8_idesc(int N, bool columns) {
    return (1u << 4) | (columns ? 1u << 16 : 0u) | (uint32_t)(N >> 3) << 17 | (128u >> 4) << 24;
}
__device__ __forceinline__ void a8_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(d),
                 "l"(a), "l"(b), "r"(idesc), "r"(acc)
                 : "memory");
}
__device__ __forceinline__ void a8_alloc(uint32_t *at, int columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(at)), "r"((uint32_t)columns)
                 : "memory");
}
__device__ __forceinline__ void a8_dealloc(uint32_t at, int columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"((uint32_t)columns) : "memory");
}
__device__ __forceinline__ float a8_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float a8_warp_max(float x) {
    float y;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <int N>
__device__ __forceinline__ void a8_ld(uint32_t addr, float *v) {
    uint32_t r[N];
    if constexpr (N == 4) {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
    } else {
        static_assert(N == 8, "columns");
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "r"(addr));
    }
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = __uint_as_float(r[j]);
}

// The nearest e4m3 of four floats as a word of codes; `rest`: what they leave, 16 times, in their place.
__device__ __forceinline__ uint32_t a8_quad(f2 &x, f2 &y, bool rest) {
    float x0, x1, y0, y1, f0, f1, g0, g1;
    un2(x, x0, x1);
    un2(y, y0, y1);
    uint32_t w;
    asm("{\n.reg .b16 a, b, c, d;\n.reg .b32 h;\n"
        "cvt.rn.satfinite.e4m3x2.f32 a, %6, %5;\ncvt.rn.satfinite.e4m3x2.f32 b, %8, %7;\nmov.b32 %0, {a, b};\n"
        "cvt.rn.f16x2.e4m3x2 h, a;\nmov.b32 {c, d}, h;\ncvt.f32.f16 %1, c;\ncvt.f32.f16 %2, d;\n"
        "cvt.rn.f16x2.e4m3x2 h, b;\nmov.b32 {c, d}, h;\ncvt.f32.f16 %3, c;\ncvt.f32.f16 %4, d;\n}"
        : "=r"(w), "=f"(f0), "=f"(f1), "=f"(g0), "=f"(g1)
        : "f"(x0), "f"(x1), "f"(y0), "f"(y1));
    if (rest) {
        const f2 sixteen = mk2(16.f, 16.f), minus = mk2(-16.f, -16.f);
        x = fma2(mk2(f0, f1), minus, mul2(x, sixteen));
        y = fma2(mk2(g0, g1), minus, mul2(y, sixteen));
    }
    return w;
}

// Planes of QW queries from TMEM column `col` on, QT columns a plane: x = sum over planes of 16^-p plane p, in pairs
template <int QT, int QW, int P>
__device__ __forceinline__ void a8_planes(uint32_t col, f2 (&x)[QW / 2]) {
    float v[P][QW];
#pragma unroll
    for (int p = 0; p < P; ++p) a8_ld<QW>(col + p * QT, v[p]);
    tc_ld_wait();
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int q = 0; q < QW; ++q) asm volatile("" : "+f"(v[p][q]));   // not before the wait
    const f2 sixteenth = mk2(0.0625f, 0.0625f);
#pragma unroll
    for (int q = 0; q < QW / 2; ++q) {
        x[q] = mk2(v[P - 1][2 * q], v[P - 1][2 * q + 1]);
#pragma unroll
        for (int p = P - 2; p >= 0; --p) x[q] = fma2(x[q], sixteenth, mk2(v[p][2 * q], v[p][2 * q + 1]));
    }
}

// A barrier of a warpgroup that tells whether any thread's flag is set.
__device__ __forceinline__ bool a8_vote(int id, bool x) {
    uint32_t r;
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbarrier.cta.red.or.pred q, %2, 128, p;\nselp.u32 %0, 1, 0, q;\n}"
                 : "=r"(r) : "r"((uint32_t)x), "r"(id) : "memory");
    return r != 0;
}

// Waits for a phase, about a second at most: then, or when another wait of the block has
// run out, false.  A phase that has ended costs one instruction.
__device__ __forceinline__ bool a8_wait(uint64_t *bar, uint32_t parity, int *abort, int32_t *status) {
    long long t0 = 0;
    for (int i = 0; !mbar_try_wait(bar, parity);) {
        if (++i < 64) continue;
        if (*(volatile int *)abort) return false;
        const long long t = clock64();
        if (!t0) t0 = t;
        if (t - t0 > 2000000000LL) {
            *(volatile int *)abort = 1;
            set_status(status, OSPREY_ERR_TIMEOUT);
            return false;
        }
        i = 0;
    }
    return true;
}

template <typename C>
__global__ void __launch_bounds__(C::THREADS, C::BPS) attn8_kernel(const __grid_constant__ Attn8Args a, int tiles) {
    constexpr int HD = C::HD, QT = C::QT, QW = C::QW, QP = C::QP, PP = C::PP, KB = C::KB, TB = C::TB, NS = C::NS;
    constexpr int W_MMA = C::CT / 32, W_K = W_MMA + 1;   // the warps that do not compute: products, K copies, V copies
    extern __shared__ __align__(1024) uint8_t sm[];
    uint8_t *sk = sm, *sv = sk + NS * TB, *sqp = sv + NS * TB, *spp = sqp + C::QB;
    float *sq = (float *)spp;                       // [QT][HD] while the tail is read
    float *sp = (float *)(spp + C::PB);             // [QT][A8_CH] the tail's weights
    float *so = (float *)sk;                        // [QT][HD] at the end
    __shared__ __align__(8) uint64_t kfull[NS], vfull[NS], kfree[NS], vfree[NS], sfull[2], pready, ofull;
    __shared__ __align__(16) float s_red[C::NWG][4][QW], s_mul[QT], s_nref[QT], s_m[QT], s_best[QT], s_corr[QT], s_by[QT];
    __shared__ float s_l[QT], s_lw[4][QT];
    __shared__ int s_pos[QT], s_bad, s_abort;
    __shared__ uint32_t s_tmem[2];
    cg::cluster_group cluster = cg::this_cluster();
    const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int unit = blockIdx.x / cs, kvh = unit % a.Hkv, tile = unit / a.Hkv % tiles, b = unit / a.Hkv / tiles;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, lg = __ffs(a.Hq / a.Hkv) - 1, G = 1 << lg;   // a power of two
    int nr, base, c8;
    bool ok = true;
    if (a.seq_len) {
        // Everything that this call reads may come from the kernel before, which this one may
        // have started beside: nothing is read before this wait, which makes that kernel's
        // writes visible to plain loads, and to the copies behind a proxy fence.  (Queries and
        // the tail through L2 alone: groups of rows 171 -> 182 us, 206 -> 214.)
        pdl_wait();
        asm volatile("fence.proxy.async.global;" ::: "memory");
        nr = __ldcg(a.n_rows + b);
        const int len = __ldcg(a.seq_len + b);
        const int64_t total = (int64_t)len + (a.advanced ? 0 : max(nr, 0));
        ok = nr >= 0 && nr <= a.max_rows && len >= 0 && total >= nr && total <= (int64_t)a.max_pages * 16;
        if (!ok && rank == 0 && tid == 0)
            set_status(a.status, nr < 0 || nr > a.max_rows || len < 0 || total < nr ? OSPREY_ERR_INVALID_ARG : OSPREY_ERR_CAPACITY);
        if (!ok) nr = min(max(nr, 0), a.max_rows);
        base = (int)(ok ? total - nr : 0);
        c8 = (int)(ok ? total / 16 : 0);
    } else {
        const int nn = a.map.valid[b] ? a.map.nnew[b] : 0;
        nr = a.map.step == 0 ? nn : min(nn, 1);
        base = a.map.pos0[b] + (a.map.step == 0 ? 0 : nn + a.map.step - 1);
        c8 = a.map.pos0[b] / 16;
    }
    const int i0 = tile * QT, nq = min(QT, nr * G - i0), nact = (nq + QW - 1) / QW;   // queries, warpgroups that have some
    if (nq <= 0) {   // the whole cluster
        pdl_wait();
        return;
    }
    // this block's finished pages; keys past the last query's position are seen by none
    const int last = base + ((i0 + nq - 1) >> lg);
    const int np_all = ok ? min(c8, last / 16 + 1) : 0, per = (np_all + cs - 1) / cs;
    const int pg0 = min(np_all, rank * per), np = min(np_all, pg0 + per) - pg0, nt = (np + 7) / 8;
    const int32_t *tab = a.page_table + (size_t)b * a.max_pages + pg0;
    // a block's number of a page id; a bad id is noted and read as page 0 (the check waits for the id, so it comes at its use)
    bool bad_id = false;
    auto block_of = [&](int id) {
        const bool good = id >= 0 && id < a.n_pages;
        bad_id |= !good;
        return (size_t)(good ? id : 0) * a.Hkv + kvh;
    };
    // Copies of a tile's K or V pages from the page ids that lanes 0 .. 7 hold, issued by one
    // lane: a copy takes a warp some 130 cycles to issue, whichever lane's, so K and V have
    // a warp each (one warp for both, and for the products: 3500 cycles a tile).
    uint8_t *const ring = warp == W_K ? sk : sv;
    uint64_t *const full = warp == W_K ? kfull : vfull, *const freed = warp == W_K ? kfree : vfree;
    auto load = [&](int t, int id) {
        const int n = min(8, np - t * 8), slot = t % NS;
        const unsigned long long at = (unsigned long long)((warp == W_K ? a.k8 : a.v8) + block_of(id) * KB);
        unsigned long long from[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) from[p] = __shfl_sync(0xffffffffu, at, p);
        if (tc_elect()) {
            mbar_arrive_expect_tx(&full[slot], (uint32_t)(n * KB));
#pragma unroll
            for (int p = 0; p < 8; ++p)
                if (p < n) bulk_g2s(ring + slot * TB + p * KB, (const void *)from[p], KB, &full[slot]);
        }
        __syncwarp();
    };
    auto lane_id = [&](int t) { return lane < 8 && t * 8 + lane < np ? __ldcg(tab + t * 8 + lane) : 0; };
    int ids = 0;   // of the next tile to ask for
    if (warp == W_MMA) {
        if (lane == 0) {
            mbar_init(&sfull[0], 1);
            mbar_init(&sfull[1], 1);
            mbar_init(&ofull, 1);
            mbar_init(&pready, 4 * nact);
            s_bad = !ok;
            s_abort = 0;
            mbar_fence_init();
        }
        __syncwarp();
        a8_alloc(&s_tmem[0], C::SCOLS);
        a8_alloc(&s_tmem[1], C::OCOLS);
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else if (warp >= W_K) {
        int first[NS];
#pragma unroll
        for (int t = 0; t < NS; ++t) first[t] = lane_id(t);
        ids = lane_id(NS);
        if (lane == 0) {
            for (int i = 0; i < NS; ++i) {
                mbar_init(&full[i], 1);
                mbar_init(&freed[i], 1);
            }
            mbar_fence_init();
        }
        __syncwarp();
        // finished pages are written by no kernel that this one may overlap
#pragma unroll
        for (int t = 0; t < NS; ++t)
            if (t < nt) load(t, first[t]);
    }
    // compute threads: the thread's key of tile t; its page's scales are loaded a tile ahead, the page's id two
    const int wt = tid & 127;
    float ksn = 0.f, vsn = 1.f;
    auto key_id = [&](int t) { return t * 8 + (wt >> 4) < np ? __ldcg(tab + t * 8 + (wt >> 4)) : 0; };
    auto scales = [&](int t) {
        if (t * 8 + (wt >> 4) < np) {
            const size_t blk = block_of(ids);
            ksn = __ldcg(a.k_scale + blk);
            vsn = __ldcg(a.v_scale + blk);
        }
    };
    const bool tail = ok && rank == cs - 1;
    if (warp < W_MMA) {
        ids = key_id(0);
        if (!a.seq_len) pdl_wait();   // queries and the tail's rows come from a draft call's kernels
        // queries: rotated, scaled to a magnitude of 128 to 256, split into planes; a lane holds pairs (d, d + HD / 2)
        constexpr int NP = HD / 64, PER = (QT + W_MMA - 1) / W_MMA;
        float xs[PER][2 * NP];
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int q = warp + u * W_MMA, i = min(i0 + q, a.max_rows * G - 1), j = i >> lg, g = i & (G - 1);
            const int64_t at = ((int64_t)b * a.max_rows + j) * a.q_stride + (kvh * G + g) * HD + lane;
#pragma unroll
            for (int k = 0; k < 2 * NP; ++k) {
                const int64_t e = at + 32 * (k % NP) + (k / NP) * (HD / 2);
                xs[u][k] = q >= nq ? 0.f : a.q_f32 ? ((const float *)a.q)[e] : bf_to_f(((const uint16_t *)a.q)[e]);
            }
        }
        scales(0);
        ids = key_id(1);
        // A bad id clears all rows of its sequence, so pages that this tile's rows do not see are checked too.
        // (A draft call's first kernel has checked them.)
        if (a.seq_len)
            for (int p = np_all + rank * C::CT + tid; p < c8; p += cs * C::CT)
                block_of(__ldcg(a.page_table + (size_t)b * a.max_pages + p));
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int q = warp + u * W_MMA, j = (i0 + q) >> lg;
            if (q >= QT) break;
            float (&x)[2 * NP] = xs[u];
            float mag = 0.f;
            bool fin = true;
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                if (a.rotate) {
                    float c, s;
                    rope_cs_fix(a.freq[lane + 32 * k], base + j, c, s);
                    const float t = x[k] * c - x[NP + k] * s;
                    x[NP + k] = x[NP + k] * c + x[k] * s;
                    x[k] = t;
                }
                fin = fin && isfinite(x[k]) && isfinite(x[NP + k]);
                mag = fmaxf(mag, fmaxf(fabsf(x[k]), fabsf(x[NP + k])));
            }
            mag = a8_warp_max(mag);
            fin = __all_sync(0xffffffffu, fin);
            const float unit = rsqrtf((float)HD) * 1.4426950408889634f;   // weights are powers of two
            const int e = fin && mag >= 0x1p-100f ? 7 - ((int)(__float_as_uint(mag) >> 23) - 127) : fin ? 107 : 0;
            const float up = kv8_pow2(e);
#pragma unroll
            for (int k = 0; k < 2 * NP; ++k) {
                const int d = lane + 32 * (k % NP) + (k / NP) * (HD / 2);
                if (tail) sq[q * HD + d] = x[k] * unit;
                float r = fin ? x[k] * up : 0.f;
#pragma unroll
                for (int p = 0; p < QP; ++p) {
                    const int n = p * QT + q;
                    const uint32_t c = e4m3x2(r, 0.f);
                    sqp[(n >> 3) * (HD * 8) + (d >> 4) * 128 + (n & 7) * 16 + (d & 15)] = (uint8_t)c;
                    r = (r - e4m3x2_f(c).x) * 16.f;
                }
            }
            if (lane == 0) {
                s_mul[q] = fin ? unit * kv8_pow2(-e) : __uint_as_float(0x7fffffffu);
                s_pos[q] = base + j;
                s_m[q] = s_best[q] = -INFINITY;
                s_nref[q] = 0.f;
                s_l[q] = 0.f;
            }
        }
        fence_async_smem();
    }
    if (warp >= W_MMA) pdl_wait();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // not before this block holds its TMEM: a dependent's blocks take theirs and wait for this kernel
    pdl_trigger();
    const uint32_t tmem = s_tmem[0], tm_o = s_tmem[1];
    // After a wait that ran out nothing is waited for or issued any more: the loops run to
    // their ends, and the cluster's outputs are 0.
    auto wait1 = [&](uint64_t *bar, uint32_t phase) { return a8_wait(bar, phase & 1, &s_abort, a.status); };
    auto wait = [&](uint64_t *bar, uint32_t phase) {
        wait1(bar, phase);
        __syncwarp();
    };
    float keep[QW];   // a block alone: its outputs
    auto stop = [&] { return __shfl_sync(0xffffffffu, *(volatile int *)&s_abort, 0) != 0; };
    if (warp == W_MMA) {
        // One lane issues the products, slots and descriptors by increments: with the whole
        // warp in the loop, slots by division, a tile's two products took 1750 cycles to issue.
        if (tc_elect()) {
            const uint64_t dK = a8_desc(smem_u32(sk), 128, HD * 8), dQ = a8_desc(smem_u32(sqp), 128, HD * 8);
            const uint64_t dV = a8_desc(smem_u32(sv), KB, 128), dP = a8_desc(smem_u32(spp), 128, A8_PG);
            int ks = 0, kph = 0, vs = 0, vph = 0;   // slots and their phases
            auto scores = [&](int t) {   // of tile t: 128 keys x (planes x queries)
                const int sb = t & 1;
                if (!wait1(&kfull[ks], kph)) return false;
                // the columns' last readers had read them before they wrote the weights of tile t - 2
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < HD / 32; ++k)
                    a8_mma(tmem + sb * C::SC, dK + (ks * TB + k * 256) / 16, dQ + k * 16, a8_idesc(C::SC, false), k > 0);
                tc_commit(&sfull[sb]);
                tc_commit(&kfree[ks]);
                if (++ks == NS) ks = 0, kph ^= 1;
                return true;
            };
            bool go = nt > 0 && scores(0);
            for (int t = 0; t < nt && go; ++t) {
                if (t + 1 < nt) go = scores(t + 1);
                // head_dim x (planes x queries) over tile t's keys, when its weights are written and the output before is read
                go = go && wait1(&vfull[vs], vph) && wait1(&pready, t);
                if (!go) break;
                tc_fence_after();
                const int n = (np - t * 8 + 1) / 2;
                if (n >= 4) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        a8_mma(tm_o, dV + (vs * TB + k * 2 * KB) / 16, dP + k * 32, a8_idesc(C::OC, true), k > 0);
                } else
                    for (int k = 0; k < n; ++k) a8_mma(tm_o, dV + (vs * TB + k * 2 * KB) / 16, dP + k * 32, a8_idesc(C::OC, true), k > 0);
                tc_commit(&ofull);
                tc_commit(&vfree[vs]);
                if (++vs == NS) vs = 0, vph ^= 1;
            }
        }
        __syncwarp();
    } else if (warp >= W_K) {
        for (int t = 0; t + NS < nt; ++t) {   // a slot is asked for again when the product that read it has ended
            wait(&freed[t % NS], t / NS);
            if (stop()) break;
            load(t + NS, ids);
            ids = lane_id(t + NS + 1);
        }
    } else if (warp < 4 * nact) {   // the columns of a warpgroup without queries hold anything, and nobody reads them
        const int wg = warp / 4, ww = warp % 4, q0 = wg * QW, bar = 1 + wg;   // this warpgroup's queries and barrier
        float o[QW];
#pragma unroll
        for (int q = 0; q < QW; ++q) o[q] = 0.f;
        if (tail)   // bf16 rows behind the finished pages, in float32
            for (int key0 = c8 * 16; key0 <= last; key0 += A8_CH) {
                const int key1 = min(last + 1, key0 + A8_CH);
                // a key is four lanes': every fourth group of 4 dims
                const int key = key0 + wt / 4, quarter = wt % 4;
                float s[QW];
#pragma unroll
                for (int q = 0; q < QW; ++q) s[q] = 0.f;
                if (key < key1) {
                    const uint16_t *kr = a.k_tail +
                                         (((size_t)b * a.tail_pages + key / 16 % a.tail_pages) * a.Hkv + kvh) * 16 * HD + (key % 16) * HD;
#pragma unroll 2
                    for (int d = quarter * 4; d < HD; d += 16) {
                        const uint2 w = *(const uint2 *)(kr + d);
                        const float f0 = bf_lo(w.x), f1 = bf_hi(w.x), f2 = bf_lo(w.y), f3 = bf_hi(w.y);
#pragma unroll
                        for (int q = 0; q < QW; ++q) {
                            const float4 u = *(const float4 *)&sq[(q0 + q) * HD + d];
                            s[q] = fmaf(u.x, f0, fmaf(u.y, f1, fmaf(u.z, f2, fmaf(u.w, f3, s[q]))));
                        }
                    }
                }
#pragma unroll
                for (int q = 0; q < QW; ++q) {
                    s[q] += __shfl_xor_sync(0xffffffffu, s[q], 1);
                    s[q] += __shfl_xor_sync(0xffffffffu, s[q], 2);
                    if (quarter == 0) sp[(q0 + q) * A8_CH + wt / 4] = s[q];
                }
                named_sync(bar, 128);
                for (int q = q0 + ww; q < q0 + QW; q += 4) {
                    const bool see = key0 + lane < key1 && key0 + lane <= s_pos[q];
                    const float x = see ? sp[q * A8_CH + lane] : -INFINITY;
                    const float mn = fmaxf(s_m[q], warp_max(x)), ref = mn == -INFINITY ? 0.f : mn;
                    const float p = see ? a8_ex2(x - ref) : 0.f, corr = s_m[q] == -INFINITY ? 0.f : a8_ex2(s_m[q] - ref);
                    const float ls = warp_sum(p);
                    __syncwarp();
                    sp[q * A8_CH + lane] = see ? p : -1.f;   // a masked key is not multiplied: its value may be anything
                    if (lane == 0) {
                        s_corr[q] = corr;
                        s_l[q] = s_l[q] * corr + ls;
                        s_m[q] = s_best[q] = mn;
                        s_nref[q] = -ref;
                    }
                }
                named_sync(bar, 128);
                if (wt < HD) {
#pragma unroll
                    for (int q = 0; q < QW; ++q) o[q] *= s_corr[q0 + q];
                    for (int k = 0; k < key1 - key0; ++k) {
                        const int kk = key0 + k;
                        const float v = bf_to_f(a.v_tail[(((size_t)b * a.tail_pages + kk / 16 % a.tail_pages) * a.Hkv + kvh) * 16 * HD +
                                                         (kk % 16) * HD + wt]);
#pragma unroll
                        for (int q = 0; q < QW; ++q) {
                            const float p = sp[(q0 + q) * A8_CH + k];
                            if (!(p < 0.f)) o[q] = fmaf(p, v, o[q]);
                        }
                    }
                }
                named_sync(bar, 128);
            }
        if (C::NWG > 1 && tail) named_sync(15, 128 * nact);   // every warpgroup has read q, whose place the weights take
        constexpr int QH = QW / 2;
        f2 o2[QH], l2[QH];   // pairs of queries
#pragma unroll
        for (int q = 0; q < QH; ++q) {
            o2[q] = mk2(o[2 * q], o[2 * q + 1]);
            l2[q] = wt == 0 ? mk2(s_l[q0 + 2 * q], s_l[q0 + 2 * q + 1]) : 0ull;
        }
        const uint32_t lanes = (uint32_t)(ww * 32) << 16;
        const int first_pos = base + (i0 >> lg);
        const f2 down = mk2(1.f / A8_UP, 1.f / A8_UP);
        bool raised = false;   // the tile before exceeded its references
        for (int t = 0; t < nt; ++t) {
            const float ks = ksn, vs = vsn;
            scales(t + 1);
            ids = key_id(t + 2);
            const int n = min(8, np - t * 8), key = (pg0 + t * 8) * 16 + wt;
            // a scale under 2^A8_LO (a block of zeros) would push the weight out of float32's range;
            // a NaN scale comes through the score, to the queries that see the key alone
            float lvs, rvs;
            asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(lvs) : "f"(vs));
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rvs) : "f"(vs));
            float fvs = A8_UP;
            if (!(lvs >= A8_LO)) {
                fvs = lvs < A8_LO ? vs * 0x1p60f * A8_UP : A8_UP;
                rvs = lvs < A8_LO ? 0x1p60f : 1.f;
                lvs = lvs < A8_LO ? A8_LO : lvs;
            }
            f2 e2[QH];   // log2 of the weights
            wait(&sfull[t & 1], t >> 1);
            tc_fence_after();
            a8_planes<QT, QW, QP>(tmem + lanes + (t & 1) * C::SC + q0, e2);
            const f2 ks2 = mk2(ks, ks), lv2 = mk2(lvs, lvs);
            float e[QW];
#pragma unroll
            for (int q = 0; q < QH; q += 2) {
                const ulonglong2 mu = *(const ulonglong2 *)&s_mul[q0 + 2 * q], rf = *(const ulonglong2 *)&s_nref[q0 + 2 * q];
                e2[q] = fma2(e2[q], mul2(mu.x, ks2), add2(lv2, rf.x));
                e2[q + 1] = fma2(e2[q + 1], mul2(mu.y, ks2), add2(lv2, rf.y));
            }
#pragma unroll
            for (int q = 0; q < QH; ++q) un2(e2[q], e[2 * q], e[2 * q + 1]);
            if ((pg0 + t * 8 + n) * 16 - 1 > first_pos || n < 8) {   // a key that is no one's, or not every query's
                const bool in = wt < n * 16;
#pragma unroll
                for (int q = 0; q < QW; ++q)
                    if (!in || key > s_pos[q0 + q]) e[q] = -INFINITY;
            }
            float top = e[0];
#pragma unroll
            for (int q = 1; q + 1 < QW; q += 2) asm("max.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(e[q]), "f"(e[q + 1]));
            top = fmaxf(top, e[QW - 1]);
            const bool renew = t == 0 || t % A8_RENEW == 2 || raised, over = a8_vote(bar, renew || top > A8_OVER);
            raised = over && !renew;
            if (t > 0) {   // the output of the tile before: a thread is a dim
                wait(&ofull, t - 1);
                tc_fence_after();
                f2 x[QH];
                a8_planes<QT, QW, PP>(tm_o + lanes + q0, x);
#pragma unroll
                for (int q = 0; q < QH; ++q) o2[q] = fma2(x[q], down, o2[q]);
            }
            if (over) {   // new references: the tile's maxima
#pragma unroll
                for (int q = 0; q < QW; ++q) {
                    const float x = a8_warp_max(e[q]);
                    if (lane == 0) s_red[wg][ww][q] = x;
                }
                named_sync(bar, 128);
                if (wt < QW) {   // a thread each; the old references have been read
                    const int q = q0 + wt;
                    const float x = fmaxf(fmaxf(s_red[wg][0][wt], s_red[wg][1][wt]), fmaxf(s_red[wg][2][wt], s_red[wg][3][wt]));
                    const float m = s_m[q], ref = -s_nref[q], r = rintf(ref + x), best = fmaxf(s_best[q], r);
                    const float to = x == -INFINITY ? m : fmaxf(r, best - A8_DROP);   // the query sees none of the tile's keys
                    s_corr[q] = to == m ? 1.f : m == -INFINITY ? 0.f : a8_ex2(m - to);
                    s_by[q] = to == -INFINITY ? 0.f : to - ref;
                    s_m[q] = to;
                    s_nref[q] = to == -INFINITY ? 0.f : -to;
                    s_best[q] = best;
                }
                named_sync(bar, 128);
#pragma unroll
                for (int q = 0; q < QW; ++q) e[q] -= s_by[q0 + q];
#pragma unroll
                for (int q = 0; q < QH; ++q) {
                    const f2 c = *(const f2 *)&s_corr[q0 + 2 * q];
                    l2[q] = mul2(l2[q], c);
                    o2[q] = mul2(o2[q], c);
                }
            }
            // weights, as planes: column n of key k at group n / 16, then k, then n % 16
            uint8_t *dst = spp + wt * 16;
            const f2 rv2 = mk2(rvs, rvs), fv2 = mk2(fvs, fvs);
            f2 x[QH];
#pragma unroll
            for (int q = 0; q < QH; ++q) {
                x[q] = mk2(a8_ex2(e[2 * q]), a8_ex2(e[2 * q + 1]));
                l2[q] = fma2(x[q], rv2, l2[q]);
                x[q] = mul2(x[q], fv2);
            }
#pragma unroll
            for (int p = 0; p < PP; ++p) {
                uint32_t w[QH / 2];
#pragma unroll
                for (int q = 0; q < QH; q += 2) w[q / 2] = a8_quad(x[q], x[q + 1], p + 1 < PP);
                const int n = p * QT + q0;
                if constexpr (QW == 8) *(uint2 *)(dst + (n >> 4) * A8_PG + (n & 15)) = make_uint2(w[0], w[1]);
                else *(uint32_t *)(dst + (n >> 4) * A8_PG + (n & 15)) = w[0];
            }
            // an odd number of pages: the reduction's last 16 keys are no one's, and 0 x anything has to be 0
            if ((n & 1) && tid < KB / 16) *(uint4 *)(sv + t % NS * TB + n * KB + tid * 16) = make_uint4(0, 0, 0, 0);
            fence_async_smem();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&pready);
        }
        if (nt > 0) {
            wait(&ofull, nt - 1);
            tc_fence_after();
            f2 x[QH];
            a8_planes<QT, QW, PP>(tm_o + lanes + q0, x);
#pragma unroll
            for (int q = 0; q < QH; ++q) o2[q] = fma2(x[q], down, o2[q]);
        }
        float l[QW];
#pragma unroll
        for (int q = 0; q < QH; ++q) {
            un2(o2[q], o[2 * q], o[2 * q + 1]);
            un2(l2[q], l[2 * q], l[2 * q + 1]);
        }
        if (s_abort && tid == 0)   // let what is on its way land before the slots are written
            for (int i = 0; i < NS; ++i)
                for (int ph = 0; ph < 2; ++ph) {
                    mbar_wait(&kfull[i], ph, 20000000LL);
                    mbar_wait(&vfull[i], ph, 20000000LL);
                }
        tc_fence_before();
        // the block's partial: every product has ended, the K slots take the outputs
#pragma unroll
        for (int q = 0; q < QW; ++q)
            if (wt < HD && cs > 1) so[(q0 + q) * HD + wt] = o[q];
        // the warp's sums: lanes hand half of their queries to one another until each has one
#pragma unroll
        for (int h = QW / 2, d = 16; h >= 1; h /= 2, d /= 2)
#pragma unroll
            for (int q = 0; q < h; ++q) {
                const bool up = lane & d;
                const float x = __shfl_xor_sync(0xffffffffu, up ? l[q] : l[q + h], d);
                l[q] = (up ? l[q + h] : l[q]) + x;
            }
#pragma unroll
        for (int d = 16 / QW; d >= 1; d /= 2) l[0] += __shfl_xor_sync(0xffffffffu, l[0], d);
        if (lane % (32 / QW) == 0) s_lw[ww][q0 + lane / (32 / QW)] = l[0];
        named_sync(bar, 128);
        if (wt < QW) s_l[q0 + wt] = s_lw[0][q0 + wt] + s_lw[1][q0 + wt] + s_lw[2][q0 + wt] + s_lw[3][q0 + wt];
        if (tid == 0 && s_abort) s_bad = 1;
#pragma unroll
        for (int q = 0; q < QW; ++q) keep[q] = o[q];
    }
    if (bad_id) {
        s_bad = 1;
        set_status(a.status, OSPREY_ERR_CAPACITY);
    }
    auto store = [&](int q, float y) {   // dim wt of query q
        const int i = i0 + q, j = i >> lg, col = (kvh * G + (i & (G - 1))) * HD + wt;
        const size_t at = ((size_t)b * a.max_rows + j) * a.Hq * HD + col;
        if (a.planes.q) attn_store(a.planes, b * a.max_rows + j, col, y);
        else if (a.q_f32) ((float *)a.out)[at] = y;
        else ((uint16_t *)a.out)[at] = (uint16_t)kv8_bf2(y, 0.f);
    };
    __syncwarp();
    if (cs > 1) cluster.sync();
    else __syncthreads();
    if (warp == W_MMA) {
        tc_fence_after();
        a8_dealloc(tmem, C::SCOLS);
        a8_dealloc(tm_o, C::OCOLS);
    } else if (warp < W_MMA) {
        // lane r holds what rank r left of a query; a thread is a dim of the output
        if (cs == 1 && wt < HD && warp < 4 * nact) {
#pragma unroll
            for (int q = 0; q < QW; ++q)
                if (warp / 4 * QW + q < nq) store(warp / 4 * QW + q, s_bad ? 0.f : keep[q] / s_l[warp / 4 * QW + q]);
        }
        for (int q = rank + warp / 4 * cs; q < nq && cs > 1; q += cs * C::NWG) {
            const bool on = lane < cs;
            const float mr = on ? *cluster.map_shared_rank(&s_m[q], on ? lane : 0) : -INFINITY;
            const float lr = on ? *cluster.map_shared_rank(&s_l[q], on ? lane : 0) : 0.f;
            const int br = on ? *cluster.map_shared_rank(&s_bad, on ? lane : 0) : 0;
            float v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = r < cs && wt < HD ? *cluster.map_shared_rank(&so[q * HD + wt], r) : 0.f;
            const float M = a8_warp_max(mr), f = mr == -INFINITY ? 0.f : a8_ex2(mr - M);
            const float den = warp_sum(f * lr);   // a rank whose scores were all NaN: 0 x NaN
            const bool bad = __any_sync(0xffffffffu, br);
            float num = 0.f;
#pragma unroll
            for (int r = 0; r < 8; ++r) num = fmaf(__shfl_sync(0xffffffffu, f, r), v[r], num);
            if (wt < HD) store(q, bad ? 0.f : num / den);
        }
    }
    if (cs > 1) cluster.sync();   // a block's shared memory stays until its cluster has read it
}

template <typename C>
static cudaError_t launch_attn8_t(const Attn8Args &a, int sms, cudaStream_t s) {
    static std::atomic<int> done[kMaxDevices];
    cudaError_t e = once_per_device(done, [] {
        return cudaFuncSetAttribute(attn8_kernel<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    });
    if (e != cudaSuccess) return e;
    const int tiles = (a.max_rows * (a.Hq / a.Hkv) + C::QT - 1) / C::QT;
    const long long units = (long long)a.B * a.Hkv * tiles;
    const int cs = attn8_split(units, (long long)sms * C::BPS, (a.max_pages + 7) / 8);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * cs));
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cs;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, attn8_kernel<C>, a, tiles);
    count_launch();
    return e;
}

// A block takes as many queries as a call can have of one sequence and KV head (rows x
// heads of a group), up to 8 with two blocks an SM.  More go 16 at a time, two blocks an
// SM, up to 32 of them, else 32 at a time: a block of 32 has the SM to itself.  Numbers of
// rows mostly differ from sequence to sequence, and blocks of 16 leave fewer warps idle
// where they do.  us a call, 16 / 32 at a time, 1024..4096 keys: 1..8 rows of 96 sequences,
// groups of four 171 / 193; 1..16 rows of 64, groups of two 121 / 133; 4, 8 and 16 rows of
// each of 32 sequences, groups of four 59 / 75, 88 / 89 and 141 / 135; 50..64 rows of 8
// sequences of 2000..8192 keys 226 / 206; four prompts of 2048 rows 967 / 918.
template <int HD>
static cudaError_t launch_attn8_h(const Attn8Args &a, int sms, cudaStream_t s) {
    const int nq = a.max_rows * (a.Hq / a.Hkv);
    if (a.q_f32) return nq <= 4 ? launch_attn8_t<A8_4F<HD>>(a, sms, s) : launch_attn8_t<A8_8F<HD>>(a, sms, s);
    if (nq <= 4) return launch_attn8_t<A8_4<HD>>(a, sms, s);
    if (nq <= 8) return launch_attn8_t<A8_8<HD>>(a, sms, s);
    // a rotated bf16 query has more bits than its type: four planes keep 16, as for fewer queries
    if (nq <= 32) return a.rotate ? launch_attn8_t<A8_16R<HD>>(a, sms, s) : launch_attn8_t<A8_16<HD>>(a, sms, s);
    return a.rotate ? launch_attn8_t<A8_32R<HD>>(a, sms, s) : launch_attn8_t<A8_32<HD>>(a, sms, s);
}

cudaError_t launch_attn8(const Attn8Args &a, int sms, cudaStream_t s) {
    return a.hd == 128 ? launch_attn8_h<128>(a, sms, s) : launch_attn8_h<64>(a, sms, s);
}

}  // namespace osp
