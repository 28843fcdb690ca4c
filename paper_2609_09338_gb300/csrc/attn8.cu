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
// float32, so no product of unlike sizes shares an accumulator.  bf16 queries are two
// planes exactly.
//
// Per tile of 128 keys a thread is a key: it reads its scores from TMEM, the block
// finds each query's running maximum, the thread writes its weights' planes, and the
// output of the tile before, a thread now being a dim, is added from TMEM to registers
// in float32.  The V block's scale goes into the weight: w' = 2^(s + log2(vs) - m'),
// the sum adds w' / vs.
#include <cooperative_groups.h>

#include <algorithm>

#include "attn8.cuh"
#include "internal.h"
#include "tcgen05.cuh"
#include "tma.cuh"

namespace osp {

namespace cg = cooperative_groups;

constexpr int A8_C = 128;            // compute threads
constexpr int A8_T = A8_C + 32;      // and the warp that copies and issues
constexpr int A8_CH = 32;            // tail keys of a step
constexpr float A8_LO = -40.f;       // smallest log2 of a V scale that moves the maximum (a8_scales)

template <int HD_, int QT_, int QP_, int PP_, int BPS_>
struct A8 {
    static constexpr int HD = HD_, QT = QT_, QP = QP_, PP = PP_, BPS = BPS_;
    static constexpr int KB = 16 * HD, TB = 8 * KB;     // bytes of a page, of a tile's slot
    static constexpr int NS = HD == 128 ? 2 : 4;        // slots of K and of V
    static constexpr int SC = QP * QT, OC = PP * QT;    // TMEM columns of the scores, of the output
    static constexpr int TM = 512 / BPS;                // columns a block may take
    static constexpr int NSB = 2 * SC + OC <= TM ? 2 : 1;
    static constexpr int COLS = NSB * SC + OC <= 32 ? 32 : NSB * SC + OC <= 64 ? 64 : NSB * SC + OC <= 128 ? 128
                              : NSB * SC + OC <= 256 ? 256 : 512;
    static constexpr int QB = SC * HD;                               // bytes of q's planes
    static constexpr int PB = OC * 128 > QT * HD * 4 ? OC * 128 : QT * HD * 4;   // the weights' planes, or q for the tail
    static constexpr int SMEM = 2 * NS * TB + QB + PB + QT * A8_CH * 4;
    static_assert(COLS <= TM && SC % 16 == 0 && OC % 16 == 0 && QB + PB >= KB, "operands");
    static_assert(QT * HD * 4 <= NS * TB, "the merge's outputs take the K slots");
};

// Shared-memory matrix descriptor of a K-major operand without swizzle: core matrices
// of 8 rows x 16 bytes, lbo bytes apart along the reduction, sbo along the rows.
__device__ __forceinline__ uint64_t a8_desc(uint32_t addr, uint32_t lbo, uint32_t sbo) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(sbo >> 4) << 32 | (uint64_t)1 << 46;
}
// kind::f8f6f4, e4m3 operands, both K-major, float32 accumulator, M 128
__host__ __device__ constexpr uint32_t a8_idesc(int N) { return (1u << 4) | (uint32_t)(N >> 3) << 17 | (128u >> 4) << 24; }
__device__ __forceinline__ void a8_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(d),
                 "l"(a), "l"(b), "r"(idesc), "r"(acc)
                 : "memory");
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

// TMEM columns [c0, c0 + P x QT) of the warp's lanes, plane by plane: x[q] = sum over planes of 16^-p column p QT + q
template <int QT, int P>
__device__ __forceinline__ void a8_planes(uint32_t col, float (&x)[QT]) {
    if constexpr (QT == 8) {   // a load holds two planes
        float v[P / 2][16];
#pragma unroll
        for (int c = 0; c < P / 2; ++c) tc_ld16(col + c * 16, v[c]);
        tc_ld_wait();
#pragma unroll
        for (int c = 0; c < P / 2; ++c) tc_ld_tie(v[c]);
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            float s = 0.f;
#pragma unroll
            for (int p = P - 1; p >= 0; --p) s = fmaf(s, 0.0625f, v[p / 2][(p & 1) * 8 + q]);
            x[q] = s;
        }
    } else {
#pragma unroll
        for (int q = 0; q < QT; ++q) x[q] = 0.f;
#pragma unroll
        for (int p = P - 1; p >= 0; --p) {
            float v[QT / 16][16];
#pragma unroll
            for (int c = 0; c < QT / 16; ++c) tc_ld16(col + p * QT + c * 16, v[c]);
            tc_ld_wait();
#pragma unroll
            for (int c = 0; c < QT / 16; ++c) tc_ld_tie(v[c]);
#pragma unroll
            for (int q = 0; q < QT; ++q) x[q] = fmaf(x[q], 0.0625f, v[q / 16][q % 16]);
        }
    }
}

template <typename C>
__global__ void __launch_bounds__(A8_T, C::BPS) attn8_kernel(const __grid_constant__ Attn8Args a, int tiles) {
    constexpr int HD = C::HD, QT = C::QT, QP = C::QP, PP = C::PP, KB = C::KB, TB = C::TB, NS = C::NS;
    extern __shared__ __align__(1024) uint8_t sm[];
    uint8_t *sk = sm, *sv = sk + NS * TB, *sqp = sv + NS * TB, *spp = sqp + C::QB;
    float *sq = (float *)spp;                       // [QT][HD] while the tail is read
    float *sp = (float *)(spp + C::PB);             // [QT][A8_CH] the tail's weights
    float *so = (float *)sk;                        // [QT][HD] at the end
    __shared__ __align__(8) uint64_t kfull[NS], vfull[NS], sfull[2], pready, ofull;
    __shared__ __align__(16) float s_red[2][4][QT], s_mul[QT];
    __shared__ float s_m[QT], s_l[QT], s_corr[QT], s_lw[4][QT];
    __shared__ int s_pos[QT], s_bad, s_abort;
    __shared__ uint32_t s_tmem;
    cg::cluster_group cluster = cg::this_cluster();
    const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int unit = blockIdx.x / cs, kvh = unit % a.Hkv, tile = unit / a.Hkv % tiles, b = unit / a.Hkv / tiles;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = a.Hq / a.Hkv;
    int nr, base, c8;
    bool ok = true;
    if (a.seq_len) {
        nr = a.n_rows[b];
        const int len = a.seq_len[b];
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
    const int i0 = tile * QT, nq = min(QT, nr * G - i0);
    if (nq <= 0) {   // the whole cluster
        pdl_wait();
        return;
    }
    // this block's finished pages; keys past the last query's position are seen by none
    const int last = base + (i0 + nq - 1) / G;
    const int np_all = ok ? min(c8, last / 16 + 1) : 0, per = (np_all + cs - 1) / cs;
    const int pg0 = min(np_all, rank * per), np = min(np_all, pg0 + per) - pg0, nt = (np + 7) / 8;
    const int32_t *tab = a.page_table + (size_t)b * a.max_pages + pg0;
    auto page_of = [&](int p) {   // page p of the range as a block's number, 0 for a bad id
        const int id = __ldg(tab + p);
        const bool good = id >= 0 && id < a.n_pages;
        if (!good) s_bad = 1;
        return (size_t)(good ? id : 0) * a.Hkv + kvh;
    };
    if (tid == A8_C) {
        for (int i = 0; i < NS; ++i) {
            mbar_init(&kfull[i], 1);
            mbar_init(&vfull[i], 1);
        }
        mbar_init(&sfull[0], 1);
        mbar_init(&sfull[1], 1);
        mbar_init(&ofull, 1);
        mbar_init(&pready, 4);
        s_bad = !ok;
        s_abort = 0;
        mbar_fence_init();
    }
    if (warp == 4) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)),
                     "r"((uint32_t)C::COLS));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    // copies of a tile's K or V pages, a lane a page
    auto load = [&](int t, uint8_t *ring, const uint8_t *src, size_t blk, uint64_t *full) {
        const int n = min(8, np - t * 8), slot = t % NS;
        if (lane == 0) mbar_arrive_expect_tx(&full[slot], (uint32_t)(n * KB));
        __syncwarp();
        if (lane < n) bulk_g2s(ring + slot * TB + lane * KB, src + blk * KB, KB, &full[slot]);
    };
    size_t blk_k = 0, blk_v = 0;   // control warp: the lane's page of the next K tile, of the next V tile
    auto lane_page = [&](int t) { return lane < 8 && t * 8 + lane < np ? page_of(t * 8 + lane) : (size_t)0; };
    if (warp == 4) {
        // finished pages are written by no kernel that this one may overlap
        for (int t = 0; t < min(NS, nt); ++t) {
            const size_t blk = lane_page(t);
            load(t, sk, a.k8, blk, kfull);
            load(t, sv, a.v8, blk, vfull);
        }
        blk_k = lane_page(NS);
    }
    pdl_wait();   // queries and the tail's rows
    const bool tail = ok && rank == cs - 1;
    if (warp < 4) {
        // queries: rotated, scaled to a magnitude of 128 to 256, split into planes; a lane holds pairs (d, d + HD / 2)
        constexpr int NP = HD / 64;
        for (int q = warp; q < QT; q += 4) {
            const int i = min(i0 + q, i0 + nq - 1), j = i / G, g = i - j * G;   // queries past the last one are copies of it
            const int64_t at = ((int64_t)b * a.max_rows + j) * a.q_stride + (kvh * G + g) * HD + lane;
            float x[2 * NP], mag = 0.f;
            bool fin = true;
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                const int d = lane + 32 * k;
                float u, w;
                if (a.q_f32) {
                    u = ((const float *)a.q)[at + 32 * k];
                    w = ((const float *)a.q)[at + 32 * k + HD / 2];
                } else {
                    u = bf_to_f(((const uint16_t *)a.q)[at + 32 * k]);
                    w = bf_to_f(((const uint16_t *)a.q)[at + 32 * k + HD / 2]);
                }
                if (a.rotate) {
                    float c, s;
                    rope_cs_fix(a.freq[d], base + j, c, s);
                    const float t = u * c - w * s;
                    w = w * c + u * s;
                    u = t;
                }
                x[k] = u;
                x[NP + k] = w;
                fin = fin && isfinite(u) && isfinite(w);
                mag = fmaxf(mag, fmaxf(fabsf(u), fabsf(w)));
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
                s_m[q] = -INFINITY;
                s_l[q] = 0.f;
            }
        }
        fence_async_smem();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // not before this block holds its TMEM: a dependent's blocks take theirs and wait for this kernel
    pdl_trigger();
    const uint32_t tmem = s_tmem, tm_o = tmem + C::NSB * C::SC;
    // After a wait that ran out nothing is waited for or issued any more: the loops run to
    // their ends, and the cluster's outputs are 0.
    auto wait = [&](uint64_t *bar, int phase) {
        if (!*(volatile int *)&s_abort && !mbar_wait(bar, (uint32_t)phase & 1)) {
            s_abort = 1;
            set_status(a.status, OSPREY_ERR_TIMEOUT);
        }
        __syncwarp();
    };
    if (warp == 4) {
        auto scores = [&](int t) {   // scores of tile t, 128 keys x (planes x queries)
            wait(&kfull[t % NS], t / NS);
            if (lane == 0 && !s_abort) {
                tc_fence_after();
                const uint32_t A = smem_u32(sk + t % NS * TB), Q = smem_u32(sqp);
#pragma unroll
                for (int k = 0; k < HD / 32; ++k)
                    a8_mma(tmem + (C::NSB == 2 ? (t & 1) * C::SC : 0), a8_desc(A + k * 256, 128, HD * 8),
                           a8_desc(Q + k * 256, 128, HD * 8), a8_idesc(C::SC), k > 0);
                tc_commit(&sfull[C::NSB == 2 ? t & 1 : 0]);
            }
            __syncwarp();
        };
        auto output = [&](int t) {   // head_dim x (planes x queries) over tile t's keys
            wait(&pready, t);   // its weights are written; its scores are read, the output of the tile before too
            wait(&vfull[t % NS], t / NS);
            if (lane == 0 && !s_abort) {
                tc_fence_after();
                const uint32_t A = smem_u32(sv + t % NS * TB), P = smem_u32(spp);
                const int n = min(8, np - t * 8);
                for (int k = 0; k < (n + 1) / 2; ++k)
                    a8_mma(tm_o, a8_desc(A + k * 2 * KB, KB, 128), a8_desc(P + k * 256, 128, 1024), a8_idesc(C::OC), k > 0);
                tc_commit(&ofull);
            }
            if (__shfl_sync(0xffffffffu, *(volatile int *)&s_abort, 0)) return;
            if (t >= 1 && t - 1 + NS < nt) load(t - 1 + NS, sv, a.v8, blk_v, vfull);   // the slot of tile t - 1
            if (t + NS < nt) {
                load(t + NS, sk, a.k8, blk_k, kfull);
                blk_v = blk_k;
                blk_k = lane_page(t + NS + 1);
            }
        };
        for (int t = 0; t <= nt && nt > 0; ++t) {
            if (C::NSB == 2 && t < nt) scores(t);
            if (t > 0) output(t - 1);
            if (C::NSB == 1 && t < nt) scores(t);
            if (__shfl_sync(0xffffffffu, *(volatile int *)&s_abort, 0)) break;
        }
        if (s_abort)   // let what is on its way land before the block ends
            for (int i = 0; i < NS; ++i)
                for (int ph = 0; ph < 2; ++ph) {
                    mbar_wait(&kfull[i], ph, 20000000LL);
                    mbar_wait(&vfull[i], ph, 20000000LL);
                }
    } else {
        float o[QT], l[QT], m[QT];
#pragma unroll
        for (int q = 0; q < QT; ++q) o[q] = 0.f;
        if (tail)   // bf16 rows behind the finished pages, in float32
            for (int key0 = c8 * 16; key0 <= last; key0 += A8_CH) {
                const int key1 = min(last + 1, key0 + A8_CH);
                // a key is four lanes': every fourth group of 4 dims
                const int key = key0 + tid / 4, quarter = tid % 4;
                float s[QT];
#pragma unroll
                for (int q = 0; q < QT; ++q) s[q] = 0.f;
                if (key < key1) {
                    const uint16_t *kr = a.k_tail +
                                         (((size_t)b * a.tail_pages + key / 16 % a.tail_pages) * a.Hkv + kvh) * 16 * HD + (key % 16) * HD;
                    for (int d = quarter * 4; d < HD; d += 16) {
                        const uint2 w = *(const uint2 *)(kr + d);
                        const float f0 = bf_lo(w.x), f1 = bf_hi(w.x), f2 = bf_lo(w.y), f3 = bf_hi(w.y);
#pragma unroll
                        for (int q = 0; q < QT; ++q) {
                            const float4 u = *(const float4 *)&sq[q * HD + d];
                            s[q] = fmaf(u.x, f0, fmaf(u.y, f1, fmaf(u.z, f2, fmaf(u.w, f3, s[q]))));
                        }
                    }
                }
#pragma unroll
                for (int q = 0; q < QT; ++q) {
                    s[q] += __shfl_xor_sync(0xffffffffu, s[q], 1);
                    s[q] += __shfl_xor_sync(0xffffffffu, s[q], 2);
                    if (quarter == 0) sp[q * A8_CH + tid / 4] = s[q];
                }
                named_sync(1, A8_C);
                for (int q = warp; q < QT; q += 4) {
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
                        s_m[q] = mn;
                    }
                }
                named_sync(1, A8_C);
                if (tid < HD) {
#pragma unroll
                    for (int q = 0; q < QT; ++q) o[q] *= s_corr[q];
                    for (int k = 0; k < key1 - key0; ++k) {
                        const int kk = key0 + k;
                        const float v = bf_to_f(a.v_tail[(((size_t)b * a.tail_pages + kk / 16 % a.tail_pages) * a.Hkv + kvh) * 16 * HD +
                                                         (kk % 16) * HD + tid]);
#pragma unroll
                        for (int q = 0; q < QT; ++q) {
                            const float p = sp[q * A8_CH + k];
                            if (!(p < 0.f)) o[q] = fmaf(p, v, o[q]);
                        }
                    }
                }
                named_sync(1, A8_C);
            }
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            m[q] = s_m[q];
            l[q] = tid == 0 ? s_l[q] : 0.f;
        }
        // the thread's key of tile t: its page's scales are loaded a tile ahead
        float ks = 0.f, vs = 1.f, ksn = 0.f, vsn = 1.f;
        auto scales = [&](int t, float &k, float &v) {
            const int p = t * 8 + (tid >> 4);
            if (p < np) {
                const size_t blk = page_of(p);
                k = __ldg(a.k_scale + blk);
                v = __ldg(a.v_scale + blk);
            }
        };
        scales(0, ksn, vsn);
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        const int first_pos = base + i0 / G;
        for (int t = 0; t < nt; ++t) {
            ks = ksn;
            vs = vsn;
            scales(t + 1, ksn, vsn);
            const int n = min(8, np - t * 8), key = (pg0 + t * 8) * 16 + tid;
            // a scale under 2^A8_LO (a block of zeros) would push the weight out of float32's range
            const float lv = __log2f(vs), lvs = lv < A8_LO ? A8_LO : lv;
            // a NaN scale comes through the score, to the queries that see the key alone
            const float rvs = lv < A8_LO ? a8_ex2(-A8_LO) : isnan(vs) ? 1.f : 1.f / vs, fvs = lv < A8_LO ? vs * a8_ex2(-A8_LO) : 1.f;
            float s[QT];
            if (C::NSB == 2) wait(&sfull[t & 1], t >> 1);
            else wait(&sfull[0], t);
            tc_fence_after();
            a8_planes<QT, QP>(tmem + lanes + (C::NSB == 2 ? (t & 1) * C::SC : 0), s);
            const bool in = tid < n * 16;
            const bool whole = (pg0 + t * 8 + n) * 16 - 1 <= first_pos;   // every query sees the tile
#pragma unroll
            for (int q = 0; q < QT; ++q) s[q] = in ? fmaf(s[q] * ks, s_mul[q], lvs) : -INFINITY;
            if (!whole)
#pragma unroll
                for (int q = 0; q < QT; ++q)
                    if (key > s_pos[q]) s[q] = -INFINITY;
            float4 mx[QT / 4];
#pragma unroll
            for (int q = 0; q < QT; ++q) ((float *)mx)[q] = a8_warp_max(s[q]);
            if (lane == 0)
#pragma unroll
                for (int q = 0; q < QT; q += 4) *(float4 *)&s_red[t & 1][warp][q] = mx[q / 4];
            named_sync(1, A8_C);
            float corr[QT];
#pragma unroll
            for (int q = 0; q < QT; q += 4) {
                float4 v[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) v[w] = *(const float4 *)&s_red[t & 1][w][q];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    auto at = [&](const float4 &f) { return e == 0 ? f.x : e == 1 ? f.y : e == 2 ? f.z : f.w; };
                    const float mn = fmaxf(fmaxf(m[q + e], fmaxf(at(v[0]), at(v[1]))), fmaxf(at(v[2]), at(v[3])));
                    corr[q + e] = mn == -INFINITY ? 1.f : a8_ex2(m[q + e] - mn);
                    m[q + e] = mn;
                    l[q + e] *= corr[q + e];
                }
            }
            if (t > 0) {   // the output of the tile before: a thread is a dim
                wait(&ofull, t - 1);
                tc_fence_after();
                float x[QT];
                a8_planes<QT, PP>(tm_o + lanes, x);
#pragma unroll
                for (int q = 0; q < QT; ++q) o[q] = (o[q] + x[q] * 0x1p-8f) * corr[q];
            } else {
#pragma unroll
                for (int q = 0; q < QT; ++q) o[q] *= corr[q];
            }
            // weights, times 256 as planes
            uint8_t *dst = spp + (tid >> 4) * 128 + (tid & 15);
#pragma unroll
            for (int q = 0; q < QT; q += 2) {
                float x[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float p = a8_ex2(s[q + e] - (m[q + e] == -INFINITY ? 0.f : m[q + e]));
                    l[q + e] = fmaf(p, rvs, l[q + e]);
                    x[e] = p * fvs * 256.f;
                }
#pragma unroll
                for (int p = 0; p < PP; ++p) {
                    const int r = p * QT + q;
                    const uint32_t c = e4m3x2(x[0], x[1]);
                    dst[(r >> 3) * 1024 + (r & 7) * 16] = (uint8_t)c;
                    dst[(r >> 3) * 1024 + (r & 7) * 16 + 16] = (uint8_t)(c >> 8);
                    const float2 f = e4m3x2_f(c);
                    x[0] = (x[0] - f.x) * 16.f;
                    x[1] = (x[1] - f.y) * 16.f;
                }
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
            float x[QT];
            a8_planes<QT, PP>(tm_o + lanes, x);
#pragma unroll
            for (int q = 0; q < QT; ++q) o[q] = fmaf(x[q], 0x1p-8f, o[q]);
        }
        tc_fence_before();
        // the block's partial: every MMA has ended, the K slots take the outputs
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const float x = warp_sum(l[q]);
            if (lane == 0) s_lw[warp][q] = x;
            if (tid < HD) so[q * HD + tid] = o[q];
            if (tid == 0) s_m[q] = m[q];
        }
        named_sync(1, A8_C);
        if (tid < QT) s_l[tid] = s_lw[0][tid] + s_lw[1][tid] + s_lw[2][tid] + s_lw[3][tid];
        if (tid == 0) {
            if (s_bad && ok) set_status(a.status, OSPREY_ERR_CAPACITY);
            if (s_abort) s_bad = 1;
        }
    }
    __syncwarp();
    cluster.sync();
    if (warp == 4) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)C::COLS));
    } else {
        for (int q = rank; q < nq; q += cs) {
            float M = -INFINITY;
            bool bad = false;
            for (int r = 0; r < cs; ++r) {
                M = fmaxf(M, *cluster.map_shared_rank(&s_m[q], r));
                bad |= *cluster.map_shared_rank(&s_bad, r) != 0;
            }
            float num = 0.f, den = 0.f;
            for (int r = 0; r < cs; ++r) {
                const float mr = *cluster.map_shared_rank(&s_m[q], r), lr = *cluster.map_shared_rank(&s_l[q], r);
                if (mr == -INFINITY && !isnan(lr)) continue;
                const float f = mr == -INFINITY ? 0.f : a8_ex2(mr - M);
                den = fmaf(f, lr, den);
                if (tid < HD) num = fmaf(f, *cluster.map_shared_rank(&so[q * HD + tid], r), num);
            }
            if (tid < HD) {
                const int j = (i0 + q) / G, col = (kvh * G + (i0 + q) % G) * HD + tid;
                const float y = bad ? 0.f : num / den;
                const size_t at = ((size_t)b * a.max_rows + j) * a.Hq * HD + col;
                if (a.planes.q) attn_store(a.planes, b * a.max_rows + j, col, y);
                else if (a.q_f32) ((float *)a.out)[at] = y;
                else ((uint16_t *)a.out)[at] = (uint16_t)kv8_bf2(y, 0.f);
            }
        }
    }
    cluster.sync();
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
    int cs = 8;
    while (cs > 1 && units * cs > 16LL * sms) cs >>= 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * cs));
    cfg.blockDim = dim3(A8_T);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cs;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = a.seq_len == nullptr;   // behind a draft call's own kernels
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, attn8_kernel<C>, a, tiles);
    count_launch();
    return e;
}

template <int HD>
static cudaError_t launch_attn8_h(const Attn8Args &a, int sms, cudaStream_t s) {
    const int nq = a.max_rows * (a.Hq / a.Hkv);
    if (a.q_f32) return launch_attn8_t<A8<HD, 8, 6, 6, 2>>(a, sms, s);
    if (nq <= 8) return launch_attn8_t<A8<HD, 8, 4, 4, 3>>(a, sms, s);
    if (nq <= 16 || a.rotate) return launch_attn8_t<A8<HD, 16, 3, 3, 2>>(a, sms, s);
    return launch_attn8_t<A8<HD, 32, 2, 3, 2>>(a, sms, s);
}

cudaError_t launch_attn8(const Attn8Args &a, int sms, cudaStream_t s) {
    return a.hd == 128 ? launch_attn8_h<128>(a, sms, s) : launch_attn8_h<64>(a, sms, s);
}

}  // namespace osp
