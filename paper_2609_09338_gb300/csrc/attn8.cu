// Causal attention of a sequence's newest rows over the 8-bit paged cache.
//
//   out_i = sum_j w_ij V_j / sum_j w_ij,  w_ij = exp(q_i . K_j / sqrt(hd)),  j <= position of i
//
// A cluster of blocks takes up to A8_Q (row, head) queries of one KV head; each block a
// range of the finished pages, the last one the tail's bf16 rows too.  The blocks'
// (max, sum, output) are merged through distributed shared memory, so a call is one
// launch without a workspace.
#include <cooperative_groups.h>

#include <algorithm>

#include "attn8.cuh"
#include "internal.h"
#include "tma.cuh"

namespace osp {

namespace cg = cooperative_groups;

constexpr int A8_T = 128;     // threads
constexpr int A8_Q = 8;       // queries of a block
constexpr int A8_CH = 32;     // keys of a step

template <int HD>
__global__ void __launch_bounds__(A8_T) attn8_kernel(const Attn8Args a, int tiles) {
    __shared__ __align__(16) float sq[A8_Q][HD];
    __shared__ float sp[A8_Q][A8_CH], s_m[A8_Q], s_l[A8_Q], s_corr[A8_Q];
    __shared__ float so[A8_Q][HD];
    __shared__ int s_bad;
    cg::cluster_group cluster = cg::this_cluster();
    const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int unit = blockIdx.x / cs, kvh = unit % a.Hkv, tile = unit / a.Hkv % tiles, b = unit / a.Hkv / tiles;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = a.Hq / a.Hkv;
    pdl_trigger();
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
    const int i0 = tile * A8_Q, nq = min(A8_Q, nr * G - i0);
    if (nq <= 0) {   // the whole cluster
        pdl_wait();
        return;
    }
    if (tid == 0) s_bad = !ok;
    pdl_wait();
    for (int i = tid; i < A8_Q * (HD / 2); i += A8_T) {
        const int q = i / (HD / 2), d = i % (HD / 2);
        float x = 0.f, y = 0.f;
        if (q < nq) {
            const int j = (i0 + q) / G, g = (i0 + q) % G;
            const int64_t at = ((int64_t)b * a.max_rows + j) * a.q_stride + (kvh * G + g) * HD + d;
            if (a.q_f32) {
                x = ((const float *)a.q)[at];
                y = ((const float *)a.q)[at + HD / 2];
            } else {
                x = bf_to_f(((const uint16_t *)a.q)[at]);
                y = bf_to_f(((const uint16_t *)a.q)[at + HD / 2]);
            }
            if (a.rotate) {
                float c, s;
                rope_cs_fix(a.freq[d], base + j, c, s);
                const float t = x * c - y * s;
                y = y * c + x * s;
                x = t;
            }
        }
        const float f = rsqrtf((float)HD) * 1.4426950408889634f;   // weights are powers of two
        sq[q][d] = x * f;
        sq[q][d + HD / 2] = y * f;
    }
    if (tid < A8_Q) {
        s_m[tid] = -INFINITY;
        s_l[tid] = 0.f;
    }
    __syncthreads();
    const int32_t *tab = a.page_table + (size_t)b * a.max_pages;
    float o[A8_Q];
#pragma unroll
    for (int q = 0; q < A8_Q; ++q) o[q] = 0.f;
    auto chunk = [&](int key0, int key1, bool tail) {
        // a key is four lanes': every fourth group of 4 dims
        const int key = key0 + tid / 4, quarter = tid % 4;
        float s[A8_Q];
#pragma unroll
        for (int q = 0; q < A8_Q; ++q) s[q] = 0.f;
        size_t blk = 0;
        float scale = 1.f;
        bool good = true;
        if (key < key1) {
            if (tail) {
                blk = ((size_t)b * a.tail_pages + key / 16 % a.tail_pages) * a.Hkv + kvh;
            } else {
                const int page = tab[key / 16];
                good = page >= 0 && page < a.n_pages;
                if (!good) s_bad = 1;
                blk = (size_t)(good ? page : 0) * a.Hkv + kvh;
                scale = good ? a.k_scale[blk] : 0.f;
            }
            for (int d = quarter * 4; good && d < HD; d += 16) {
                float f[4];
                if (tail) {
                    const uint2 w = *(const uint2 *)(a.k_tail + blk * 16 * HD + (key % 16) * HD + d);
                    f[0] = bf_lo(w.x), f[1] = bf_hi(w.x), f[2] = bf_lo(w.y), f[3] = bf_hi(w.y);
                } else {
                    const uint32_t w = *(const uint32_t *)(a.k8 + blk * 16 * HD + ((key % 16 >> 3) * (HD / 16) + (d >> 4)) * 128 +
                                                           (key & 7) * 16 + (d & 15));
                    const float2 lo = e4m3x2_f(w & 0xffff), hi = e4m3x2_f(w >> 16);
                    f[0] = lo.x, f[1] = lo.y, f[2] = hi.x, f[3] = hi.y;
                }
#pragma unroll
                for (int q = 0; q < A8_Q; ++q) {
                    const float4 w = *(const float4 *)&sq[q][d];
                    s[q] = fmaf(w.x, f[0], fmaf(w.y, f[1], fmaf(w.z, f[2], fmaf(w.w, f[3], s[q]))));
                }
            }
        }
#pragma unroll
        for (int q = 0; q < A8_Q; ++q) {
            s[q] += __shfl_xor_sync(0xffffffffu, s[q], 1);
            s[q] += __shfl_xor_sync(0xffffffffu, s[q], 2);
            if (quarter == 0) sp[q][tid / 4] = s[q] * scale;
        }
        __syncthreads();
        for (int q = warp; q < A8_Q; q += A8_T / 32) {
            const int pos = base + (i0 + q) / G;
            const bool see = q < nq && key0 + lane < key1 && key0 + lane <= pos;
            const float x = see ? sp[q][lane] : -INFINITY;
            const float m = fmaxf(s_m[q], warp_max(x)), ref = m == -INFINITY ? 0.f : m;
            const float p = see ? exp2f(x - ref) : 0.f, corr = s_m[q] == -INFINITY ? 0.f : exp2f(s_m[q] - ref);
            const float l = warp_sum(p);
            __syncwarp();
            sp[q][lane] = see ? p : -1.f;   // a masked key is not multiplied: its value may be anything
            if (lane == 0) {
                s_corr[q] = corr;
                s_l[q] = s_l[q] * corr + l;
                s_m[q] = m;
            }
        }
        __syncthreads();
        if (tid < HD) {
#pragma unroll
            for (int q = 0; q < A8_Q; ++q) o[q] *= s_corr[q];
            for (int k = 0; k < min(A8_CH, key1 - key0); ++k) {
                const int kk = key0 + k;
                float v;
                if (tail) {
                    const size_t vb = ((size_t)b * a.tail_pages + kk / 16 % a.tail_pages) * a.Hkv + kvh;
                    v = bf_to_f(a.v_tail[vb * 16 * HD + (kk % 16) * HD + tid]);
                } else {
                    const int page = tab[kk / 16];
                    const bool g = page >= 0 && page < a.n_pages;
                    const size_t vb = (size_t)(g ? page : 0) * a.Hkv + kvh;
                    v = e4m3x2_f(a.v8[vb * 16 * HD + tid * 16 + kk % 16]).x * a.v_scale[vb];
                }
#pragma unroll
                for (int q = 0; q < A8_Q; ++q) {
                    const float p = sp[q][k];
                    if (!(p < 0.f)) o[q] = fmaf(p, v, o[q]);
                }
            }
        }
        __syncthreads();
    };
    // this block's finished pages; keys past the last query's position are seen by none
    const int last = base + (i0 + nq - 1) / G;
    const int np = min(c8, last / 16 + 1), per = (np + cs - 1) / cs;
    const int k0 = min(np, rank * per) * 16, k1 = min(np, (rank + 1) * per) * 16;
    if (ok) {
        for (int k = k0; k < k1; k += A8_CH) chunk(k, min(k1, k + A8_CH), false);
        if (rank == cs - 1)
            for (int k = c8 * 16; k <= last; k += A8_CH) chunk(k, min(last + 1, k + A8_CH), true);
    }
    if (tid < HD)
#pragma unroll
        for (int q = 0; q < A8_Q; ++q) so[q][tid] = o[q];
    if (s_bad && tid == 0 && ok) set_status(a.status, OSPREY_ERR_CAPACITY);
    cluster.sync();
    for (int q = rank; q < nq; q += cs) {
        float M = -INFINITY;
        bool bad = false;
        for (int r = 0; r < cs; ++r) {
            M = fmaxf(M, *cluster.map_shared_rank(&s_m[q], r));
            bad |= *cluster.map_shared_rank(&s_bad, r) != 0;
        }
        float num = 0.f, den = 0.f;
        for (int r = 0; r < cs; ++r) {
            const float m = *cluster.map_shared_rank(&s_m[q], r), f = m == -INFINITY ? 0.f : exp2f(m - M);
            if (m == -INFINITY && !isnan(*cluster.map_shared_rank(&s_l[q], r))) continue;
            den = fmaf(f, *cluster.map_shared_rank(&s_l[q], r), den);
            if (tid < HD) num = fmaf(f, *cluster.map_shared_rank(&so[q][tid], r), num);
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
    cluster.sync();
}

cudaError_t launch_attn8(const Attn8Args &a, int sms, cudaStream_t s) {
    const int tiles = (a.max_rows * (a.Hq / a.Hkv) + A8_Q - 1) / A8_Q;
    const long long units = (long long)a.B * a.Hkv * tiles;
    int cs = 8;
    while (cs > 1 && units * cs > 16LL * sms) cs >>= 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * cs));
    cfg.blockDim = dim3(A8_T);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cs;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = a.seq_len == nullptr;   // behind a draft call's own kernels
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = a.hd == 128 ? cudaLaunchKernelEx(&cfg, attn8_kernel<128>, a, tiles)
                                      : cudaLaunchKernelEx(&cfg, attn8_kernel<64>, a, tiles);
    count_launch();
    return e;
}

}  // namespace osp
