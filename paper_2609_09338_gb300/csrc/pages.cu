// Pages of the bf16 paged cache: taken for new rows, bounded by their keys, chosen by
// those bounds.
#include "pages.cuh"

#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "internal.h"
#include "kv8.cuh"
#include "tma.cuh"

namespace osp {

namespace cg = cooperative_groups;

template <typename... P, typename... A>
static cudaError_t pages_launch(void (*k)(P...), dim3 grid, dim3 block, int cluster, cudaStream_t s, size_t smem, const A &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k, args...);
    count_launch();
    return e;
}

// ---------------------------------------------------------------- pages for new rows
// Demands are summed over the batch by every block (4 sequences a thread at most), then
// the cluster's warps write the table's entries and the slots, a sequence each or several
// a sequence.  Nothing is written before the whole call has been checked.  One row of 64
// sequences 8 us, 200 k rows of 96 12 us: dependent loads, 1 us each, barriers and the code's
// fetch.  (Slots 128 rows a warp, a row's sequence by bisection, and two barriers of the
// cluster: 10 and 18 us.)
constexpr int KR_MAXB = 4096, KR_T = 1024, KR_CLUSTER = 16, KR_SMEM = (5 * KR_MAXB + 1) * 4;

template <bool HELD>
__global__ void __launch_bounds__(KR_T) kv_reserve_kernel(const KvReserveArgs a) {
    extern __shared__ int s_dyn[];
    int *s_row = s_dyn, *s_first = s_row + KR_MAXB + 1, *s_len = s_first + KR_MAXB, *s_id = s_len + KR_MAXB, *s_held = s_id + KR_MAXB;
    // first row, first new page (-1: the sequence gets none), length, the id of the page that the rows continue, pages held
    __shared__ long long s_part[32][2];
    __shared__ int s_bad, s_any, s_used;
    cg::cluster_group cluster = cg::this_cluster();
    const int nb = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    pdl_trigger();
    if (tid == 0) s_bad = s_used = s_any = 0;
    if (nb > 1) cluster.barrier_arrive();   // that every block's s_any is 0
    const int taken = *a.n_taken, per = (a.B + KR_T - 1) / KR_T, b0 = tid * per;
    int n[4], need[4], error = 0;
    long long rows = 0, pages = 0;
    bool bad = taken < 0 || taken > a.n_free;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int b = b0 + i;
        n[i] = need[i] = 0;
        if (i >= per || b >= a.B) continue;
        n[i] = a.n_rows[b];
        if (n[i] < 0) {
            bad = true;
            n[i] = 0;
        }
        rows += n[i];
        const int len = a.seq_len[b], from = a.share ? a.share[b] : -1;
        s_len[b] = len;
        int code = len < 0 ? OSPREY_ERR_INVALID_ARG : 0;
        if (from != -1 && from != b && !code) {
            if (from < 0 || from >= a.B || len % 16 || a.seq_len[from] < len) code = OSPREY_ERR_INVALID_ARG;
            else if (a.share[from] != -1 && a.share[from] != from) code = OSPREY_ERR_INVALID_ARG;
        }
        if (!code && (long long)len + n[i] > (long long)a.max_pages * 16) code = OSPREY_ERR_CAPACITY;
        int held = code ? 0 : (len + 15) / 16;
        if (HELD && !code) {
            const int h = a.held[b];
            if (h < (from != -1 && from != b ? 0 : held) || h > a.max_pages) code = OSPREY_ERR_INVALID_ARG;
            held = max(held, h);
        }
        if (HELD) s_held[b] = held;
        if (!code && n[i]) {   // pages held that the rows go to: the one that they continue, and those of rows taken back
            const int end = HELD ? min(held, (len + n[i] + 15) / 16) : held;
            for (int p = len / 16; p < end && !code;) {
                const int id = a.page_table[(size_t)b * a.max_pages + p];
                if (id < 0 || id >= a.n_pages) code = OSPREY_ERR_CAPACITY;
                if (p == len / 16) s_id[b] = id;
                if (!HELD || ++p == end) break;
            }
        }
        if (code) {
            need[i] = -1;
            if (!error) error = code;
            continue;
        }
        need[i] = max(0, (len + n[i] + 15) / 16 - held);
        pages += need[i];
    }
    long long ir = rows, ip = pages;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, ir, o), y = __shfl_up_sync(0xffffffffu, ip, o);
        if (lane >= o) ir += x, ip += y;
    }
    if (lane == 31) s_part[warp][0] = ir, s_part[warp][1] = ip;
    __syncthreads();
    long long all = 0;
    ir -= rows;
    ip -= pages;
    for (int w = 0; w < (a.B + 32 * per - 1) / (32 * per); ++w) {   // warps with sequences
        if (w < warp) ir += s_part[w][0], ip += s_part[w][1];
        all += s_part[w][0];
    }
    if (bad || all != a.total_rows) s_bad = 1;
    const long long have = (long long)a.n_free - taken;
    int used = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int b = b0 + i;
        if (i >= per || b >= a.B) continue;
        s_row[b] = (int)min(ir, (long long)INT32_MAX);
        ir += n[i];
        int first = -1;
        if (need[i] >= 0) {
            if (need[i] == 0 || ip + need[i] <= have) {
                first = (int)(need[i] ? ip : 0);
                if (need[i]) used = (int)ip + need[i];
            } else if (!error) {
                error = OSPREY_ERR_CAPACITY;
            }
            ip += need[i];
        }
        s_first[b] = first;
    }
    if (tid == 0) s_row[a.B] = a.total_rows;
    if (used) atomicMax(&s_used, used);
    __syncthreads();
    // the pages to be handed out are pages
    bool odd = s_bad;
    const int thread = rank * KR_T + tid, threads = nb * KR_T;
    if (!s_bad)
        for (int i = thread; i < s_used; i += threads) {
            const int id = a.free_pages[taken + i];
            odd |= id < 0 || id >= a.n_pages;
        }
    if (nb > 1) {
        cluster.barrier_wait();
        if (odd)
            for (int r = 0; r < nb; ++r) *cluster.map_shared_rank(&s_any, r) = 1;
        cluster.sync();   // (every block has read n_taken too)
    } else {
        if (odd) s_any = 1;
        __syncthreads();
    }
    const bool refuse = s_any;
    const int w0 = rank * (KR_T / 32) + warp, ws = nb * (KR_T / 32);
    if (refuse) {
        if (rank == 0 && tid == 0) set_status(a.status, OSPREY_ERR_INVALID_ARG);
        if (a.slots)
            for (int i = thread; i < a.total_rows; i += threads) a.slots[i] = -1;
        return;
    }
    if (rank == 0 && error) set_status(a.status, error);
    if (rank == 0 && tid == 0) *a.n_taken = taken + s_used;
    // a warp, or several, a sequence: 32 of its pages, a lane each, and their rows
    const int wide = max(1, ws / a.B);
    for (int x = w0; x < a.B * wide; x += ws) {
        const int b = x / wide, part = x - b * wide, at = s_row[b], n = s_row[b + 1] - at, first = s_first[b];
        if (first < 0) {
            if (a.slots)
                for (int i = part * 32 + lane; i < n; i += 32 * wide) a.slots[at + i] = -1;
            continue;
        }
        const int len = s_len[b], held = HELD ? s_held[b] : (len + 15) / 16, end = (len + n + 15) / 16, from = a.share ? a.share[b] : -1;
        int32_t *row = a.page_table + (size_t)b * a.max_pages;
        if (HELD && part == 0 && lane == 0) a.held[b] = max(held, end);
        if (from >= 0 && from != b) {
            const int32_t *src = a.page_table + (size_t)from * a.max_pages;
            for (int p0 = part * 128; p0 < len / 16; p0 += 128 * wide) {
                int id[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) id[i] = p0 + 32 * i + lane < len / 16 ? src[p0 + 32 * i + lane] : 0;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (p0 + 32 * i + lane < len / 16) row[p0 + 32 * i + lane] = id[i];
            }
        }
        for (int p0 = len / 16 + part * 32; p0 < end; p0 += 32 * wide) {
            const int p = p0 + lane, id = p >= end ? 0 : p >= held ? a.free_pages[taken + first + p - held] : !HELD || p == len / 16 ? s_id[b] : row[p];
            if (p >= held && p < end) row[p] = id;
            if (!a.slots) continue;
            const int lim = min(len + n, (p0 + 32) * 16);
            for (int pos0 = max(len, p0 * 16); pos0 < lim; pos0 += 32) {
                const int pos = pos0 + lane, y = __shfl_sync(0xffffffffu, id, min(pos / 16 - p0, 31));
                if (pos < lim) a.slots[at + pos - len] = (int64_t)y * 16 + pos % 16;
            }
        }
    }
}

cudaError_t launch_kv_reserve(const KvReserveArgs &a, cudaStream_t s) {
    // One block where that is enough work for it, else a cluster of 16, the most there is.  One block and 16, us back to back:
    // 8 rows of each of 32 sequences 5.7 and 6.1, of 48 5.8 and 5.7, of 128 7.5 and 6.2; behind a shared prefix, where a
    // table's entries are copied, 16 rows and 4 k entries 5.4 and 5.7, 16 k 6.9 and 6.2, 96 rows and 49 k 10.4 and 6.4.
    const bool few = a.B <= 40 && a.total_rows <= 1024 && (!a.share || (int64_t)a.B * a.max_pages <= 8192);
    const int blocks = few ? 1 : KR_CLUSTER;
    static std::atomic<int> done[kMaxDevices];
    const cudaError_t e = once_per_device(done, [] {
        for (auto *k : {kv_reserve_kernel<false>, kv_reserve_kernel<true>}) {
            cudaError_t x = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, KR_SMEM);
            if (x == cudaSuccess) x = cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
            if (x != cudaSuccess) return x;
        }
        return cudaSuccess;
    });
    if (e != cudaSuccess) return e;
    return pages_launch(a.held ? kv_reserve_kernel<true> : kv_reserve_kernel<false>, dim3(blocks), dim3(KR_T), blocks, s, KR_SMEM, a);
}

// ---------------------------------------------------------------- bounds of a page's keys
// A warp takes a page, two heads at a time: 32 rows, 16 bytes a lane, on their way together;
// largest and smallest two channels an instruction, where NaN and infinities stay, then across
// the lanes that hold a channel.  33 k rows of two layers of 4 heads, 75 MB: 16 us from memory
// (0.70 of the copy's rate: loads behind two dependent ones), 12 where L2 has them; a channel
// an instruction, each tested for being finite, 18 there.
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t y;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
}
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
    uint32_t y;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
}
template <int HD>
__global__ void __launch_bounds__(128) kv_bound_kernel(const KvBoundArgs a, int per_seq) {
    constexpr int RL = HD / 8, RW = 32 / RL, NL = 16 / RW;   // lanes of a row, rows of a read, reads of a page
    const int lane = threadIdx.x & 31, pairs = (a.Hkv + 1) / 2;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int h0 = (int)(item % pairs) * 2, slot = (int)(item / pairs % per_seq);
    const int b = (int)(item / pairs / per_seq % a.B), layer = (int)(item / pairs / per_seq / a.B);
    pdl_wait();
    pdl_trigger();
    if (layer >= a.layers) return;
    const SeqRows r = seq_rows(a.n_rows[b], a.seq_len[b], a.advanced, a.max_rows, a.max_pages);
    if (r.code) {
        if (lane == 0 && slot == 0) set_status(a.status, r.code);
        return;
    }
    const int p = r.base / 16 + slot, end = r.base + r.n;
    if (!r.n || p * 16 >= end) return;
    const int id = a.page_table[(size_t)b * a.max_pages + p];
    if (id < 0 || id >= a.n_pages) {
        if (lane == 0) set_status(a.status, OSPREY_ERR_CAPACITY);
        return;
    }
    const int live = min(16, end - p * 16);
    const int rl = lane % RL, rr = lane / RL;
    uint4 x[2][NL];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const size_t blk = ((size_t)layer * a.n_pages + id) * a.Hkv + min(h0 + k, a.Hkv - 1);
        const uint16_t *src = a.k_pages + blk * 16 * HD + rl * 8;
#pragma unroll
        // rows past the page's are read as its last one: one more of the same changes nothing
        for (int i = 0; i < NL; ++i) x[k][i] = *(const uint4 *)(src + min(i * RW + rr, live - 1) * HD);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (h0 + k >= a.Hkv) break;
        const size_t blk = ((size_t)layer * a.n_pages + id) * a.Hkv + h0 + k;
        uint32_t hi[4] = {x[k][0].x, x[k][0].y, x[k][0].z, x[k][0].w}, lo[4] = {hi[0], hi[1], hi[2], hi[3]}, m2 = 0;
#pragma unroll
        for (int i = 1; i < NL; ++i) {
            const uint32_t y[4] = {x[k][i].x, x[k][i].y, x[k][i].z, x[k][i].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                hi[q] = max2(hi[q], y[q]);
                lo[q] = min2(lo[q], y[q]);
            }
        }
#pragma unroll
        for (int o = RL; o < 32; o <<= 1)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                hi[q] = max2(hi[q], __shfl_xor_sync(0xffffffffu, hi[q], o));
                lo[q] = min2(lo[q], __shfl_xor_sync(0xffffffffu, lo[q], o));
            }
#pragma unroll
        for (int q = 0; q < 4; ++q) m2 = max2(m2, max2(hi[q] & 0x7fff7fffu, lo[q] & 0x7fff7fffu));
        const uint32_t mag = __reduce_max_sync(0xffffffffu, max(m2 << 16, m2 & 0xffff0000u));
        const bool fin = mag < 0x7f800000u;
        const int e = fin ? exp127(mag) : 0;
        // 2^-e in two factors: e goes up to 122, and 2^-e has to be a normal number
        const float u1 = kv8_pow2(-e / 2), u2 = kv8_pow2(-e - -e / 2);
        // the first lanes of a channel round its largest up, the next ones its smallest, whose sign is turned, too
        uint32_t code[2] = {0, 0};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t y = rr == 0 ? hi[q] : lo[q] ^ 0x80008000u;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const float f = s ? bf_hi(y) : bf_lo(y);
                int c = fin ? __float2int_ru(f * u1 * u2) : 0;
                if (fin && f > 0.f) c = max(c, 1);   // a product may be too small for a float
                code[q / 2] |= (uint32_t)(uint8_t)(int8_t)(rr == 0 ? c : -c) << (16 * (q & 1) + 8 * s);
            }
        }
        if (rr < 2) *(uint2 *)(a.codes + (blk * 2 + rr) * HD + rl * 8) = make_uint2(code[0], code[1]);
        if (lane == 0) a.scale[blk] = fin ? kv8_pow2(e) : __uint_as_float(0x7fffffffu);
    }
}

cudaError_t launch_kv_bound(const KvBoundArgs &a, cudaStream_t s) {
    const int per_seq = (a.max_rows + 14) / 16 + 1;   // pages that max_rows rows may touch
    const int64_t items = (int64_t)a.layers * a.B * per_seq * ((a.Hkv + 1) / 2);
    return a.hd == 128 ? pages_launch(kv_bound_kernel<128>, dim3((unsigned)((items + 3) / 4)), dim3(128), 1, s, 0, a, per_seq)
                       : pages_launch(kv_bound_kernel<64>, dim3((unsigned)((items + 3) / 4)), dim3(128), 1, s, 0, a, per_seq);
}

// ---------------------------------------------------------------- pages to read
// Keys of a row's pages, larger for a page that goes first: a float's bits in order, and
// above all of them pages with a key that is not finite, then those that are always read.
constexpr uint32_t SEL_NAN = 0xfffffffdu, SEL_ALWAYS = 0xfffffffeu, SEL_BAD = 0xffffffffu;
constexpr int SEL_R = 16;      // rows of a block
constexpr int SEL_T = 256;
constexpr int SEL_SPLIT = 4;   // blocks an SM that scores are split into (6 or 2 of them: 1 us more)
// Rows an SM up to which 512 threads choose, else 128.  Both kernels, us, 128 and 512 threads, one row of 8 heads a sequence
// unless said: 1 sequence of 250 pages 8.3 and 7.9, 1000 pages 11.3 and 9.3; 38 of 250 pages 15.9 and 15.3, of 1000 32.2 and
// 30.1; 128 of 250 26.7 and 29.5; 1..8 rows of 48 of 256..1024 33.0 and 41.0.  How many pages a row has the host does not
// know: where the rule takes 128 threads and rows have 1000 pages and more, 512 would be faster, 300 of 1000 pages 233 and
// 184, 4 rows of 40 of 1000..2000 67 and 60; and where it takes 512 and rows have 100 pages, 128: 38 of them 10.5 and 11.5.
constexpr int SEL_FEW = 2;

// A score is sum_d Q+_d hi_d + Q-_d lo_d times the page's scale, Q+ and Q- the sums of a
// group's positive and negative 8-bit queries: whole numbers, 1016 at most, which fp16
// holds, and their products add up to less than 2^24, which float32 holds, so every order of
// summing gives the same float.  Pages x rows are a product of mma.sync's shape (a tcgen05
// tile has 128 columns of queries, and its codes would go through shared memory once more
// as fp16): 16 pages by 8 rows, with a page's 16 codes as a lane loads them its part of four
// steps.  `split` blocks share the pages of a sequence's head, 16 a warp at a time, the next
// ones' codes on their way.  1..8 rows of 48 sequences of 4096..16384 positions, 64 MB of codes:
// 19 us, a block 6, of which its reads that wait for one another take 2.  (Sums of dp2a by
// lanes that shared a page and added up by shuffles: 33 us.)
__device__ __forceinline__ void sel_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// four codes as fp16: 1024 + (code + 128), whose bits are 0x6400 + (code + 128), less 1152
__device__ __forceinline__ void sel_half(uint32_t w, uint32_t &lo, uint32_t &hi) {
    const uint32_t u = w ^ 0x80808080u, x = __byte_perm(u, 0x64646464u, 0x4140), y = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 off = __half2half2(__ushort_as_half(0x6480));
    const __half2 l = __hsub2(*(const __half2 *)&x, off), h = __hsub2(*(const __half2 *)&y, off);
    lo = *(const uint32_t *)&l;
    hi = *(const uint32_t *)&h;
}
__device__ __forceinline__ float q_value(float x) { return x; }
__device__ __forceinline__ float q_value(uint16_t x) { return bf_to_f(x); }
template <int HD>
__global__ void __launch_bounds__(SEL_T, 3) kv_score_kernel(const KvSelectArgs a, int split) {
    constexpr int C = HD / 32;   // 64 bytes of a page's codes, the largest first, then the smallest: 16 a lane of four
    __shared__ __align__(16) __half s_q[SEL_R][2 * HD + 8];   // 16 bytes more: a row's reads in other banks than the next one's
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, G = a.Hq / a.Hkv;
    const int unit = blockIdx.x / split, b = unit / a.Hkv, h = unit % a.Hkv, j0 = blockIdx.y * SEL_R;
    const int g = lane / 4, sub = lane % 4, first = blockIdx.x % split * (SEL_T / 32), step = split * (SEL_T / 32);   // 16 pages a pass, a warp a pass
    auto entry = [&](int pass) {
        const int p = pass * 16 + lane % 16;
        return p < a.max_pages ? a.page_table[(size_t)b * a.max_pages + p] : -1;
    };
    constexpr int N = HD / 32;
    float x[8][N];
    auto read = [&](auto *q, int j) {   // a row's queries
        const int64_t at = ((int64_t)b * a.max_rows + j0 + j) * a.q_stride + (int64_t)h * G * HD + lane;
#pragma unroll
        for (int g = 0; g < 8; ++g)
#pragma unroll
            for (int k = 0; k < N; ++k) x[g][k] = g < G ? q_value(q[at + g * HD + 32 * k]) : 0.f;
    };
    auto read_row = [&](int j) {
        if (a.q_f32) read((const float *)a.q, j);
        else read((const uint16_t *)a.q, j);
    };
    pdl_wait();
    pdl_trigger();
    // lengths, ids and queries on their way together: an id and a row count once the lengths say so
    const int n = a.n_rows[b], len = a.seq_len[b];
    int id = entry(first + warp), id1 = entry(first + warp + step);
    if (j0 + warp < a.max_rows) read_row(warp);
    const SeqRows r = seq_rows(n, len, a.advanced, a.max_rows, a.max_pages);
    if (r.code) {
        if (tid == 0 && h == 0 && j0 == 0) set_status(a.status, r.code);
        return;
    }
    const int nr = min(SEL_R, r.n - j0);
    if (nr <= 0) return;
    const int last = (r.base + j0 + nr - 1) / 16;             // the last page that a row of the block sees
    if (first > last / 16) return;
    auto id_of = [&](int id, int pass) {   // -1: bad or past the last
        if (pass * 16 + lane % 16 > last) return -1;
        if (id >= 0 && id < a.n_pages) return id;
        set_status(a.status, OSPREY_ERR_CAPACITY);
        return -1;
    };
    // 2^-24 of the scale: no score leaves float's range.  A bad page's scale is -1
    auto scale_of = [&](int id) { return id < 0 ? -1.f : a.scale[(size_t)id * a.Hkv + h] * 0x1p-24f; };
    id = id_of(id, first + warp);
    id1 = id_of(id1, first + warp + step);
    int4 code[C][2];   // of pages g and g + 8
    const int8_t *src[2];
    auto at_pages = [&](int id) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int y = __shfl_sync(0xffffffffu, id, k * 8 + g);
            src[k] = y < 0 ? nullptr : a.codes + ((size_t)y * a.Hkv + h) * 2 * HD + sub * 16;
        }
    };
    auto load = [&](int c) {
#pragma unroll
        for (int k = 0; k < 2; ++k) code[c][k] = src[k] ? *(const int4 *)(src[k] + c * 64) : make_int4(0, 0, 0, 0);
    };
    // to L2 while the queries are rounded (in registers they would leave room for two blocks an SM, not three)
    if (id >= 0 && lane < 16)
#pragma unroll
        for (int c = 0; c < 2 * HD; c += 128)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(a.codes + ((size_t)id * a.Hkv + h) * 2 * HD + c));
    float scale = scale_of(id);
    for (int j = warp; j < nr; j += SEL_T / 32) {
        if (j != warp) read_row(j);
        if (a.rotate) {
#pragma unroll
            for (int k = 0; k < N / 2; ++k) {
                float c, s;
                rope_cs_fix(a.freq[lane + 32 * k], r.base + j0 + j, c, s);
#pragma unroll
                for (int g = 0; g < 8; ++g) {
                    const float t = x[g][k] * c - x[g][k + N / 2] * s;
                    x[g][k + N / 2] = x[g][k + N / 2] * c + x[g][k] * s;
                    x[g][k] = t;
                }
            }
            if (!a.q_f32)
#pragma unroll
                for (int g = 0; g < 8; ++g)
#pragma unroll
                    for (int k = 0; k < N; ++k) x[g][k] = bf_to_f(f_to_bf(x[g][k]));
        }
        uint32_t mag = 0;   // bits: a number that is not finite has the largest
#pragma unroll
        for (int g = 0; g < 8; ++g)
            if (g < G)
#pragma unroll
                for (int k = 0; k < N; ++k) mag = max(mag, __float_as_uint(x[g][k]) & 0x7fffffffu);
        mag = __reduce_max_sync(0xffffffffu, mag);
        const bool fin = mag < 0x7f800000u;
        const int e = fin ? exp127(mag) : 0;
        const float u1 = kv8_pow2(-e / 2), u2 = kv8_pow2(-e - -e / 2);
        float up[N], down[N];
#pragma unroll
        for (int k = 0; k < N; ++k) up[k] = down[k] = 0.f;
#pragma unroll
        for (int g = 0; g < 8; ++g)
            if (g < G)
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float c = fmaf(x[g][k] * u1, u2, 0x1.8p23f) - 0x1.8p23f;   // to the nearest whole number, ties to even ones
                    up[k] += fmaxf(c, 0.f);
                    down[k] += fminf(c, 0.f);
                }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            s_q[j][lane + 32 * k] = __float2half_rn(fin ? up[k] : 0.f);
            s_q[j][HD + lane + 32 * k] = __float2half_rn(fin ? down[k] : 0.f);
        }
    }
    __syncthreads();
    at_pages(id);
#pragma unroll
    for (int c = 0; c < C; ++c) load(c);
    const int pos0 = r.base + j0 + sub * 2;   // of a lane's first row
    uint32_t *keys = a.keys + (((size_t)b * a.max_rows + j0 + sub * 2) * a.Hkv + h) * a.max_pages;
#pragma unroll 1
    for (int i = first + warp; i <= last / 16; i += step) {
        at_pages(id1);
        const float scale1 = scale_of(id1);
        id1 = id_of(entry(i + 2 * step), i + 2 * step);
        float sum[SEL_R / 8][4] = {};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const uint32_t w0[4] = {(uint32_t)code[c][0].x, (uint32_t)code[c][0].y, (uint32_t)code[c][0].z, (uint32_t)code[c][0].w};
            const uint32_t w1[4] = {(uint32_t)code[c][1].x, (uint32_t)code[c][1].y, (uint32_t)code[c][1].z, (uint32_t)code[c][1].w};
            load(c);
            uint32_t p[4][4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                sel_half(w0[w], p[w][0], p[w][2]);
                sel_half(w1[w], p[w][1], p[w][3]);
            }
#pragma unroll
            for (int n = 0; n < SEL_R / 8; ++n) {   // (rows past the last are whatever lies there: nothing reads their columns)
                if (n * 8 >= nr) break;
                const uint4 *q4 = (const uint4 *)&s_q[n * 8 + g][c * 64 + sub * 16];
                const uint4 qa = q4[0], qb = q4[1];
                sel_mma(sum[n], p[0][0], p[0][1], p[0][2], p[0][3], qa.x, qa.y);
                sel_mma(sum[n], p[1][0], p[1][1], p[1][2], p[1][3], qa.z, qa.w);
                sel_mma(sum[n], p[2][0], p[2][1], p[2][2], p[2][3], qb.x, qb.y);
                sel_mma(sum[n], p[3][0], p[3][1], p[3][2], p[3][3], qb.z, qb.w);
            }
        }
        const uint32_t odd = isnan(scale) ? SEL_NAN : scale < 0.f ? SEL_BAD : 0u;   // of the page, in place of its scores
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int p = i * 16 + k * 8 + g;
            const float sc = __shfl_sync(0xffffffffu, scale, k * 8 + g);
            const uint32_t od = __shfl_sync(0xffffffffu, odd, k * 8 + g);
#pragma unroll
            for (int n = 0; n < SEL_R / 8; ++n) {
                if (n * 8 >= nr) break;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int j = n * 8 + e, mine = (pos0 + j) / 16;
                    if (j + sub * 2 >= nr || p > mine) continue;
                    const uint32_t bits = __float_as_uint(sum[n][k * 2 + e] * sc);
                    uint32_t key = od ? od : bits ^ ((uint32_t)((int32_t)bits >> 31) | 0x80000000u);
                    if ((p < a.n_first || p > mine - a.n_last) && od != SEL_BAD) key = SEL_ALWAYS;
                    keys[(size_t)j * a.Hkv * a.max_pages + p] = key;
                }
            }
        }
        scale = scale1;
    }
}

// The n_select largest keys of a row and head, in page order, the lower page first among
// equals: the smallest key taken is found by passes of 256 bins, until a bin is taken
// whole, then a thread's pages, side by side, go behind those of the threads before it.  K
// threads a row.  (512 bins between the smallest and the largest score, half the passes: 2 us
// more, its bins cost as much to clear and to add up as the keys to count.)
constexpr int SEL_KEYS = 4096;   // keys that are kept in shared memory: of 64 k positions
template <int K>
__global__ void __launch_bounds__(K) kv_select_kernel(const KvSelectArgs a) {
    __shared__ uint32_t s_key[SEL_KEYS];
    __shared__ int s_bin[256], s_w[K / 32], s_e[K / 32], s_found[3], s_bad;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int h = blockIdx.x % a.Hkv, j = blockIdx.x / a.Hkv, b = blockIdx.y;
    pdl_wait();
    pdl_trigger();
    const SeqRows r = seq_rows(a.n_rows[b], a.seq_len[b], a.advanced, a.max_rows, a.max_pages);
    if (j >= r.n) return;
    const size_t row = ((size_t)b * a.max_rows + j) * a.Hkv + h;
    int32_t *out = a.pages + row * a.n_select;
    const int have = r.code ? 0 : (r.base + j) / 16 + 1;
    const uint32_t *keys = a.keys + row * a.max_pages;
    if (tid == 0) s_bad = 0;
    for (int i = tid; i < 256; i += K) s_bin[i] = 0;
    __syncthreads();
    const bool near = have <= SEL_KEYS;
    bool bad = false;
    for (int p = tid; p < have; p += K) {
        const uint32_t k = keys[p];
        if (near) s_key[p] = k;
        bad |= k == SEL_BAD;
        atomicAdd(&s_bin[k >> 24], 1);
    }
    if (bad) s_bad = 1;
    auto key = [&](int p) { return near ? s_key[p] : keys[p]; };
    __syncthreads();
    if (s_bad || have <= a.n_select) {
        for (int i = tid; i < a.n_select; i += K) out[i] = !s_bad && i < have ? i : -1;
        return;
    }
    uint32_t thr = 0, mask = 0;   // keys above thr are taken, of those equal to it in the mask's bits `left`
    int left = a.n_select;
    for (int shift = 24;; shift -= 8) {
        if (warp == 0) {   // a lane has 8 bins, from the top
            int c[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                c[i] = s_bin[255 - lane * 8 - i];
                sum += c[i];
            }
            int before = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before += x;
            }
            before -= sum;
            if (before < left && before + sum >= left)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (before < left && before + c[i] >= left) {
                        s_found[0] = 255 - lane * 8 - i;
                        s_found[1] = left - before;
                        s_found[2] = c[i];
                    }
                    before += c[i];
                }
        }
        __syncthreads();
        thr |= (uint32_t)s_found[0] << shift;
        left = s_found[1];
        mask |= 255u << shift;
        if (shift == 0 || left == s_found[2]) break;
        for (int i = tid; i < 256; i += K) s_bin[i] = 0;
        __syncthreads();
        for (int p = tid; p < have; p += K) {
            const uint32_t k = key(p);
            if ((k & mask) == thr) atomicAdd(&s_bin[k >> (shift - 8) & 255], 1);
        }
        __syncthreads();
    }
    const int per = (have + K - 1) / K | 1, p0 = min(have, tid * per), p1 = min(have, p0 + per);   // odd: no two lanes in a bank
    int above = 0, same = 0;
    for (int p = p0; p < p1; ++p) {
        const uint32_t k = key(p) & mask;
        above += k > thr;
        same += k == thr;
    }
    int ia = above, ie = same;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, ia, o), y = __shfl_up_sync(0xffffffffu, ie, o);
        if (lane >= o) ia += x, ie += y;
    }
    if (lane == 31) s_w[warp] = ia, s_e[warp] = ie;
    __syncthreads();
    ia -= above;
    ie -= same;
    for (int w = 0; w < warp; ++w) ia += s_w[w], ie += s_e[w];
    for (int p = p0; p < p1; ++p) {
        const uint32_t k = key(p) & mask;
        if (k > thr || (k == thr && ie < left)) out[ia + min(ie, left)] = p;
        ia += k > thr;
        ie += k == thr;
    }
}

cudaError_t launch_kv_select(const KvSelectArgs &a, int sms, cudaStream_t s) {
    // blocks that share a sequence's head: SEL_SPLIT an SM, none without 16 pages a warp of the longest context
    const int split = std::max(1, std::min((a.max_pages + SEL_T / 2 - 1) / (SEL_T / 2), (SEL_SPLIT * sms + a.B * a.Hkv - 1) / (a.B * a.Hkv)));
    const dim3 grid((unsigned)split * a.B * a.Hkv, (a.max_rows + SEL_R - 1) / SEL_R);
    cudaError_t e = a.hd == 128 ? pages_launch(kv_score_kernel<128>, grid, dim3(SEL_T), 1, s, 0, a, split)
                                : pages_launch(kv_score_kernel<64>, grid, dim3(SEL_T), 1, s, 0, a, split);
    if (e != cudaSuccess) return e;
    const dim3 rows((unsigned)a.Hkv * a.max_rows, a.B);
    return (int64_t)rows.x * a.B <= SEL_FEW * sms ? pages_launch(kv_select_kernel<512>, rows, dim3(512), 1, s, 0, a)
                                                  : pages_launch(kv_select_kernel<128>, rows, dim3(128), 1, s, 0, a);
}

}  // namespace osp
