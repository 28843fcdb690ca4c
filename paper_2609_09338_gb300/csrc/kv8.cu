// Appending K/V rows with the position rotation on the way, to the bf16 paged cache
// and to the 8-bit one (kv8.cuh).
#include "kv8.cuh"

#include <algorithm>

#include "internal.h"
#include "tma.cuh"

namespace osp {

constexpr int KR_THREADS = 256;
constexpr int KR_WARPS = KR_THREADS / 32;
constexpr int KR_BLOCKS_PER_SM = 3;

// Exclusive prefix of one int64 per thread over the block; *total: the sum.
__device__ __forceinline__ int64_t kr_scan(int64_t v, int64_t *sh, int64_t *total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int64_t inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t n = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += n;
    }
    if (lane == 31) sh[w] = inc;
    __syncthreads();
    int64_t before = 0, tot = 0;
#pragma unroll
    for (int k = 0; k < KR_WARPS; ++k) {
        if (k < w) before += sh[k];
        tot += sh[k];
    }
    __syncthreads();
    *total = tot;
    return before + inc - v;
}

// Pages that n rows after L0 touch.
__device__ __forceinline__ int kr_pages(int L0, int n) { return n > 0 ? (L0 + n - 1) / 16 - L0 / 16 + 1 : 0; }

// One warp's block of one page and head while it is in registers, as bf16 pairs.
// K: the lane's items are (row, 8 dims, the 8 dims hd / 2 further), the halves that the
// rotation mixes.  V: the lane holds HD / 32 dims of all 16 rows, so that it can write
// a dim's 16 slots at once.
template <int HD>
struct KvBlock {
    static constexpr int C = HD / 16;       // K: 8-dim chunks of half a row
    static constexpr int RPI = 32 / C;      // K: rows an iteration
    static constexpr int NK = 16 / RPI;     // K: iterations
    static constexpr int NV = HD / 64;      // V: 32-bit words of a lane's dims
    uint4 lo[NK], hi[NK];
    uint32_t v[16][NV];
};

// codes of the block and its scale, from bf16 values
template <int HD>
__device__ __forceinline__ void kv8_quantise(const KvBlock<HD> &x, uint8_t *k8, uint8_t *v8, float *ks, float *vs) {
    using B = KvBlock<HD>;
    const int lane = threadIdx.x & 31;
    auto mag2 = [](uint32_t w) { return max(w & 0x7fffu, (w >> 16) & 0x7fffu); };
    uint32_t km = 0, vm = 0;
#pragma unroll
    for (int i = 0; i < B::NK; ++i)
        km = max(km, max(max(max(mag2(x.lo[i].x), mag2(x.lo[i].y)), max(mag2(x.lo[i].z), mag2(x.lo[i].w))),
                         max(max(mag2(x.hi[i].x), mag2(x.hi[i].y)), max(mag2(x.hi[i].z), mag2(x.hi[i].w)))));
#pragma unroll
    for (int t = 0; t < 16; ++t)
#pragma unroll
        for (int j = 0; j < B::NV; ++j) vm = max(vm, mag2(x.v[t][j]));
    km = __reduce_max_sync(0xffffffffu, km);
    vm = __reduce_max_sync(0xffffffffu, vm);
    const bool kbad = km >= 0x7f80u, vbad = vm >= 0x7f80u;   // an infinity or a NaN
    const int ke = kv8_exp(km), ve = kv8_exp(vm);
    if (lane == 0) {
        *ks = kbad ? __uint_as_float(0x7fffffffu) : kv8_pow2(ke);
        *vs = vbad ? __uint_as_float(0x7fffffffu) : kv8_pow2(ve);
    }
    const float ki = kv8_pow2(kbad ? 0 : -ke), vi = kv8_pow2(vbad ? 0 : -ve);
    auto code8 = [&](const uint4 &w) {
        uint2 r;
        r.x = e4m3x2(bf_lo(w.x) * ki, bf_hi(w.x) * ki) | e4m3x2(bf_lo(w.y) * ki, bf_hi(w.y) * ki) << 16;
        r.y = e4m3x2(bf_lo(w.z) * ki, bf_hi(w.z) * ki) | e4m3x2(bf_lo(w.w) * ki, bf_hi(w.w) * ki) << 16;
        return kbad ? make_uint2(0, 0) : r;
    };
    const int c = lane % B::C;
#pragma unroll
    for (int i = 0; i < B::NK; ++i) {
        const int r = lane / B::C + i * B::RPI;
        auto at = [&](int d) { return ((r >> 3) * (HD / 16) + (d >> 4)) * 128 + (r & 7) * 16 + (d & 15); };
        *(uint2 *)(k8 + at(c * 8)) = code8(x.lo[i]);
        *(uint2 *)(k8 + at(HD / 2 + c * 8)) = code8(x.hi[i]);
    }
#pragma unroll
    for (int j = 0; j < B::NV; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t w[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                auto val = [&](int t) { return (h ? bf_hi(x.v[t][j]) : bf_lo(x.v[t][j])) * vi; };
                w[g] = e4m3x2(val(4 * g), val(4 * g + 1)) | e4m3x2(val(4 * g + 2), val(4 * g + 3)) << 16;
            }
            const int d = lane * (HD / 32) + 2 * j + h;
            *(uint4 *)(v8 + d * 16) = vbad ? make_uint4(0, 0, 0, 0) : make_uint4(w[0], w[1], w[2], w[3]);
        }
}

// rows r0 .. r1 - 1 of the block from the page of bf16 rows (16 x HD) at kp and vp
template <int HD>
__device__ __forceinline__ void kv8_from_tail(KvBlock<HD> &x, const uint16_t *kp, const uint16_t *vp, int r0, int r1) {
    using B = KvBlock<HD>;
    const int lane = threadIdx.x & 31, c = lane % B::C;
#pragma unroll
    for (int i = 0; i < B::NK; ++i) {
        const int r = lane / B::C + i * B::RPI;
        if (r < r0 || r >= r1) continue;
        x.lo[i] = *(const uint4 *)(kp + r * HD + c * 8);
        x.hi[i] = *(const uint4 *)(kp + r * HD + HD / 2 + c * 8);
    }
#pragma unroll
    for (int t = 0; t < 16; ++t) {
        if (t < r0 || t >= r1) continue;
        const uint16_t *p = vp + t * HD + lane * (HD / 32);
        if constexpr (HD == 128) {
            const uint2 w = *(const uint2 *)p;
            x.v[t][0] = w.x;
            x.v[t][1] = w.y;
        } else {
            x.v[t][0] = *(const uint32_t *)p;
        }
    }
}

// Bound by memory for prompts, by latency for a decode step.  A unit is one page of
// one sequence, for all layers and heads: the angles of its new positions are made
// once (fixed-point turns, then sincospif) and shared by its warps, which take one
// layer and head at a time through registers: rows are read once, rotated, and
// written in bf16 (to the page, or to the tail) or, where the page is finished,
// as codes.  Units are found by a scan over the batch that each block keeps in
// registers.
template <int HD, bool EIGHT, bool RF32>
__global__ void __launch_bounds__(KR_THREADS, 2) kv_rope_kernel(const KvRopeArgs a) {
    __shared__ int64_t sh[KR_WARPS];
    __shared__ float2 cs[16][HD / 2];
    __shared__ int s_b, s_page;
    __shared__ int64_t s_row;
    using Blk = KvBlock<HD>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int per = (a.B + KR_THREADS - 1) / KR_THREADS;
    const int b0 = min(a.B, (int)threadIdx.x * per), b1 = min(a.B, b0 + per);
    int64_t rows = 0, pages = 0, total, units;
    int neg = 0;
    for (int b = b0; b < b1; ++b) {
        const int n = a.n_rows[b], L0 = a.seq_len[b];
        neg |= n < 0;
        rows += n;
        // a sequence that does not fit has one unit, which reports it
        pages += n > 0 && (L0 < 0 || (int64_t)L0 + n > (int64_t)a.max_pages * 16) ? 1 : kr_pages(L0, n);
    }
    const int64_t row0 = kr_scan(rows, sh, &total), unit0 = kr_scan(pages, sh, &units);
    if (__syncthreads_or(neg) || total != a.total_rows) {
        if (threadIdx.x == 0) set_status(a.status, OSPREY_ERR_INVALID_ARG);
        return;
    }
    pdl_trigger();
    int last_b = -1;
    bool last_ok = false;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        if (u >= unit0 && u < unit0 + pages) {
            int64_t at = unit0, r = row0;
            for (int b = b0; b < b1; ++b) {
                const int n = a.n_rows[b], L0 = a.seq_len[b];
                const int np = n > 0 && (L0 < 0 || (int64_t)L0 + n > (int64_t)a.max_pages * 16) ? 1 : kr_pages(L0, n);
                if (u < at + np) {
                    s_b = b;
                    s_page = (int)(u - at);
                    s_row = r;
                    break;
                }
                at += np;
                r += n;
            }
        }
        __syncthreads();
        const int b = s_b;
        const int64_t row = s_row;
        const int L0 = a.seq_len[b], n = a.n_rows[b], end = L0 + n;
        const int32_t *tab = a.page_table + (size_t)b * a.max_pages;
        if (b != last_b) {   // every page that the rows touch has to be good: the sequence is left as it is otherwise
            bool bad = L0 < 0 || (int64_t)L0 + n > (int64_t)a.max_pages * 16;
            if (!bad)
                for (int p = L0 / 16 + threadIdx.x; p <= (end - 1) / 16; p += KR_THREADS)
                    bad |= tab[p] < 0 || tab[p] >= a.n_pages;
            last_ok = !__syncthreads_or(bad);
            last_b = b;
            if (!last_ok && threadIdx.x == 0) set_status(a.status, OSPREY_ERR_CAPACITY);
        }
        if (!last_ok) {
            __syncthreads();   // s_b is read by all before the next unit writes it
            continue;
        }
        const int p0 = L0 / 16, plast = (end - 1) / 16, TP = EIGHT ? a.tail_pages : 1;
        // One page.  The ring page of p0 holds older rows that its block needs; the new
        // page that falls on the same ring page is written by p0's unit after that.
        auto page_rows = [&](int p, bool codes, bool tail) {
            const int t0 = max(0, L0 - p * 16), t1 = min(16, end - p * 16);
            if (a.rotate)
                for (int i = threadIdx.x; i < (t1 - t0) * (HD / 2); i += KR_THREADS) {
                    const int t = t0 + i / (HD / 2), d = i % (HD / 2);
                    rope_cs_fix(a.freq[d], p * 16 + t, cs[t][d].x, cs[t][d].y);
                }
            __syncthreads();
            const bool full = EIGHT && codes && t1 == 16;
            if (EIGHT && !full && !tail) return;
            const int page = tab[p];
            for (int it = warp; it < a.layers * a.Hkv; it += KR_WARPS) {
                const int l = it / a.Hkv, h = it - l * a.Hkv, layer = a.layer0 + l;
                const size_t blk = ((size_t)layer * a.n_pages + page) * a.Hkv + h;
                uint16_t *kd, *vd;   // this page's bf16 rows
                if (EIGHT) {
                    const size_t t = (((size_t)layer * a.B + b) * TP + p % TP) * a.Hkv + h;
                    kd = a.k_tail + t * 16 * HD;
                    vd = a.v_tail + t * 16 * HD;
                } else {
                    kd = a.k_pages + blk * 16 * HD;
                    vd = a.v_pages + blk * 16 * HD;
                }
                Blk x;
                const int64_t first = (int64_t)l * a.total_rows + row + (int64_t)p * 16 - L0;   // row of slot 0
                const int c = lane % Blk::C;
#pragma unroll
                for (int i = 0; i < Blk::NK; ++i) {
                    const int r = lane / Blk::C + i * Blk::RPI;
                    x.lo[i] = x.hi[i] = make_uint4(0, 0, 0, 0);
                    if (r < t0 || r >= t1) continue;
                    const int64_t at = (first + r) * a.row_stride + h * HD + c * 8;
                    float f[8], g[8];
                    if constexpr (RF32) {
                        const float *src = (const float *)a.k_rows + at;
                        *(uint4 *)f = ld_stream(src);
                        *(uint4 *)(f + 4) = ld_stream(src + 4);
                        *(uint4 *)g = ld_stream(src + HD / 2);
                        *(uint4 *)(g + 4) = ld_stream(src + HD / 2 + 4);
                    } else {
                        const uint16_t *src = (const uint16_t *)a.k_rows + at;
                        unpack8(ld_stream(src), f);
                        unpack8(ld_stream(src + HD / 2), g);
                    }
                    if (a.rotate)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float2 w = cs[r][c * 8 + e];
                            const float y = f[e] * w.x - g[e] * w.y;
                            g[e] = g[e] * w.x + f[e] * w.y;
                            f[e] = y;
                        }
                    x.lo[i] = make_uint4(kv8_bf2(f[0], f[1]), kv8_bf2(f[2], f[3]), kv8_bf2(f[4], f[5]), kv8_bf2(f[6], f[7]));
                    x.hi[i] = make_uint4(kv8_bf2(g[0], g[1]), kv8_bf2(g[2], g[3]), kv8_bf2(g[4], g[5]), kv8_bf2(g[6], g[7]));
                }
#pragma unroll
                for (int t = 0; t < 16; ++t) {
#pragma unroll
                    for (int j = 0; j < Blk::NV; ++j) x.v[t][j] = 0;
                    if (t < t0 || t >= t1) continue;
                    const int64_t at = (first + t) * a.row_stride + h * HD + lane * (HD / 32);
                    if constexpr (RF32) {
                        const float *src = (const float *)a.v_rows + at;
                        if constexpr (HD == 128) {
                            const float4 f = *(const float4 *)src;
                            x.v[t][0] = kv8_bf2(f.x, f.y);
                            x.v[t][1] = kv8_bf2(f.z, f.w);
                        } else {
                            const float2 f = *(const float2 *)src;
                            x.v[t][0] = kv8_bf2(f.x, f.y);
                        }
                    } else {
                        const uint16_t *src = (const uint16_t *)a.v_rows + at;
                        if constexpr (HD == 128) {
                            const uint2 w = *(const uint2 *)src;
                            x.v[t][0] = w.x;
                            x.v[t][1] = w.y;
                        } else {
                            x.v[t][0] = *(const uint32_t *)src;
                        }
                    }
                }
                if (!EIGHT || tail) {
#pragma unroll
                    for (int i = 0; i < Blk::NK; ++i) {
                        const int r = lane / Blk::C + i * Blk::RPI;
                        if (r < t0 || r >= t1) continue;
                        *(uint4 *)(kd + r * HD + c * 8) = x.lo[i];
                        *(uint4 *)(kd + r * HD + HD / 2 + c * 8) = x.hi[i];
                    }
#pragma unroll
                    for (int t = 0; t < 16; ++t) {
                        if (t < t0 || t >= t1) continue;
                        uint16_t *dst = vd + t * HD + lane * (HD / 32);
                        if constexpr (HD == 128) *(uint2 *)dst = make_uint2(x.v[t][0], x.v[t][1]);
                        else *(uint32_t *)dst = x.v[t][0];
                    }
                }
                if (full) {
                    kv8_from_tail<HD>(x, kd, vd, 0, t0);   // older rows (t0 > 0: p is p0, its own ring page)
                    kv8_quantise<HD>(x, a.k8 + blk * 16 * HD, a.v8 + blk * 16 * HD, a.k_scale + blk, a.v_scale + blk);
                }
            }
        };
        const int p = p0 + s_page;
        // the last page on p0's ring page, where that holds older rows
        const int clash = EIGHT && L0 % 16 ? plast - (plast - p0) % TP : p0;
        page_rows(p, true, p > plast - TP && (p == p0 || p != clash));
        if (EIGHT && p == p0 && clash != p0) {
            __syncthreads();   // p0's older rows are read, and so are its angles
            page_rows(clash, false, true);
        }
        __syncthreads();   // cs and s_b are read
    }
}

template <int HD, bool EIGHT, bool RF32>
static cudaError_t launch_kv_rope_t(const KvRopeArgs &a, cudaStream_t s) {
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    // units: n rows touch at most n / 16 + 2 pages, and no more pages than rows
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(a.total_rows, a.total_rows / 16 + 2LL * a.B));
    const int64_t cap = (int64_t)KR_BLOCKS_PER_SM * sms;
    kv_rope_kernel<HD, EIGHT, RF32><<<(unsigned)std::min(most, cap), KR_THREADS, 0, s>>>(a);
    count_launch();
    return cudaGetLastError();
}

cudaError_t launch_kv_rope(const KvRopeArgs &a, bool eight, bool advance, cudaStream_t s) {
    cudaError_t e;
    if (a.hd == 128)
        e = eight ? (a.rows_f32 ? launch_kv_rope_t<128, true, true>(a, s) : launch_kv_rope_t<128, true, false>(a, s))
                  : (a.rows_f32 ? launch_kv_rope_t<128, false, true>(a, s) : launch_kv_rope_t<128, false, false>(a, s));
    else
        e = eight ? (a.rows_f32 ? launch_kv_rope_t<64, true, true>(a, s) : launch_kv_rope_t<64, true, false>(a, s))
                  : (a.rows_f32 ? launch_kv_rope_t<64, false, true>(a, s) : launch_kv_rope_t<64, false, false>(a, s));
    if (e != cudaSuccess || !advance) return e;
    KvAppendArgs v{};
    v.page_table = a.page_table;
    v.seq_len = a.seq_len;
    v.n_rows = a.n_rows;
    v.total_rows = a.total_rows;
    v.B = a.B;
    v.P = 16;
    v.max_pages = a.max_pages;
    v.n_pages = a.n_pages;
    v.status = a.status;
    return launch_kv_advance(v, true, s);
}

// Finished pages of a draft call's committed rows, from the tail: one warp a layer and
// head, one block a page.
template <int HD>
__global__ void __launch_bounds__(KR_THREADS) kv8_pack_kernel(const Kv8PackArgs a) {
    const int b = blockIdx.y, warp = threadIdx.x >> 5;
    if (!a.valid[b]) return;
    const int p = a.pos0[b] / 16 + blockIdx.x;
    if ((p + 1) * 16 > a.pos0[b] + a.nnew[b]) return;
    const int page = a.page_table[(size_t)b * a.max_pages + p];   // in range: the call's first kernel has checked it
    for (int it = warp; it < a.L * a.Hkv; it += KR_WARPS) {
        const int l = it / a.Hkv, h = it - l * a.Hkv;
        const size_t t = ((((size_t)l * a.B + b) * a.tail_pages + p % a.tail_pages) * a.Hkv + h) * 16 * HD;
        const size_t blk = ((size_t)l * a.n_pages + page) * a.Hkv + h;
        KvBlock<HD> x;
        kv8_from_tail<HD>(x, a.k_tail + t, a.v_tail + t, 0, 16);
        kv8_quantise<HD>(x, a.k8 + blk * 16 * HD, a.v8 + blk * 16 * HD, a.k_scale + blk, a.v_scale + blk);
    }
}

cudaError_t launch_kv8_pack(const Kv8PackArgs &a, cudaStream_t s) {
    const dim3 grid((a.max_new + 14) / 16 + 1, a.B);   // pages that max_new rows finish, at most
    if (a.hd == 128) kv8_pack_kernel<128><<<grid, KR_THREADS, 0, s>>>(a);
    else kv8_pack_kernel<64><<<grid, KR_THREADS, 0, s>>>(a);
    count_launch();
    return cudaGetLastError();
}

}  // namespace osp
