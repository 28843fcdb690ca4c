// Appending K/V rows with the position rotation on the way, to the bf16 paged cache
// and to the 8-bit one (kv8.cuh).
#include "kv8.cuh"

#include <algorithm>

#include "internal.h"
#include "tma.cuh"

namespace osp {

constexpr int KR_THREADS = 128;
constexpr int KR_WARPS = KR_THREADS / 32;
constexpr int PK_THREADS = 256;   // of kv8_pack_kernel

// Exclusive prefixes of two int64 a thread over the block, and their sums.
__device__ __forceinline__ void kr_scan(int64_t &x, int64_t &y, int64_t (*sh)[2], int64_t &sum_x, int64_t &sum_y) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int64_t ix = x, iy = y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t nx = __shfl_up_sync(0xffffffffu, ix, o), ny = __shfl_up_sync(0xffffffffu, iy, o);
        if (lane >= o) ix += nx, iy += ny;
    }
    if (lane == 31) sh[w][0] = ix, sh[w][1] = iy;
    __syncthreads();
    x = ix - x;
    y = iy - y;
    sum_x = sum_y = 0;
#pragma unroll
    for (int k = 0; k < KR_WARPS; ++k) {
        if (k < w) x += sh[k][0], y += sh[k][1];
        sum_x += sh[k][0];
        sum_y += sh[k][1];
    }
}

// Pages that n rows after L0 touch.
__device__ __forceinline__ int kr_pages(int L0, int n) { return n > 0 ? (L0 + n - 1) / 16 - L0 / 16 + 1 : 0; }

__device__ __forceinline__ void cp16(void *dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}

// One warp's block of one page and head (K or V) in registers, 16 rows x HD as bf16 pairs.
// K: the lane's items are (row, 8 dims, the 8 dims hd / 2 further), the halves that the
// rotation mixes.  V: the lane holds HD / 32 dims of all 16 rows, so that it can write
// a dim's 16 slots at once.
template <int HD>
struct KvBlock {
    static constexpr int C = HD / 16;       // K: 8-dim chunks of half a row
    static constexpr int RPI = 32 / C;      // K: rows an iteration
    static constexpr int NK = 16 / RPI;     // K: iterations
    static constexpr int NV = HD / 64;      // V: 32-bit words of a lane's dims of one row
    static constexpr int W = 16 * NV;       // words of a lane's share, of K too (8 an iteration: low, then high half)
};

// max(m, |x|) of a pair of bf16; a NaN stays (its bits are above infinity's)
__device__ __forceinline__ uint32_t bf2_max_abs(uint32_t m, uint32_t x) {
    uint32_t r;
    asm("{\n.reg .b32 t;\nabs.bf16x2 t, %2;\nmax.NaN.bf16x2 %0, %1, t;\n}" : "=r"(r) : "r"(m), "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t bf2_mul(uint32_t x, uint32_t y) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    return r;
}
// 2^-e twice in bf16: a block's values times it are exact, or under the least code's half
__device__ __forceinline__ uint32_t kv8_inv2(int e) { return (uint32_t)(127 - e) << 7 | (uint32_t)(127 - e) << 23; }

// The block's scale: its exponent (0 for a block with an infinity or a NaN, *bad)
template <int W>
__device__ __forceinline__ int kv8_scale(const uint32_t (&x)[W], float *scale, bool &bad) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) m = bf2_max_abs(m, x[i]);
    m = __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
    bad = m >= 0x7f80u;
    const int e = bad ? 0 : kv8_exp(m);
    if ((threadIdx.x & 31) == 0) *scale = bad ? __uint_as_float(0x7fffffffu) : kv8_pow2(e);
    return e;
}

template <int HD>
__device__ __forceinline__ void kv8_zero(uint8_t *dst) {
    for (int i = threadIdx.x & 31; i < HD; i += 32) *(uint4 *)(dst + i * 16) = make_uint4(0, 0, 0, 0);
}

// codes of a K block and its scale, from bf16 values
template <int HD>
__device__ __forceinline__ void kv8_quantise_k(const uint32_t (&x)[KvBlock<HD>::W], uint8_t *dst, float *scale) {
    using B = KvBlock<HD>;
    const int lane = threadIdx.x & 31, c = lane % B::C;
    bool bad;
    const uint32_t inv = kv8_inv2(kv8_scale(x, scale, bad));
    if (bad) return kv8_zero<HD>(dst);
#pragma unroll
    for (int i = 0; i < B::NK; ++i) {
        const int r = lane / B::C + i * B::RPI;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t w[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t u = bf2_mul(x[8 * i + 4 * half + 2 * j], inv), v = bf2_mul(x[8 * i + 4 * half + 2 * j + 1], inv);
                w[j] = e4m3x4(bf_lo(u), bf_hi(u), bf_lo(v), bf_hi(v));
            }
            const int d = half * (HD / 2) + c * 8;
            *(uint2 *)(dst + ((r >> 3) * (HD / 16) + (d >> 4)) * 128 + (r & 7) * 16 + (d & 15)) =
                make_uint2(w[0], w[1]);
        }
    }
}

// ... of a V block
template <int HD>
__device__ __forceinline__ void kv8_quantise_v(const uint32_t (&x)[KvBlock<HD>::W], uint8_t *dst, float *scale) {
    using B = KvBlock<HD>;
    const int lane = threadIdx.x & 31;
    bool bad;
    const uint32_t inv = kv8_inv2(kv8_scale(x, scale, bad));
    if (bad) return kv8_zero<HD>(dst);
    uint32_t y[B::W];
#pragma unroll
    for (int i = 0; i < B::W; ++i) y[i] = bf2_mul(x[i], inv);
#pragma unroll
    for (int j = 0; j < B::NV; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t w[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                auto val = [&](int t) { return h ? bf_hi(y[t * B::NV + j]) : bf_lo(y[t * B::NV + j]); };
                w[g] = e4m3x4(val(4 * g), val(4 * g + 1), val(4 * g + 2), val(4 * g + 3));
            }
            *(uint4 *)(dst + (lane * (HD / 32) + 2 * j + h) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
        }
}

// rows r0 .. r1 - 1 of a block from (or to) a page of bf16 rows (16 x HD)
template <int HD, bool STORE, typename T>
__device__ __forceinline__ void kv8_rows_k(uint32_t (&x)[KvBlock<HD>::W], T *page, int r0, int r1) {
    using B = KvBlock<HD>;
    const int lane = threadIdx.x & 31, c = lane % B::C;
#pragma unroll
    for (int i = 0; i < B::NK; ++i) {
        const int r = lane / B::C + i * B::RPI;
        if (r < r0 || r >= r1) continue;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            auto *at = page + r * HD + half * (HD / 2) + c * 8;
            uint32_t *w = x + 8 * i + 4 * half;
            if constexpr (STORE) {
                *(uint4 *)at = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                const uint4 v = *(const uint4 *)at;
                w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
            }
        }
    }
}
template <int HD, bool STORE, typename T>
__device__ __forceinline__ void kv8_rows_v(uint32_t (&x)[KvBlock<HD>::W], T *page, int r0, int r1) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int t = 0; t < 16; ++t) {
        if (t < r0 || t >= r1) continue;
        auto *at = page + t * HD + lane * (HD / 32);
        if constexpr (HD == 128) {
            if constexpr (STORE) {
                *(uint2 *)at = make_uint2(x[2 * t], x[2 * t + 1]);
            } else {
                const uint2 w = *(const uint2 *)at;
                x[2 * t] = w.x;
                x[2 * t + 1] = w.y;
            }
        } else {
            if constexpr (STORE) *(uint32_t *)at = x[t];
            else x[t] = *(const uint32_t *)at;
        }
    }
}

// Blocks an SM.  float32 rows come through registers, twice as many as bf16 ones: with
// three blocks (160 registers) nothing is spilled; four took 9.3 us instead of 7.5 for 1..8
// rows of 96 sequences in 8 bits, 47 instead of 43 for 17 k rows of two layers.
template <int HD, bool RF32>
constexpr int kr_blocks = RF32 ? (HD == 128 ? 3 : 4) : 5;

// A unit is one page of one sequence, for all layers and heads: the angles of its new
// positions are made once and shared by its warps, which take K or V of one layer and head
// at a time through registers: rows are read once, rotated, and written in bf16 (to the
// page, or to the tail) or, where the page is finished, as codes.  bf16 rows come by way of
// shared memory, a warp's next ones while it works on these.  Where units are few, several
// blocks (grid y) share one's layers and heads.  Units are found by a scan over the batch
// that each block keeps in registers.
//
// 33 k rows of 16 sequences, two layers of 4 heads of 128, with the lengths' update: to the
// bf16 cache 50 us, 5.5 TB/s, bound by memory (0.82 of a plain copy's rate); to the 8-bit
// one 42 us, 4.9 TB/s (0.72): some 900 instructions a 4 KB block (unpack, turn, round,
// maximum, scale, round) take 53 % of the issue slots, and the four warps meet three times
// a page.  A decode step (one row of 64 sequences) takes 4.2 and 5.4 us: the chain of
// lengths, page, rows and angles.
template <int HD, bool EIGHT, bool RF32>
__global__ void __launch_bounds__(KR_THREADS, (kr_blocks<HD, RF32>)) kv_rope_kernel(const __grid_constant__ KvRopeArgs a) {
    __shared__ int64_t sh[KR_WARPS][2];
    __shared__ float4 cs[16][HD / 4];   // cos, cos, sin, sin of dims e, e + 1 of chunk c at (e / 2) C + c: lanes side by side
    __shared__ __align__(16) uint16_t stage[RF32 ? 1 : KR_WARPS][2][RF32 ? 8 : 16 * HD];   // a warp's rows, and its next ones
    __shared__ int s_b, s_page, s_L0, s_n;
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
    const int64_t my_pages = pages;
    int64_t row0 = rows, unit0 = pages;
    kr_scan(row0, unit0, sh, total, units);
    if (__syncthreads_or(neg) || total != a.total_rows) {
        if (threadIdx.x == 0) set_status(a.status, OSPREY_ERR_INVALID_ARG);
        return;
    }
    pdl_trigger();
    // An item is K or V of a layer and head.  A warp takes K and V in turn (K, with its
    // rotation, is twice V's work): of the items 2 i and 2 i + 1 the first is K in even rounds.
    const int step = KR_WARPS * gridDim.y, step_log = __ffs(step) - 1;
    auto is_v = [&](int it) { return (it + (it >> step_log)) & 1; };
    int last_b = -1;
    bool last_ok = false;
    // a contiguous range of the units: a sequence's pages are checked once a block
    const int64_t u0 = units * blockIdx.x / gridDim.x, u1 = units * (blockIdx.x + 1) / gridDim.x;
    for (int64_t u = u0; u < u1; ++u) {
        if (u >= unit0 && u < unit0 + my_pages) {
            int64_t at = unit0, r = row0;
            for (int b = b0; b < b1; ++b) {
                const int n = a.n_rows[b], L0 = a.seq_len[b];
                const int np = n > 0 && (L0 < 0 || (int64_t)L0 + n > (int64_t)a.max_pages * 16) ? 1 : kr_pages(L0, n);
                if (u < at + np) {
                    s_b = b;
                    s_page = (int)(u - at);
                    s_row = r;
                    s_L0 = L0;
                    s_n = n;
                    break;
                }
                at += np;
                r += n;
            }
        }
        __syncthreads();
        const int b = s_b;
        const int64_t row = s_row;
        const int L0 = s_L0, n = s_n, end = L0 + n;
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
        const int p0 = L0 / 16, plast = (end - 1) / 16, TP = EIGHT ? a.tail_pages : 1, mine = p0 + s_page;
        // The ring page of p0 holds older rows that its block needs; the last new page that
        // falls on the same ring page (`clash`) is written by p0's unit, after that.
        const int clash = EIGHT && L0 % 16 ? plast - (plast - p0) % TP : p0;
        for (int pass = 0; pass < 2; ++pass) {
            if (pass == 1 && !(EIGHT && mine == p0 && clash != p0)) break;
            const int p = pass == 0 ? mine : clash;
            const bool tail = pass == 1 || (p > plast - TP && (p == p0 || p != clash));
            const int t0 = max(0, L0 - p * 16), t1 = min(16, end - p * 16);
            const bool full = EIGHT && pass == 0 && t1 == 16, work = !EIGHT || full || tail;
            const int page = tab[p], items = work ? 2 * a.layers * a.Hkv : 0;
            __align__(16) uint32_t x[Blk::W], f[RF32 ? 2 * Blk::W : 1];   // the lane's share of the block; float32 rows as they come
            // float32 rows, to registers
            auto fetch = [&](int it, int l, int h) {
                if constexpr (RF32) {
                    const int64_t first = (int64_t)l * a.total_rows + row + (int64_t)p * 16 - L0;   // row of slot 0
                    const float *src = (const float *)(is_v(it) ? a.v_rows : a.k_rows) + first * a.row_stride + h * HD;
#pragma unroll
                    for (int i = 0; i < 2 * Blk::W; ++i) f[i] = 0;
                    if (!is_v(it)) {
#pragma unroll
                        for (int i = 0; i < Blk::NK; ++i) {
                            const int r = lane / Blk::C + i * Blk::RPI;
                            if (r < t0 || r >= t1) continue;
                            const uint4 *at = (const uint4 *)(src + r * a.row_stride + lane % Blk::C * 8);
#pragma unroll
                            for (int j = 0; j < 4; ++j) *(uint4 *)(f + 16 * i + 4 * j) = __ldg(at + (j >> 1) * (HD / 8) + (j & 1));
                        }
                    } else {
#pragma unroll
                        for (int t = 0; t < 16; ++t) {
                            if (t < t0 || t >= t1) continue;
                            const float *at = src + t * a.row_stride + lane * (HD / 32);
                            if constexpr (HD == 128) *(uint4 *)(f + 4 * t) = __ldg((const uint4 *)at);
                            else *(uint2 *)(f + 2 * t) = __ldg((const uint2 *)at);
                        }
                    }
                }
            };
            // bf16 rows come by way of shared memory, the next item's while this one's are worked on
            auto ask = [&](int it, int l, int h, int slot) {
                const int64_t first = (int64_t)l * a.total_rows + row + (int64_t)p * 16 - L0;
                const uint16_t *src = (const uint16_t *)(is_v(it) ? a.v_rows : a.k_rows) + first * a.row_stride + h * HD;
                uint16_t *dst = &stage[warp][slot][0];
#pragma unroll
                for (int i = 0; i < HD / 16; ++i) {
                    const int j = lane + 32 * i, r = j / (HD / 8), d = j % (HD / 8) * 8;
                    if (r >= t0 && r < t1) cp16(dst + r * HD + d, src + r * a.row_stride + d);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            if (pass == 1) __syncthreads();   // p0's older rows are read, and so are its angles
            const int it0 = warp + blockIdx.y * KR_WARPS;
            int l = (it0 >> 1) / a.Hkv, h = (it0 >> 1) - l * a.Hkv;   // the item's layer and head
            if (it0 < items) {
                if constexpr (RF32) fetch(it0, l, h);
                else ask(it0, l, h, 0);
            }
            if (a.rotate && work)
                for (int i = threadIdx.x; i < (t1 - t0) * (HD / 2); i += KR_THREADS) {
                    const int t = t0 + i / (HD / 2), d = i % (HD / 2);
                    float *w = (float *)&cs[t][(d >> 1 & 3) * Blk::C + (d >> 3)] + (d & 1);
                    rope_cs_fix(a.freq[d], p * 16 + t, w[0], w[2]);
                }
            __syncthreads();
            int slot = 0;
            for (int it = it0; it < items; it += step, slot ^= 1) {
                const int layer = a.layer0 + l;
                int next_l = l, next_h = h + (step >> 1);
                while (next_h >= a.Hkv) next_h -= a.Hkv, ++next_l;
                const size_t blk = ((size_t)layer * a.n_pages + page) * a.Hkv + h;
                // this page's bf16 rows: the tail's, or the page's own
                const size_t at = (EIGHT ? (((size_t)layer * a.B + b) * TP + p % TP) * a.Hkv + h : blk) * 16 * HD;
                if constexpr (RF32) {
                    if (it != it0) fetch(it, l, h);
                } else {
                    __syncwarp();   // the slot has been read
                    if (it + step < items) {
                        ask(it + step, next_l, next_h, slot ^ 1);
                        asm volatile("cp.async.wait_group 1;" ::: "memory");
                    } else
                        asm volatile("cp.async.wait_group 0;" ::: "memory");
                    __syncwarp();
                    if (!is_v(it)) kv8_rows_k<HD, false>(x, &stage[warp][slot][0], 0, 16);
                    else kv8_rows_v<HD, false>(x, &stage[warp][slot][0], 0, 16);
                }
                if (!is_v(it)) {
#pragma unroll
                    for (int i = 0; i < Blk::NK; ++i) {
                        const int r = lane / Blk::C + i * Blk::RPI;
                        if (r < t0 || r >= t1 || (!RF32 && !a.rotate)) continue;
#pragma unroll
                        for (int e = 0; e < 8; e += 2) {   // pairs of dims and their partners
                            float u[2], v[2];
                            uint32_t &lo = x[8 * i + e / 2], &hi = x[8 * i + 4 + e / 2];
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                u[k] = RF32 ? __uint_as_float(f[(RF32 ? 16 * i + e + k : 0)]) : k ? bf_hi(lo) : bf_lo(lo);
                                v[k] = RF32 ? __uint_as_float(f[(RF32 ? 16 * i + 8 + e + k : 0)]) : k ? bf_hi(hi) : bf_lo(hi);
                            }
                            if (a.rotate) {
                                const float4 w = cs[r][e / 2 * Blk::C + lane % Blk::C];
                                const f2 c = mk2(w.x, w.y), u2 = mk2(u[0], u[1]), v2 = mk2(v[0], v[1]);
                                un2(fma2(v2, mk2(-w.z, -w.w), mul2(u2, c)), u[0], u[1]);
                                un2(fma2(u2, mk2(w.z, w.w), mul2(v2, c)), v[0], v[1]);
                            }
                            lo = kv8_bf2(u[0], u[1]);
                            hi = kv8_bf2(v[0], v[1]);
                        }
                    }
                    uint16_t *bf = (EIGHT ? a.k_tail : a.k_pages) + at;
                    if (!EIGHT || tail) kv8_rows_k<HD, true>(x, bf, t0, t1);
                    if (full) {
                        if (t0 > 0) kv8_rows_k<HD, false>(x, bf, 0, t0);   // older rows (t0 > 0: p is p0, its own ring page)
                        kv8_quantise_k<HD>(x, a.k8 + blk * 16 * HD, a.k_scale + blk);
                    }
                } else {
                    if constexpr (RF32)
#pragma unroll
                        for (int i = 0; i < Blk::W; ++i) x[i] = kv8_bf2(__uint_as_float(f[2 * i]), __uint_as_float(f[2 * i + 1]));
                    uint16_t *bf = (EIGHT ? a.v_tail : a.v_pages) + at;
                    if (!EIGHT || tail) kv8_rows_v<HD, true>(x, bf, t0, t1);
                    if (full) {
                        if (t0 > 0) kv8_rows_v<HD, false>(x, bf, 0, t0);
                        kv8_quantise_v<HD>(x, a.v8 + blk * 16 * HD, a.v_scale + blk);
                    }
                }
                l = next_l;
                h = next_h;
            }
        }
        __syncthreads();   // cs and s_b are read
    }
}

template <int HD, bool EIGHT, bool RF32>
static cudaError_t launch_kv_rope_t(const KvRopeArgs &a, int sms, cudaStream_t s) {
    // units: n rows touch at most n / 16 + 2 pages, and no more pages than rows
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(a.total_rows, a.total_rows / 16 + 2LL * a.B));
    const int64_t cap = kr_blocks<HD, RF32> * (int64_t)sms;   // as many as are resident
    // few units: up to four blocks share one's layers and heads
    const int share = most * 4 <= cap && 2 * a.layers * a.Hkv > 2 * KR_WARPS ? 4 : most * 2 <= cap && 2 * a.layers * a.Hkv > KR_WARPS ? 2 : 1;
    // More units than that: a block takes several in a row; but one where a unit is little more
    // than its copy (bf16) or made of small items (head_dim 64), and finding it is cheap (up to
    // four sequences a thread).  us, one a block / several: bf16, 16 sequences 50.0 / 53.7, 100
    // 43.3 / 45.3, 512 50.2 / 53.1, 2048 74 / 47; 8 bits, 16 sequences 44.0 / 42.2, of head_dim
    // 64 54.6 / 60.1, 2048 91 / 65.
    const int64_t most_blocks = ((!EIGHT || HD == 64) && a.B <= 4 * KR_THREADS ? 16 : 1) * cap;
    kv_rope_kernel<HD, EIGHT, RF32><<<dim3((unsigned)std::min(most, most_blocks), share), KR_THREADS, 0, s>>>(a);
    count_launch();
    return cudaGetLastError();
}

cudaError_t launch_kv_rope(const KvRopeArgs &a, bool eight, bool advance, int sms, cudaStream_t s) {
    cudaError_t e;
    if (a.hd == 128)
        e = eight ? (a.rows_f32 ? launch_kv_rope_t<128, true, true>(a, sms, s) : launch_kv_rope_t<128, true, false>(a, sms, s))
                  : (a.rows_f32 ? launch_kv_rope_t<128, false, true>(a, sms, s) : launch_kv_rope_t<128, false, false>(a, sms, s));
    else
        e = eight ? (a.rows_f32 ? launch_kv_rope_t<64, true, true>(a, sms, s) : launch_kv_rope_t<64, true, false>(a, sms, s))
                  : (a.rows_f32 ? launch_kv_rope_t<64, false, true>(a, sms, s) : launch_kv_rope_t<64, false, false>(a, sms, s));
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

// Finished pages of a draft call's committed rows, from the tail: one warp K or V of a
// layer and head, one block a page.
template <int HD>
__global__ void __launch_bounds__(PK_THREADS) kv8_pack_kernel(const Kv8PackArgs a) {
    const int b = blockIdx.y, warp = threadIdx.x >> 5;
    if (!a.valid[b]) return;
    const int p = a.pos0[b] / 16 + blockIdx.x;
    if ((p + 1) * 16 > a.pos0[b] + a.nnew[b]) return;
    const int page = a.page_table[(size_t)b * a.max_pages + p];   // in range: the call's first kernel has checked it
    for (int it = warp; it < 2 * a.L * a.Hkv; it += PK_THREADS / 32) {
        const int lh = it >> 1, l = lh / a.Hkv, h = lh - l * a.Hkv;
        const size_t t = ((((size_t)l * a.B + b) * a.tail_pages + p % a.tail_pages) * a.Hkv + h) * 16 * HD;
        const size_t blk = ((size_t)l * a.n_pages + page) * a.Hkv + h;
        __align__(16) uint32_t x[KvBlock<HD>::W];
        if ((it + it / (PK_THREADS / 32)) % 2 == 0) {   // K and V in turn, as above
            kv8_rows_k<HD, false>(x, a.k_tail + t, 0, 16);
            kv8_quantise_k<HD>(x, a.k8 + blk * 16 * HD, a.k_scale + blk);
        } else {
            kv8_rows_v<HD, false>(x, a.v_tail + t, 0, 16);
            kv8_quantise_v<HD>(x, a.v8 + blk * 16 * HD, a.v_scale + blk);
        }
    }
}

cudaError_t launch_kv8_pack(const Kv8PackArgs &a, cudaStream_t s) {
    const dim3 grid((a.max_new + 14) / 16 + 1, a.B);   // pages that max_new rows finish, at most
    if (a.hd == 128) kv8_pack_kernel<128><<<grid, PK_THREADS, 0, s>>>(a);
    else kv8_pack_kernel<64><<<grid, PK_THREADS, 0, s>>>(a);
    count_launch();
    return cudaGetLastError();
}

}  // namespace osp
