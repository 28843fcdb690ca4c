// Operators of the bf16 paged cache for long and shared contexts: pages for new rows,
// bounds of a page's keys, the choice of pages by them, attention.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "osprey.h"

namespace osp {

// ---------------------------------------------------------------- pages for new rows
struct KvReserveArgs {
    int B;
    const int32_t *n_rows, *seq_len, *share;   // share may be null
    int32_t *page_table;
    int max_pages, n_pages;
    const int32_t *free_pages;
    int n_free;
    int32_t *n_taken;
    int32_t *held;                             // pages of each sequence's row, or null: those that seq_len needs
    int64_t *slots;                            // may be null
    int total_rows;
    int32_t *status;
};
cudaError_t launch_kv_reserve(const KvReserveArgs &a, cudaStream_t s);

// ---------------------------------------------------------------- bounds of a page's keys
struct KvBoundArgs {
    int B, max_rows, layers, Hkv, hd, advanced;   // from the first layer of the pointers on
    const int32_t *n_rows, *seq_len, *page_table;
    int max_pages, n_pages;
    const uint16_t *k_pages;
    int8_t *codes;   // [layers][n_pages][Hkv][2][hd]
    float *scale;    // [layers][n_pages][Hkv]
    int32_t *status;
};
cudaError_t launch_kv_bound(const KvBoundArgs &a, cudaStream_t s);

// ---------------------------------------------------------------- pages to read
struct KvSelectArgs {
    int B, max_rows, Hq, Hkv, hd, advanced;
    const int32_t *n_rows, *seq_len, *page_table;
    int max_pages, n_pages;
    const int8_t *codes;    // this layer's
    const float *scale;
    const void *q;
    int q_f32, rotate;
    int64_t q_stride;
    uint64_t freq[64];
    int n_select, n_first, n_last;
    int32_t *pages;         // [B][max_rows][Hkv][n_select]
    uint32_t *keys;         // workspace: [B][max_rows][Hkv][max_pages]
    int32_t *status;
};
cudaError_t launch_kv_select(const KvSelectArgs &a, int sms, cudaStream_t s);

// ---------------------------------------------------------------- attention
struct KvAttendArgs {
    int B, max_rows, Hq, Hkv, hd, advanced;
    const int32_t *n_rows, *seq_len, *page_table;
    int max_pages, n_pages;
    const uint16_t *k_pages, *v_pages;     // this layer's
    const int32_t *share, *shared_len;     // both or neither
    const int32_t *pages;                  // lists of n_select pages a row and KV head, or null
    int n_select;
    const void *q;
    int q_f32, rotate;
    int64_t q_stride;
    uint64_t freq[64];
    void *out;
    int32_t *status;
};
cudaError_t launch_kv_attend(const KvAttendArgs &a, void *workspace, int sms, cudaStream_t s);
size_t kv_attend_workspace(int B, int max_rows, int Hq, int Hkv, int hd, bool lists, int sms);

// What a call has of one sequence: its rows and their positions.
struct SeqRows {
    int n, base;        // rows, position of the first one
    int code;           // an error's code, or 0
};
__device__ __forceinline__ SeqRows seq_rows(int n, int len, int advanced, int max_rows, int max_pages) {
    SeqRows r;
    const int64_t total = (int64_t)len + (advanced ? 0 : max(n, 0));
    r.code = n < 0 || n > max_rows || len < 0 || total < n ? OSPREY_ERR_INVALID_ARG
             : total > (int64_t)max_pages * 16             ? OSPREY_ERR_CAPACITY
                                                           : 0;
    r.n = r.code ? min(max(n, 0), max_rows) : n;
    r.base = r.code ? 0 : (int)(total - n);
    return r;
}

// Smallest e, -100 at least, with |x| <= 127 * 2^e, of a finite magnitude's bits.
__device__ __forceinline__ int exp127(uint32_t mag) {
    const int e = (int)(mag >> 23) - 127 - 6 + ((mag & 0x7fffffu) > 0x7e0000u ? 1 : 0);
    return e < -100 ? -100 : e;
}

}  // namespace osp
