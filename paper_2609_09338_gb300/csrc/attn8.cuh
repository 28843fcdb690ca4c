// Attention over the 8-bit paged cache (kv8.cuh).
#pragma once

#include "draft.cuh"
#include "kv8.cuh"

namespace osp {

struct Attn8Args {
    int B, Hq, Hkv, hd, max_rows;     // query rows of a sequence: at most max_rows
    // rows: the newest n_rows[b] positions of seq_len[b] (advanced) or of seq_len[b] + n_rows[b], every page
    // that these complete in 8 bits; or, in a draft call, a row map: the rows of a step, 8 bits up to pos0
    const int32_t *seq_len, *n_rows;
    int advanced;
    RowMap map;                       // used when seq_len is null
    const uint8_t *k8, *v8;           // this layer's pages
    const float *k_scale, *v_scale;
    const uint16_t *k_tail, *v_tail;  // this layer's tail
    const int32_t *page_table;
    int max_pages, n_pages, tail_pages;
    const void *q;                    // [B][max_rows] rows q_stride elements apart, each [Hq][hd]
    int q_f32, rotate;
    int64_t q_stride;
    uint64_t freq[64];
    void *out;                        // [B][max_rows][Hq][hd], of q's type; or
    AttnArgs planes;                  // a draft call's output (attn_store), when planes.q is set
    int32_t *status;
};
cudaError_t launch_attn8(const Attn8Args &a, int sms, cudaStream_t s);

}  // namespace osp
