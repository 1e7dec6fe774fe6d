// The paged cache's kernels: their arguments and launchers (kl_paged.hip), for
// the host entry points (kl_paged_host.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "kl.h"

namespace kl {

constexpr int kMaxGroup = 16;        // query heads per KV head
constexpr int kMaxPagedBatch = 4096; // sequences of an attention call
constexpr int kPagedGroups = 256;    // workgroups of an attention call, at most
// The workspace of an attention call: parts for any group and head_dim, then
// the arrival counters (at the same place whatever the call's shape, so that a
// workspace serves calls of all shapes).
constexpr size_t kPagedPartBytes = (size_t)kPagedGroups * 2 * kMaxGroup * (128 + 2) * sizeof(float);

// One layer of a pool.
struct PagedLayer {
    uint8_t *k, *v;                  // rows of values or codes
    uint8_t *ks, *vs;                // scale bytes (e4m3)
    int n_pages, nkv, page_log2, d;
    bool e4m3;
};

struct PagedTable {
    const int32_t *pages;
    int batch, max_pages, stride;
};

// kl_paged_append and kl_paged_read
struct RowParams {
    PagedLayer c;
    PagedTable t;
    const int32_t *seq, *positions;
    long long rows;
    void *k, *v;                     // the caller's rows
    int k_type, v_type;
    long long k_row, k_head, v_row, v_head;   // strides, elements
    bool k_vec, v_vec;               // 8 elements of a head may be moved as 16-byte words
    int32_t *error;
};
// A paged step's sequences: position and length of each for its launches.
// Sequence b attends lengths[b] positions and its row goes to append_pos[b] (-1:
// none); step_pos[b] is its position, -1 where its pages are bad (checked up to
// that position's; KL_DEVERR_PAGE).
struct StepRowsParams {
    const int32_t *tokens, *positions;
    int vocab, cap, n_pages, page_log2, batch;
    PagedTable t;
    int32_t *step_pos, *append_pos, *lengths;
    int32_t *error;
};
hipError_t launch_paged_step_rows(const StepRowsParams &p, hipStream_t stream);

hipError_t launch_paged_append(const RowParams &p, hipStream_t stream);
hipError_t launch_paged_read(const RowParams &p, hipStream_t stream);

// kl_paged_attention
struct AttnParams {
    PagedLayer c;
    PagedTable t;
    const int32_t *lengths;
    const void *q;
    void *out;
    int q_type, out_type, nq, group;
    bool q_vec, out_vec;             // as k_vec
    long long q_row, q_head, out_row, out_head;
    float scale;
    int window;
    uint16_t *out_lo;                // with bf16 'out': its second bf16 term (a step's attention)
    float *lse;
    float *parts;                    // workspace: [workgroup][2][group][d + 2]
    unsigned *arrived;               // workspace: [batch][nkv], zero between calls
    int32_t *error;
};
hipError_t launch_paged_attention(const AttnParams &p, hipStream_t stream);
hipError_t launch_paged_attention_d64(const AttnParams &p, hipStream_t stream);
hipError_t launch_paged_attention_d128(const AttnParams &p, hipStream_t stream);

// Host checks shared by the entry points (kl_paged_host.cpp).
kl_status check_paged_pool(const kl_paged_cache *c, int32_t layer, const kl_page_table *t,
                           const char *who);
PagedLayer paged_layer(const kl_paged_cache &c, int32_t layer);

}  // namespace kl
