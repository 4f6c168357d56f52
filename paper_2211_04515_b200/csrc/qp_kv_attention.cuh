// What the attention kernels over the 4-bit cache are given.
#pragma once

#include <type_traits>

#include "qp_kv.cuh"

constexpr int QP_KV_MAX_DEVICES = 64;
constexpr int QP_KV_COUNTERS = 4096;             // of a plan's workspace: two levels, two for each block

struct qp_kv_attn_args {
    qp_kv_rows rows;
    qp_kv_pages pages;
    const char* pool;                            // of the layer
    int heads, slices;                           // cached heads, slices of a page
    int q_heads, group, max_new, window;
    float scale_log2;                            // scale * log2(e)
    const void* q;
    int64_t qt, qh;
    void* out;
    int64_t ot, oh;
    float* lse;
    bool vec, out_vec;                           // 16-byte loads of q; stores of four elements
    bool zero_rest;                              // rows that no sequence writes become 0
    unsigned* count;
    float* part;
    unsigned* status;
    int many;                                    // sequences with so many query rows to a cached head, or more, are qp_kv_chunk.cu's
    long long wait_cycles;
};

// qp_kv_chunk.cu: the sequences with many rows.  Workspace for parts of items, and the launch.
uint64_t qp_kv_chunk_part_bytes(int head_dim, int sm_count);
int32_t qp_kv_chunk_launch(qp_ctx* ctx, const qp_kv_attn_args& a, int head_dim, cudaStream_t s);
