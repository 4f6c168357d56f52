// The 4-bit cache of keys and values, as its kernels see it: memory format, batch look-ups, argument checks.
#pragma once

#include "qp_internal.cuh"

constexpr int QP_KV_SLICE = 16;                  // tokens of a slice
constexpr int QP_KV_MAX_PAGE = 1024;

static inline bool qp_kv_dim_ok(int d) { return d == 64 || d == 128 || d == 256; }

// places inside a slice of 16 tokens
template <int D>
struct qp_kv_slice {
    static constexpr int ROW = D / 2;                            // bytes of a row's codes
    static constexpr int CODES = QP_KV_SLICE * ROW;
    static constexpr int QUANT = QP_KV_SLICE * 8;
    static constexpr int KQ = CODES, V = CODES + QUANT, VQ = 2 * CODES + QUANT;
    static constexpr int BYTES = 2 * (CODES + QUANT);
};

int32_t qp_kv_check_cache(qp_ctx* ctx, const qp_kv_cache_t* c);                     // (qp_kv_rows.cu)
int32_t qp_kv_check_batch(qp_ctx* ctx, const qp_kv_batch_t* b);
int32_t qp_kv_check_layer(qp_ctx* ctx, const qp_kv_cache_t* c, int layer);

#ifdef __CUDACC__

// The cache's calls follow one another in a stream, and the small ones are little more than their launches.  So each kernel
// may be set up while the one before it still runs (programmatic dependent launch): its first statement waits until that one
// is through and its writes are there, and it lets the next be set up in turn.  What a kernel reads may therefore have been written
// during its lifetime, though never after that wait: its loads are ordinary ones, not those of the read-only path.
__device__ __forceinline__ void qp_kv_begin()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
template <typename T> __device__ __forceinline__ T qp_kv_ld(const T* p) { return *p; }

template <typename... P, typename... A>
static inline void qp_kv_launch(void (*f)(P...), unsigned blocks, unsigned threads, size_t smem, cudaStream_t s, A... args)
{
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(blocks);
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &at;
    c.numAttrs = 1;
    cudaLaunchKernelEx(&c, f, args...);                          // (an error is found by qp_check_launch)
}

// the batch, from the device's side
struct qp_kv_rows {
    const int32_t *slots, *start, *pos;
    int batch, tokens;
};
static inline qp_kv_rows qp_kv_rows_of(const qp_kv_batch_t* b) { return {b->d_slots, b->d_start, b->d_pos, b->batch, b->tokens}; }

// row that sequence b begins with, the end of the one before it; within the rows that there are, so that no row at or behind
// `tokens` is anybody's
__device__ __forceinline__ int qp_kv_start(const qp_kv_rows& r, int b)
{
    const int s = r.start ? qp_kv_ld(r.start + b) : b;
    return s < 0 ? 0 : s > r.tokens ? r.tokens : s;
}
__device__ __forceinline__ int qp_kv_slot(const qp_kv_rows& r, int b) { return r.slots ? qp_kv_ld(r.slots + b) : b; }

// page of token position p of a slot, -1 if the cache has none
struct qp_kv_pages {
    const int32_t* table;
    int num_pages, page_size, max_seqs, max_pages;
};
static inline qp_kv_pages qp_kv_pages_of(const qp_kv_cache_t* c)
{
    return {c->d_table, c->num_pages, c->page_size, c->max_seqs, c->max_pages};
}
__device__ __forceinline__ int qp_kv_page(const qp_kv_pages& c, int slot, int p)
{
    const int i = p / c.page_size;
    if (slot < 0 || slot >= c.max_seqs || p < 0 || i >= c.max_pages) return -1;
    const int page = qp_kv_ld(c.table + (size_t)slot * c.max_pages + i);
    return page >= 0 && page < c.num_pages ? page : -1;
}

#endif
