// Pages of the 4-bit cache of keys and values: growing, forking and freeing sequences, copying pages, compacting the pool.
//
// Which pages a call takes is decided by one block, from the tables alone: the free pages are those with refs 0, and the k-th
// one wanted is the k-th lowest.  Ranks come from ballots and prefix sums, so the outcome does not depend on timing.
// These tables are small (a pool of 8192 pages has 32 KB of refs) and one block reads them in a few round trips, which
// is what the call costs: 3 to 5 us.  A second launch over the whole GPU then moves the bytes, where there are any:
// 16 bytes a thread, eight loads in flight, bound by HBM at 2 bytes per byte copied.  1001 pages of 73728 bytes in 2 layers: 50.9 us,
// 43.6 of them the move (6.8 TB/s); compacting 4096 pages, 2 layers: 35.3, 25.5 of them the move.
#include "qp_kv.cuh"

QP_CK_UNIT

namespace {

constexpr int PLAN = 1024;                       // threads of a deciding block
constexpr int PW = PLAN / 32;
constexpr int NONE = 0x7FFFFFFF;
constexpr int SMEM_CLAIMS = 4096;                // slots whose claims fit shared memory
constexpr int SMEM_TAKEN = 2048;                 // pages

struct Cache {
    int32_t *table, *lens, *refs;
    int num_pages, page_size, max_seqs, max_pages;
    int32_t *head, *a, *b, *c;                   // d_work: [64] and three lists of pages,
    int32_t *s0, *s1, *s2;                       // three of slots
    unsigned* status;
};

Cache cache_of(const qp_ctx* ctx, const qp_kv_cache_t* c)
{
    Cache r;
    r.table = c->d_table; r.lens = c->d_lens; r.refs = c->d_refs;
    r.num_pages = c->num_pages; r.page_size = c->page_size; r.max_seqs = c->max_seqs; r.max_pages = c->max_pages;
    r.head = c->d_work;
    r.a = r.head + 64; r.b = r.a + c->num_pages; r.c = r.b + c->num_pages;
    r.s0 = r.c + c->num_pages; r.s1 = r.s0 + c->max_seqs; r.s2 = r.s1 + c->max_seqs;
    r.status = ctx->d_status;
    return r;
}

__device__ __forceinline__ int pages_of(int tokens, int page_size) { return (int)(((unsigned)tokens + page_size - 1) / page_size); }

// exclusive prefix sum of v over the block; total: the whole sum.  sh: PW + 1 ints
__device__ __forceinline__ int block_scan(int v, int* sh, int& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();                                             // sh is free
    if (lane == 31) sh[warp] = x;
    __syncthreads();
    if (warp == 0) {
        int w = sh[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xFFFFFFFFu, w, o);
            if (lane >= o) w += y;
        }
        sh[lane] = w;
    }
    __syncthreads();
    total = sh[PW - 1];
    return x - v + (warp ? sh[warp - 1] : 0);
}

// calls put(rank, page) for the pages of ascending number with which(page, refs), rank from `from` on, until `most`
// are found or the pool ends; returns how many there are so far.  PER pages a thread and round.
constexpr int PER = 8;
template <typename W, typename P>
__device__ __forceinline__ int for_pages(const Cache& c, int from, int most, int* sh, W which, P put)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int base = 0; base < c.num_pages && from < most; base += PER * PLAN) {
        // warp w takes pages base + w * 32 * PER .. , so that the ranks of a warp are consecutive
        const int p0 = base + warp * 32 * PER + lane;
        int refs[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) refs[i] = p0 + 32 * i < c.num_pages ? __ldcg(c.refs + p0 + 32 * i) : 0;
        unsigned m[PER];
        int n = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            m[i] = __ballot_sync(0xFFFFFFFFu, p0 + 32 * i < c.num_pages && which(p0 + 32 * i, refs[i]));
            n += __popc(m[i]);
        }
        int total;
        int rank = from + __shfl_sync(0xFFFFFFFFu, block_scan(lane == 0 ? n : 0, sh, total), 0);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (m[i] >> lane & 1u) {
                const int r = rank + __popc(m[i] & ((1u << lane) - 1u));
                if (r < most) put(r, p0 + 32 * i);
            }
            rank += __popc(m[i]);
        }
        from += total;
    }
    return from < most ? from : most;
}

// claim[slot] = the first of n entries that names it.  Entries out of range claim nothing.
__device__ __forceinline__ volatile int* claim_slots(const Cache& c, const int32_t* slots, int n, int* sh_claim)
{
    volatile int* claim = c.max_seqs <= SMEM_CLAIMS ? sh_claim : c.s0;
    for (int i = threadIdx.x; i < n; i += PLAN) {
        const int s = qp_kv_ld(slots + i);
        if (s >= 0 && s < c.max_seqs) claim[QP_CK(s, c.max_seqs <= SMEM_CLAIMS ? SMEM_CLAIMS : c.max_seqs)] = NONE;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += PLAN) {
        const int s = qp_kv_ld(slots + i);
        if (s >= 0 && s < c.max_seqs) atomicMin(const_cast<int*>(claim) + s, i);
    }
    __syncthreads();
    return claim;
}

// ---------------------------------------------------------------------------- growing

__global__ void __launch_bounds__(PLAN) kv_extend_kernel(const Cache c, const int32_t* slots,
                                                         const int32_t* start, int32_t* pos, int batch,
                                                         int tokens, int max_new)
{
    qp_kv_begin();
    __shared__ int sh[PW + 1], sh_claim[SMEM_CLAIMS], sh_taken[SMEM_TAKEN];
    volatile int* claim = slots ? claim_slots(c, slots, batch, sh_claim) : nullptr;
    bool range = false;
    int wanted = 0;
    for (int b0 = 0; b0 < batch; b0 += PLAN) {
        const int b = b0 + threadIdx.x;
        int need = 0, old = -1;
        if (b < batch) {
            const int s = slots ? qp_kv_ld(slots + b) : b;
            int64_t n = 1;
            if (start) {
                const int64_t s0 = qp_kv_ld(start + b), s1 = qp_kv_ld(start + b + 1);
                n = s1 - s0;
                if (s0 < 0 || n < 0 || s1 > tokens) n = -1;
            } else if (b >= tokens) {
                n = -1;
            }
            if (n >= 0 && n <= max_new && s >= 0 && s < c.max_seqs && (!claim || claim[s] == b)) {
                const int64_t l = __ldcg(c.lens + s);
                if (l >= 0 && l + n <= (int64_t)c.max_pages * c.page_size) {
                    old = (int)l;
                    need = pages_of((int)(l + n), c.page_size) - pages_of((int)l, c.page_size);
                }
            }
            range |= old < 0;
        }
        int total;
        // d_start need not ascend, so that many entries may ask for most of 2^31 tokens each: the sum is bounded first, without overflow
        // (up to 2^23 tokens an entry 1024 of them want at most 2^29 + 2^10 pages)
        if (max_new > 1 << 23) {                                 // uniform
            block_scan(need >> 11, sh, total);
            if (total > c.num_pages >> 11) { wanted = c.num_pages + 1; break; }
        }
        const int at = wanted + block_scan(need, sh, total);
        if (b < batch) { c.s1[QP_CK(b, c.max_seqs)] = at; c.s2[QP_CK(b, c.max_seqs)] = old; }
        wanted += total;                                         // (at most 2^29 before, 2^29 + 2^21 added)
        if (wanted > c.num_pages) break;                         // uniform
    }
    int* taken = wanted <= SMEM_TAKEN ? sh_taken : c.a;
    int found = 0;
    if (wanted <= c.num_pages)
        found = for_pages(c, 0, wanted, sh, [](int, int refs) { return refs == 0; }, [&](int r, int p) { taken[QP_CK(r, wanted <= SMEM_TAKEN ? SMEM_TAKEN : c.num_pages)] = p; });
    __syncthreads();
    if (found < wanted) {
        for (int b = threadIdx.x; b < batch; b += PLAN) pos[b] = -1;
        if (threadIdx.x == 0) atomicOr(c.status, QP_DEV_KV_EXHAUSTED);
    } else {
        for (int k = threadIdx.x; k < wanted; k += PLAN) {
            int lo = 0, hi = batch;                              // the last b with s1[b] <= k: entries that want none share s1 with the next
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (c.s1[mid] <= k) lo = mid; else hi = mid;
            }
            const int s = slots ? qp_kv_ld(slots + lo) : lo;
            c.table[(size_t)s * c.max_pages + QP_CK(pages_of(c.s2[lo], c.page_size) + (k - c.s1[lo]), c.max_pages)] = taken[k];
            c.refs[QP_CK(taken[k], c.num_pages)] = 1;
        }
        for (int b = threadIdx.x; b < batch; b += PLAN) {
            const int old = c.s2[b];
            pos[b] = old;
            if (old >= 0) c.lens[slots ? qp_kv_ld(slots + b) : b] = old + (start ? qp_kv_ld(start + b + 1) - qp_kv_ld(start + b) : 1);
        }
    }
    if (range) atomicOr(c.status, QP_DEV_KV_RANGE);
}

// ---------------------------------------------------------------------------- freeing

__global__ void __launch_bounds__(128) kv_free_kernel(const Cache c, const int32_t* slots, int n)
{
    qp_kv_begin();
    __shared__ int sh_len;
    for (int i = blockIdx.x; i < n; i += gridDim.x) {
        const int s = qp_kv_ld(slots + i);
        if (s < 0 || s >= c.max_seqs) {
            if (threadIdx.x == 0) atomicOr(c.status, QP_DEV_KV_RANGE);
            continue;
        }
        if (threadIdx.x == 0) sh_len = atomicExch(c.lens + s, 0);    // of several entries with one slot, one gets its length
        __syncthreads();
        const int len = sh_len;
        __syncthreads();
        int m = len > 0 ? pages_of(len, c.page_size) : 0;
        if (m > c.max_pages) m = c.max_pages;
        int32_t* row = c.table + (size_t)s * c.max_pages;
        for (int j = threadIdx.x; j < m; j += blockDim.x) {
            const int p = row[j];
            if (p >= 0 && p < c.num_pages) atomicSub(c.refs + p, 1);
            else atomicOr(c.status, QP_DEV_KV_RANGE);
            row[j] = -1;
        }
    }
}

// ---------------------------------------------------------------------------- moving pages

struct Moves {
    char* pool;
    uint64_t layer_stride, page_bytes;
    int layers, chunks;                          // pieces of a page
    const int32_t *src, *dst;                    // page pairs; src < 0: none
    int num_pages;
};

constexpr int MOVE_THREADS = 256, MOVE_VECS = 8;
constexpr int MOVE_BYTES = MOVE_THREADS * MOVE_VECS * 16;

// piece t of the moves: pair t / (layers * chunks)
__device__ __forceinline__ void move_piece(const Moves& m, int64_t t)
{
    const int per = m.layers * m.chunks;
    const int64_t k = t / per;
    const int rest = (int)(t - k * per), layer = rest / m.chunks, piece = rest - layer * m.chunks;
    const int from = m.src[k], to = m.dst[k];
    if (from < 0 || from >= m.num_pages || to < 0 || to >= m.num_pages) return;
    const uint64_t at = (uint64_t)piece * MOVE_BYTES;
    char* base = m.pool + (uint64_t)layer * m.layer_stride + at;
    const uint4* x = reinterpret_cast<const uint4*>(base + (uint64_t)from * m.page_bytes);
    uint4* y = reinterpret_cast<uint4*>(base + (uint64_t)to * m.page_bytes);
    const int n = (int)((m.page_bytes - at < MOVE_BYTES ? m.page_bytes - at : MOVE_BYTES) / 16);
    uint4 v[MOVE_VECS];
    if (n == MOVE_BYTES / 16) {
#pragma unroll
        for (int i = 0; i < MOVE_VECS; ++i) v[i] = __ldcs(x + i * MOVE_THREADS + threadIdx.x);
#pragma unroll
        for (int i = 0; i < MOVE_VECS; ++i) __stcs(y + i * MOVE_THREADS + threadIdx.x, v[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < MOVE_VECS; ++i)
        if (i * MOVE_THREADS + (int)threadIdx.x < n) v[i] = __ldcs(x + i * MOVE_THREADS + threadIdx.x);
#pragma unroll
    for (int i = 0; i < MOVE_VECS; ++i)
        if (i * MOVE_THREADS + (int)threadIdx.x < n) __stcs(y + i * MOVE_THREADS + threadIdx.x, v[i]);
}

__global__ void __launch_bounds__(MOVE_THREADS) kv_move_kernel(const Moves m, int n)
{
    qp_kv_begin();
    const int64_t pieces = (int64_t)n * m.layers * m.chunks;
    for (int64_t t = blockIdx.x; t < pieces; t += gridDim.x) move_piece(m, t);
}

Moves moves_of(const qp_kv_cache_t* c, const Cache& k)
{
    Moves m;
    m.pool = static_cast<char*>(c->d_pool);
    m.layer_stride = c->layer_stride;
    m.page_bytes = (uint64_t)c->heads * (uint64_t)(c->page_size / QP_KV_SLICE) * qp_kv_slice_bytes(c->head_dim);
    m.layers = c->layers;
    m.chunks = (int)((m.page_bytes + MOVE_BYTES - 1) / MOVE_BYTES);
    m.src = k.a; m.dst = k.b;
    m.num_pages = c->num_pages;
    return m;
}

unsigned move_grid(const qp_ctx* ctx, int64_t tasks)
{
    const int64_t cap = (int64_t)ctx->sm_count * 16;
    return (unsigned)(tasks < 1 ? 1 : tasks < cap ? tasks : cap);
}

// ---------------------------------------------------------------------------- forking

// Pair i: s2[i] = tokens it copies (-1: it is skipped), a[i], b[i] = the part-filled page and the page that takes its copy (-1: none)
__global__ void __launch_bounds__(PLAN) kv_fork_plan_kernel(const Cache c, const int32_t* src,
                                                            const int32_t* dst, int n)
{
    qp_kv_begin();
    __shared__ int sh[PW + 1], sh_claim[SMEM_CLAIMS];
    volatile int* claim = claim_slots(c, dst, n, sh_claim);
    bool range = false;
    int wanted = 0;
    for (int i0 = 0; i0 < n; i0 += PLAN) {
        const int i = i0 + threadIdx.x;
        int len = -1, tail = 0;
        if (i < n) {
            const int s = qp_kv_ld(src + i), d = qp_kv_ld(dst + i);
            if (s >= 0 && s < c.max_seqs && d >= 0 && d < c.max_seqs && claim[d] == i && __ldcg(c.lens + d) == 0) {
                len = __ldcg(c.lens + s);
                if (len < 0 || len > (int64_t)c.max_pages * c.page_size) len = -1;
                tail = len > 0 && len % c.page_size != 0;
            }
            range |= len < 0;
        }
        int total;
        const int at = wanted + block_scan(tail, sh, total);
        if (i < n) { c.s1[QP_CK(i, c.max_seqs)] = tail ? at : -1; c.s2[QP_CK(i, c.max_seqs)] = len; }
        wanted += total;
    }
    // the pages for the copies into list c, then to the pairs
    const int found = wanted <= c.num_pages
                          ? for_pages(c, 0, wanted, sh, [](int, int refs) { return refs == 0; }, [&](int r, int p) { c.c[QP_CK(r, c.num_pages)] = p; })
                          : 0;
    __syncthreads();
    const bool enough = found >= wanted;
    for (int i = threadIdx.x; i < n; i += PLAN) {
        const int at = c.s1[i], len = c.s2[i];
        if (!enough) { c.s2[i] = -1; continue; }
        if (len < 0) continue;
        c.lens[qp_kv_ld(dst + i)] = len;                            // (the lengths were all read above)
        if (at >= 0) {
            const int p = c.c[QP_CK(at, c.num_pages)];
            c.refs[QP_CK(p, c.num_pages)] = 1;
            c.s1[i] = p;
        }
    }
    if (!enough && threadIdx.x == 0) atomicOr(c.status, QP_DEV_KV_EXHAUSTED);
    if (range) atomicOr(c.status, QP_DEV_KV_RANGE);
}

// tasks 0 .. n - 1: the pairs' table rows; behind them the pieces of the part-filled pages
__global__ void __launch_bounds__(MOVE_THREADS) kv_fork_kernel(const Cache c, const Moves m, const int32_t* src,
                                                               const int32_t* dst, int n)
{
    qp_kv_begin();
    const int per = m.layers * m.chunks;
    const int64_t tasks = n + (int64_t)n * per;
    for (int64_t t = blockIdx.x; t < tasks; t += gridDim.x) {
        const int i = (int)(t < n ? t : (t - n) / per);
        const int len = c.s2[i];
        if (len <= 0) continue;
        const int full = len / c.page_size;
        const int32_t* from = c.table + (size_t)qp_kv_ld(src + i) * c.max_pages;
        const bool tail = len % c.page_size != 0;
        if (t < n) {
            int32_t* to = c.table + (size_t)qp_kv_ld(dst + i) * c.max_pages;
            for (int j = threadIdx.x; j < full; j += MOVE_THREADS) {
                const int p = from[j];
                to[j] = p;
                if (p >= 0 && p < c.num_pages) atomicAdd(c.refs + p, 1);
            }
            if (tail && threadIdx.x == 0) to[full] = c.s1[i];
        } else if (tail) {
            Moves one = m;
            const int32_t pair[2] = {from[full], c.s1[i]};
            one.src = pair; one.dst = pair + 1;
            move_piece(one, t - n - (int64_t)i * per);
        }
    }
}

// ---------------------------------------------------------------------------- copying

constexpr int SMEM_PAGES = 12288;                // pages whose claims fit shared memory

__global__ void __launch_bounds__(PLAN) kv_copy_plan_kernel(const Cache c, const int32_t* src,
                                                            const int32_t* dst, int n, bool in_shared)
{
    qp_kv_begin();
    extern __shared__ int sh_claims[];
    int* list = in_shared ? sh_claims : c.c;                     // per page: the first pair that writes it
    volatile int* claim = list;
    auto ok = [&](int p) { return p >= 0 && p < c.num_pages; };
    for (int i = threadIdx.x; i < n; i += PLAN) {
        const int s = qp_kv_ld(src + i), d = qp_kv_ld(dst + i);
        if (ok(s) && ok(d)) claim[QP_CK(s, c.num_pages)] = claim[QP_CK(d, c.num_pages)] = NONE;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += PLAN) {
        const int s = qp_kv_ld(src + i), d = qp_kv_ld(dst + i);
        if (ok(s) && ok(d)) atomicMin(list + d, i);
    }
    __syncthreads();
    bool range = false;
    for (int i = threadIdx.x; i < n; i += PLAN) {
        const int s = qp_kv_ld(src + i), d = qp_kv_ld(dst + i);
        const bool good = ok(s) && ok(d) && claim[d] == i && (s == d || claim[s] == NONE);
        range |= !good;
        c.a[QP_CK(i, c.num_pages)] = good && s != d ? s : -1;
        c.b[QP_CK(i, c.num_pages)] = d;
    }
    if (range) atomicOr(c.status, QP_DEV_KV_RANGE);
}

// ---------------------------------------------------------------------------- compacting

__global__ void __launch_bounds__(PLAN) kv_compact_plan_kernel(const Cache c, int32_t* live_out)
{
    qp_kv_begin();
    __shared__ int sh[PW + 1], sh_hole[PER * PLAN / 2];
    if (c.num_pages <= PER * PLAN) {                             // every page in a register: the table is read once
        const int lane = threadIdx.x & 31, p0 = (threadIdx.x >> 5) * 32 * PER + lane;
        int refs[PER], n = 0, live, both;
#pragma unroll
        for (int i = 0; i < PER; ++i) refs[i] = p0 + 32 * i < c.num_pages ? __ldcg(c.refs + p0 + 32 * i) : 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) n += __popc(__ballot_sync(0xFFFFFFFFu, refs[i] != 0));
        block_scan(lane == 0 ? n : 0, sh, live);
        unsigned holes[PER], movers[PER];
        n = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {                          // (at most 4096 of either: two sums to a word)
            holes[i] = __ballot_sync(0xFFFFFFFFu, p0 + 32 * i < live && refs[i] == 0);
            movers[i] = __ballot_sync(0xFFFFFFFFu, p0 + 32 * i >= live && refs[i] != 0);
            n += __popc(holes[i]) + (__popc(movers[i]) << 16);
        }
        const int at = __shfl_sync(0xFFFFFFFFu, block_scan(lane == 0 ? n : 0, sh, both), 0);
        const unsigned below = (1u << lane) - 1u;
        int rank = at & 0xFFFF;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (holes[i] >> lane & 1u) sh_hole[QP_CK(rank + __popc(holes[i] & below), PER * PLAN / 2)] = p0 + 32 * i;
            rank += __popc(holes[i]);
        }
        __syncthreads();
        rank = at >> 16;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int p = p0 + 32 * i;
            if (movers[i] >> lane & 1u) {
                const int k = QP_CK(rank + __popc(movers[i] & below), PER * PLAN / 2), to = sh_hole[k];
                c.a[QP_CK(k, c.num_pages)] = p;
                c.b[k] = to;
                c.c[p] = to;
                c.refs[QP_CK(to, c.num_pages)] = refs[i];
                c.refs[p] = 0;
            } else if (p >= live && p < c.num_pages) {
                c.c[p] = -1;
            }
            rank += __popc(movers[i]);
        }
        if (threadIdx.x == 0) {
            c.head[0] = both & 0xFFFF;
            c.head[1] = live;
            if (live_out) *live_out = live;
        }
        return;
    }
    const int live = for_pages(c, 0, c.num_pages, sh, [](int, int refs) { return refs != 0; }, [](int, int) {});
    const int holes = for_pages(c, 0, c.num_pages, sh, [&](int p, int refs) { return p < live && refs == 0; }, [&](int r, int p) { c.b[QP_CK(r, c.num_pages)] = p; });
    // every page at or above `live` has an entry in list c: where it goes, -1 for a free one
    for (int p = live + threadIdx.x; p < c.num_pages; p += PLAN) c.c[p] = -1;
    __syncthreads();
    for_pages(c, 0, c.num_pages, sh, [&](int p, int refs) { return p >= live && refs != 0; }, [&](int r, int p) { c.a[QP_CK(r, c.num_pages)] = p; });
    __syncthreads();
    for (int k = threadIdx.x; k < holes; k += PLAN) {            // as many used pages above as holes below
        const int from = QP_CK(c.a[k], c.num_pages), to = QP_CK(c.b[k], c.num_pages);
        c.c[from] = to;
        c.refs[to] = c.refs[from];
        c.refs[from] = 0;
    }
    if (threadIdx.x == 0) {
        c.head[0] = holes;
        c.head[1] = live;
        if (live_out) *live_out = live;
    }
}

__global__ void __launch_bounds__(MOVE_THREADS) kv_compact_kernel(const Cache c, const Moves m)
{
    qp_kv_begin();
    const int holes = c.head[0], live = c.head[1];
    if (holes == 0) return;
    const int64_t pieces = (int64_t)holes * m.layers * m.chunks;
    for (int64_t t = blockIdx.x; t < pieces; t += gridDim.x) move_piece(m, t);
    const int64_t entries = (int64_t)c.max_seqs * c.max_pages;
    for (int64_t e = (int64_t)blockIdx.x * MOVE_THREADS + threadIdx.x; e < entries; e += (int64_t)gridDim.x * MOVE_THREADS) {
        const int p = c.table[e];
        if (p >= live && p < c.num_pages) c.table[e] = c.c[QP_CK(p, c.num_pages)];
    }
}

int32_t begin(qp_ctx* ctx, const qp_kv_cache_t* c) { return ctx ? qp_kv_check_cache(ctx, c) : QP_ERR_INVALID_ARG; }

int32_t check_list(qp_ctx* ctx, const int32_t* p, int32_t n, int32_t most)
{
    if (n < 0 || n > most) return qp_fail(ctx, QP_ERR_INVALID_ARG, "length of a list");
    if (n > 0 && !p) return qp_fail(ctx, QP_ERR_INVALID_ARG, "null list");
    return (uintptr_t)p & 3u ? qp_fail(ctx, QP_ERR_ALIGNMENT, "list") : QP_OK;
}

}  // namespace

extern "C" int32_t qp_kv_extend(qp_ctx* ctx, const qp_kv_cache_t* h_cache, const qp_kv_batch_t* h_batch, void* stream)
{
    int32_t rc = begin(ctx, h_cache);
    if (!rc) rc = qp_kv_check_batch(ctx, h_batch);
    if (rc) return rc;
    if (h_batch->batch > h_cache->max_seqs) return qp_fail(ctx, QP_ERR_INVALID_ARG, "batch is larger than max_seqs");
    if (h_batch->batch == 0) return QP_OK;
    qp_device_guard guard(ctx->device);
    if (!guard.ok) return qp_fail(ctx, QP_ERR_CUDA, "cannot select device");
    qp_kv_launch(kv_extend_kernel, 1u, PLAN, 0, static_cast<cudaStream_t>(stream), cache_of(ctx, h_cache), h_batch->d_slots, h_batch->d_start,
                                                                        h_batch->d_pos, h_batch->batch, h_batch->tokens, h_batch->max_new);
    ctx->launches += 1;
    return qp_check_launch(ctx, "qp_kv_extend");
}

extern "C" int32_t qp_kv_free(qp_ctx* ctx, const qp_kv_cache_t* h_cache, const int32_t* d_slots, int32_t n, void* stream)
{
    int32_t rc = begin(ctx, h_cache);
    if (!rc) rc = check_list(ctx, d_slots, n, 0x7FFFFFFF);
    if (rc || n == 0) return rc;
    qp_device_guard guard(ctx->device);
    if (!guard.ok) return qp_fail(ctx, QP_ERR_CUDA, "cannot select device");
    const int cap = ctx->sm_count * 16;
    qp_kv_launch(kv_free_kernel, (unsigned)(n < cap ? n : cap), 128, 0, static_cast<cudaStream_t>(stream), cache_of(ctx, h_cache), d_slots, n);
    ctx->launches += 1;
    return qp_check_launch(ctx, "qp_kv_free");
}

extern "C" int32_t qp_kv_fork(qp_ctx* ctx, const qp_kv_cache_t* h_cache, const int32_t* d_src, const int32_t* d_dst, int32_t n, void* stream)
{
    int32_t rc = begin(ctx, h_cache);
    if (!rc) rc = check_list(ctx, d_src, n, h_cache->max_seqs);
    if (!rc) rc = check_list(ctx, d_dst, n, h_cache->max_seqs);
    if (rc || n == 0) return rc;
    qp_device_guard guard(ctx->device);
    if (!guard.ok) return qp_fail(ctx, QP_ERR_CUDA, "cannot select device");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const Cache c = cache_of(ctx, h_cache);
    const Moves m = moves_of(h_cache, c);
    qp_kv_launch(kv_fork_plan_kernel, 1u, PLAN, 0, s, c, d_src, d_dst, n);
    ctx->launches += 1;
    rc = qp_check_launch(ctx, "qp_kv_fork");
    if (rc) return rc;                                           // (lists that nobody has written are not gone by)
    qp_kv_launch(kv_fork_kernel, (unsigned)(move_grid(ctx, n + (int64_t)n * m.layers * m.chunks)), MOVE_THREADS, 0, s, c, m, d_src, d_dst, n);
    ctx->launches += 1;
    return qp_check_launch(ctx, "qp_kv_fork");
}

extern "C" int32_t qp_kv_copy_pages(qp_ctx* ctx, const qp_kv_cache_t* h_cache, const int32_t* d_src, const int32_t* d_dst, int32_t n,
                                    void* stream)
{
    int32_t rc = begin(ctx, h_cache);
    if (!rc) rc = check_list(ctx, d_src, n, h_cache->num_pages);
    if (!rc) rc = check_list(ctx, d_dst, n, h_cache->num_pages);
    if (rc || n == 0) return rc;
    qp_device_guard guard(ctx->device);
    if (!guard.ok) return qp_fail(ctx, QP_ERR_CUDA, "cannot select device");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const Cache c = cache_of(ctx, h_cache);
    const Moves m = moves_of(h_cache, c);
    const bool in_shared = h_cache->num_pages <= SMEM_PAGES;
    qp_kv_launch(kv_copy_plan_kernel, 1u, PLAN, in_shared ? (size_t)h_cache->num_pages * 4 : 0, s, c, d_src, d_dst, n, in_shared);
    ctx->launches += 1;
    rc = qp_check_launch(ctx, "qp_kv_copy_pages");
    if (rc) return rc;
    qp_kv_launch(kv_move_kernel, (unsigned)(move_grid(ctx, (int64_t)n * m.layers * m.chunks)), MOVE_THREADS, 0, s, m, n);
    ctx->launches += 1;
    return qp_check_launch(ctx, "qp_kv_copy_pages");
}

extern "C" int32_t qp_kv_compact(qp_ctx* ctx, const qp_kv_cache_t* h_cache, int32_t* d_live, void* stream)
{
    int32_t rc = begin(ctx, h_cache);
    if (rc) return rc;
    if ((uintptr_t)d_live & 3u) return qp_fail(ctx, QP_ERR_ALIGNMENT, "d_live");
    qp_device_guard guard(ctx->device);
    if (!guard.ok) return qp_fail(ctx, QP_ERR_CUDA, "cannot select device");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const Cache c = cache_of(ctx, h_cache);
    const Moves m = moves_of(h_cache, c);
    qp_kv_launch(kv_compact_plan_kernel, 1u, PLAN, 0, s, c, d_live);
    ctx->launches += 1;
    rc = qp_check_launch(ctx, "qp_kv_compact");
    if (rc) return rc;
    qp_kv_launch(kv_compact_kernel, (unsigned)(move_grid(ctx, (int64_t)h_cache->num_pages * m.layers * m.chunks)), MOVE_THREADS, 0, s, c, m);
    ctx->launches += 1;
    return qp_check_launch(ctx, "qp_kv_compact");
}
