// Rows of the 4-bit cache of keys and values: new tokens quantized into its pages, and rows read back.
//
// A row x of D elements becomes lo = min x, scale = (max x - lo) / 15 and codes rint((x - lo) * 15 / (max x - lo)).
// min and max do not depend on the order they are taken in and every other step is one rounding, so the codes are
// those of the token-wise calls bit for bit.  (A clip from sums, ACIQ, would depend on the order of the sum.)
//
// Eight lanes take the K and the V row of one (token, head): all loads go out before either row's reduction, min and
// max need three shuffles, and the two quotients are one fp64 division with another numerator in every second lane.
// Bound by the bytes: D elements in, D / 2 + 8 bytes out.
#include "qp_kv.cuh"

QP_CK_UNIT

// ---------------------------------------------------------------------------- argument checks

int32_t qp_kv_check_cache(qp_ctx* ctx, const qp_kv_cache_t* c)
{
    if (!c) return qp_fail(ctx, QP_ERR_INVALID_ARG, "null cache");
    if (!c->d_pool || !c->d_table || !c->d_lens || !c->d_refs || !c->d_work) return qp_fail(ctx, QP_ERR_INVALID_ARG, "null pointer in the cache");
    if (!qp_kv_dim_ok(c->head_dim)) return qp_fail(ctx, QP_ERR_INVALID_ARG, "head_dim must be 64, 128 or 256");
    if (c->page_size < QP_KV_SLICE || c->page_size > QP_KV_MAX_PAGE || c->page_size % QP_KV_SLICE)
        return qp_fail(ctx, QP_ERR_INVALID_ARG, "page_size must be a multiple of 16 up to 1024");
    if (c->layers < 1 || c->heads < 1 || c->heads > 65535) return qp_fail(ctx, QP_ERR_INVALID_ARG, "layers or heads");
    if (c->num_pages < 1 || c->num_pages >= (1 << 29)) return qp_fail(ctx, QP_ERR_INVALID_ARG, "num_pages");
    if (c->max_seqs < 1 || c->max_seqs >= (1 << 29) || c->max_pages < 1 || (int64_t)c->max_pages * c->page_size >= (1ll << 31) - 4096 ||
        (int64_t)c->max_pages * c->max_seqs >= (1ll << 40))
        return qp_fail(ctx, QP_ERR_INVALID_ARG, "max_seqs or max_pages (a sequence holds fewer than 2^31 - 4096 tokens)");
    if (((uintptr_t)c->d_pool & 15u) || (c->layers > 1 && (c->layer_stride & 15u))) return qp_fail(ctx, QP_ERR_ALIGNMENT, "pool or layer_stride");
    if (((uintptr_t)c->d_table | (uintptr_t)c->d_lens | (uintptr_t)c->d_refs | (uintptr_t)c->d_work) & 3u)
        return qp_fail(ctx, QP_ERR_ALIGNMENT, "table, lens, refs or work");
    if (c->layers > 1) {
        const uint64_t layer = (uint64_t)c->num_pages * (uint64_t)c->heads * (uint64_t)(c->page_size / QP_KV_SLICE) * qp_kv_slice_bytes(c->head_dim);
        if (c->layer_stride < layer) return qp_fail(ctx, QP_ERR_INVALID_ARG, "layer_stride shorter than a layer");
    }
    return QP_OK;
}

int32_t qp_kv_check_batch(qp_ctx* ctx, const qp_kv_batch_t* b)
{
    if (!b) return qp_fail(ctx, QP_ERR_INVALID_ARG, "null batch");
    if (b->batch < 0 || b->tokens < 0 || b->max_new < 0) return qp_fail(ctx, QP_ERR_INVALID_ARG, "negative size in the batch");
    if (b->batch > 0 && !b->d_pos) return qp_fail(ctx, QP_ERR_INVALID_ARG, "null d_pos");
    if (((uintptr_t)b->d_pos | (uintptr_t)b->d_slots | (uintptr_t)b->d_start) & 3u) return qp_fail(ctx, QP_ERR_ALIGNMENT, "slots, start or pos");
    return QP_OK;
}

int32_t qp_kv_check_layer(qp_ctx* ctx, const qp_kv_cache_t* c, int layer)
{
    return layer < 0 || layer >= c->layers ? qp_fail(ctx, QP_ERR_INVALID_ARG, "layer") : QP_OK;
}

extern "C" uint64_t qp_kv_slice_bytes(int head_dim)
{
    return qp_kv_dim_ok(head_dim) ? (uint64_t)QP_KV_SLICE * (uint64_t)(head_dim + 16) : 0;
}

extern "C" uint64_t qp_kv_work_ints(int32_t num_pages, int32_t max_seqs)
{
    // the page calls' scratch: a head, three lists of pages, three lists of slots
    return num_pages > 0 && max_seqs > 0 ? 64 + 3 * (uint64_t)num_pages + 3 * (uint64_t)max_seqs : 0;
}

namespace {

struct RowArgs {
    qp_kv_rows rows;
    qp_kv_pages pages;
    char* pool;                                  // of the layer
    int heads, slices;
    const void *k, *v;
    int64_t kt, kh, vt, vh;
    unsigned* status;
};

// where the slice and the row of a token and head are: 0 if nowhere (flag: the cache should have it)
template <int D>
__device__ __forceinline__ char* row_place(const RowArgs& a, int token, int head, int& row, bool& flag)
{
    const int b = qp_kv_find(a.rows, token);
    if (b < 0) return nullptr;
    const int first = __ldg(a.rows.pos + b);
    if (first < 0) return nullptr;
    const int64_t p = (int64_t)first + (token - qp_kv_start(a.rows, b));
    const int page = p < (1ll << 31) - 1 ? qp_kv_page(a.pages, qp_kv_slot(a.rows, b), (int)p) : -1;
    if (page < 0) { flag = true; return nullptr; }
    const int in = (int)p % a.pages.page_size;
    row = in % QP_KV_SLICE;
    return a.pool + (((size_t)page * a.heads + head) * a.slices + in / QP_KV_SLICE) * qp_kv_slice<D>::BYTES;
}

template <int E>
__device__ __forceinline__ void load_run(const float* p, bool vec, float (&e)[E])
{
    if (vec) {
#pragma unroll
        for (int i = 0; i < E / 4; ++i) {
            const float4 x = __ldcs(reinterpret_cast<const float4*>(p) + i);
            e[4 * i] = x.x; e[4 * i + 1] = x.y; e[4 * i + 2] = x.z; e[4 * i + 3] = x.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) e[i] = __ldcs(p + i);
    }
}
template <int E>
__device__ __forceinline__ void load_run(const unsigned short* p, bool vec, float (&e)[E])
{
    if (vec) {
#pragma unroll
        for (int i = 0; i < E / 8; ++i) {
            const uint4 x = __ldcs(reinterpret_cast<const uint4*>(p) + i);
            const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                e[8 * i + 2 * h] = __uint_as_float(w[h] << 16);
                e[8 * i + 2 * h + 1] = __uint_as_float(w[h] & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) e[i] = qp_bf16_to_f32(__ldcs(p + i));
    }
}

// this lane's E elements of a row -> the row's quantizer and the lane's codes, 8 to a word
template <int E>
__device__ __forceinline__ void quantize_run(float (&e)[E], int sub, unsigned (&words)[E / 8], float& lo, float& scale)
{
    const float inf = __int_as_float(0x7F800000);
    float mn = inf, mx = -inf;
#pragma unroll
    for (int i = 0; i < E; ++i) { mn = fminf(mn, e[i]); mx = fmaxf(mx, e[i]); }       // (NaN is passed over)
    if (mn == -inf || mx == inf) {                                                    // an infinity: over the finite ones
        mn = inf; mx = -inf;
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (qp_is_finite(e[i])) { mn = fminf(mn, e[i]); mx = fmaxf(mx, e[i]); }
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
        mn = fminf(mn, __shfl_xor_sync(0xFFFFFFFFu, mn, o, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, o, 8));
    }
    if (mn > mx) mn = mx = 0.f;                                                       // nothing finite
    const double width = (double)mx - (double)mn;
    const bool odd = sub & 1;
    const float mine = (float)((odd ? 15.0 : width) / (odd ? width : 15.0));          // even lanes: scale, odd lanes: inv_scale
    const float other = __shfl_xor_sync(0xFFFFFFFFu, mine, 1, 8);
    float inv = odd ? mine : other;
    lo = mn;
    scale = odd ? other : mine;
    if (!(inv < inf)) { scale = 0.f; inv = 0.f; }                                     // constant, or too narrow for inv_scale
    float l = mn, h = mx;
    if (__fsub_rn(mx, mn) == inf) {                                                   // the range passes fp32: halves
        l *= 0.5f; h *= 0.5f; inv *= 2.f;
#pragma unroll
        for (int i = 0; i < E; ++i) e[i] *= 0.5f;
    }
#pragma unroll
    for (int i = 0; i < E / 8; ++i) words[i] = qp_quad<4>(e + 8 * i, l, h, inv) | (qp_quad<4>(e + 8 * i + 4, l, h, inv) << 16);
}

template <int W>
__device__ __forceinline__ void put_words(char* p, const unsigned (&w)[W])
{
    if constexpr (W == 1) *reinterpret_cast<unsigned*>(p) = w[0];
    else if constexpr (W == 2) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
template <int W>
__device__ __forceinline__ void get_words(const char* p, unsigned (&w)[W])
{
    if constexpr (W == 1) w[0] = *reinterpret_cast<const unsigned*>(p);
    else if constexpr (W == 2) { const uint2 x = *reinterpret_cast<const uint2*>(p); w[0] = x.x; w[1] = x.y; }
    else { const uint4 x = *reinterpret_cast<const uint4*>(p); w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w; }
}

constexpr int ROWS = QP_THREADS / 8;

// whole groups of eight lanes take part in every round, so the shuffles are never divergent
template <typename T, int D>
__global__ void __launch_bounds__(QP_THREADS) kv_append_kernel(const RowArgs a, int n, bool vec)
{
    constexpr int E = D / 8;
    using S = qp_kv_slice<D>;
    const int sub = threadIdx.x & 7;
    bool flag = false;
    for (int r0 = blockIdx.x * ROWS; r0 < n; r0 += gridDim.x * ROWS) {
        const int r = r0 + (threadIdx.x >> 3);
        const int token = r / a.heads, head = r - token * a.heads;
        int row = 0;
        char* s = r < n ? row_place<D>(a, token, head, row, flag) : nullptr;
        float k[E], v[E];
        if (s) {
            load_run(static_cast<const T*>(a.k) + token * a.kt + head * a.kh + sub * E, vec, k);
            load_run(static_cast<const T*>(a.v) + token * a.vt + head * a.vh + sub * E, vec, v);
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) k[i] = v[i] = 0.f;
        }
        unsigned w[E / 8];
        float lo, scale;
        quantize_run(k, sub, w, lo, scale);
        if (s) {
            put_words(s + row * S::ROW + sub * (E / 2), w);
            if (sub == 0) *reinterpret_cast<float2*>(s + S::KQ + row * 8) = make_float2(lo, scale);
        }
        quantize_run(v, sub, w, lo, scale);
        if (s) {
            put_words(s + S::V + row * S::ROW + sub * (E / 2), w);
            if (sub == 0) *reinterpret_cast<float2*>(s + S::VQ + row * 8) = make_float2(lo, scale);
        }
    }
    if (flag) atomicOr(a.status, QP_DEV_KV_RANGE);
}

template <int E>
__device__ __forceinline__ void store_run(float* p, bool vec, const float (&e)[E])
{
    if (vec) {
#pragma unroll
        for (int i = 0; i < E / 4; ++i) __stcs(reinterpret_cast<float4*>(p) + i, make_float4(e[4 * i], e[4 * i + 1], e[4 * i + 2], e[4 * i + 3]));
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) p[i] = e[i];
    }
}
template <int E>
__device__ __forceinline__ void store_run(unsigned short* p, bool vec, const float (&e)[E])
{
    unsigned short h[E];
#pragma unroll
    for (int i = 0; i < E; ++i) h[i] = qp_f32_to_bf16(e[i]);
    if (vec) {
#pragma unroll
        for (int i = 0; i < E / 8; ++i) {
            uint4 x;
            x.x = h[8 * i] | ((unsigned)h[8 * i + 1] << 16);
            x.y = h[8 * i + 2] | ((unsigned)h[8 * i + 3] << 16);
            x.z = h[8 * i + 4] | ((unsigned)h[8 * i + 5] << 16);
            x.w = h[8 * i + 6] | ((unsigned)h[8 * i + 7] << 16);
            __stcs(reinterpret_cast<uint4*>(p) + i, x);
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) p[i] = h[i];
    }
}

template <int E>
__device__ __forceinline__ void values_of(const unsigned (&w)[E / 8], float2 q, float (&e)[E])
{
#pragma unroll
    for (int i = 0; i < E; ++i) e[i] = fmaf((float)((w[i / 8] >> (4 * (i & 7))) & 15u), q.y, q.x);
}

template <typename T, int D>
__global__ void __launch_bounds__(QP_THREADS) kv_gather_kernel(const RowArgs a, int n, bool vec)
{
    constexpr int E = D / 8;
    using S = qp_kv_slice<D>;
    const int sub = threadIdx.x & 7;
    bool flag = false;
    for (int r = blockIdx.x * ROWS + (threadIdx.x >> 3); r < n; r += gridDim.x * ROWS) {
        const int token = r / a.heads, head = r - token * a.heads;
        int row = 0;
        const char* s = row_place<D>(a, token, head, row, flag);
        if (!s) continue;
        unsigned kw[E / 8], vw[E / 8];
        get_words(s + row * S::ROW + sub * (E / 2), kw);
        get_words(s + S::V + row * S::ROW + sub * (E / 2), vw);
        const float2 kq = *reinterpret_cast<const float2*>(s + S::KQ + row * 8), vq = *reinterpret_cast<const float2*>(s + S::VQ + row * 8);
        float e[E];
        if (a.k) {
            values_of(kw, kq, e);
            store_run(const_cast<T*>(static_cast<const T*>(a.k)) + token * a.kt + head * a.kh + sub * E, vec, e);
        }
        if (a.v) {
            values_of(vw, vq, e);
            store_run(const_cast<T*>(static_cast<const T*>(a.v)) + token * a.vt + head * a.vh + sub * E, vec, e);
        }
    }
    if (flag) atomicOr(a.status, QP_DEV_KV_RANGE);
}

typedef void (*RowKernel)(const RowArgs, int, bool);

template <template <typename, int> class K>
RowKernel pick(int dtype, int d);

template <typename T, int D> struct AppendOf { static RowKernel get() { return kv_append_kernel<T, D>; } };
template <typename T, int D> struct GatherOf { static RowKernel get() { return kv_gather_kernel<T, D>; } };

template <template <typename, int> class K>
RowKernel pick(int dtype, int d)
{
    if (dtype == QP_F32) return d == 64 ? K<float, 64>::get() : d == 128 ? K<float, 128>::get() : K<float, 256>::get();
    return d == 64 ? K<unsigned short, 64>::get() : d == 128 ? K<unsigned short, 128>::get() : K<unsigned short, 256>::get();
}

int32_t launch_rows(qp_ctx* ctx, bool append, const qp_kv_cache_t* c, const qp_kv_batch_t* b, int layer, const void* k, const void* v,
                    int dtype, int64_t kt, int64_t kh, int64_t vt, int64_t vh, void* stream)
{
    if (!ctx) return QP_ERR_INVALID_ARG;
    int32_t rc = qp_kv_check_cache(ctx, c);
    if (!rc) rc = qp_kv_check_batch(ctx, b);
    if (!rc) rc = qp_kv_check_layer(ctx, c, layer);
    if (rc) return rc;
    if (dtype != QP_F32 && dtype != QP_BF16) return qp_fail(ctx, QP_ERR_UNSUPPORTED_DTYPE, "dtype must be QP_F32 or QP_BF16");
    if ((int64_t)b->tokens * c->heads >= (1ll << 31) - (1 << 26)) return qp_fail(ctx, QP_ERR_INVALID_ARG, "tokens * heads must be below 2^31 - 2^26");
    if (b->tokens == 0 || b->batch == 0) return QP_OK;
    if (append ? !k || !v : !k && !v) return qp_fail(ctx, QP_ERR_INVALID_ARG, "null d_k or d_v");
    const int64_t es = dtype == QP_F32 ? 4 : 2;
    if (((uintptr_t)k | (uintptr_t)v) & (uintptr_t)(es - 1)) return qp_fail(ctx, QP_ERR_ALIGNMENT, "d_k or d_v");
    // 16-byte accesses where every row allows them
    const bool vec = ((((uintptr_t)k | (uintptr_t)v) & 15u) | (uintptr_t)(((kt | kh | vt | vh) * es) & 15)) == 0;
    qp_device_guard guard(ctx->device);
    if (!guard.ok) return qp_fail(ctx, QP_ERR_CUDA, "cannot select device");
    RowArgs a;
    a.rows = qp_kv_rows_of(b);
    a.pages = qp_kv_pages_of(c);
    a.pool = static_cast<char*>(c->d_pool) + (size_t)layer * c->layer_stride;
    a.heads = c->heads;
    a.slices = c->page_size / QP_KV_SLICE;
    a.k = k; a.v = v;
    a.kt = kt; a.kh = kh; a.vt = vt; a.vh = vh;
    a.status = ctx->d_status;
    const int n = b->tokens * c->heads;
    const uint64_t want = ((uint64_t)n + ROWS - 1) / ROWS, cap = (uint64_t)ctx->sm_count * 64;
    const RowKernel f = append ? pick<AppendOf>(dtype, c->head_dim) : pick<GatherOf>(dtype, c->head_dim);
    f<<<(unsigned)(want < cap ? want : cap), QP_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(a, n, vec);
    ctx->launches += 1;
    return qp_check_launch(ctx, append ? "qp_kv_append" : "qp_kv_gather");
}

}  // namespace

extern "C" int32_t qp_kv_append(qp_ctx* ctx, const qp_kv_cache_t* h_cache, const qp_kv_batch_t* h_batch, int layer, const void* d_k,
                                const void* d_v, int dtype, int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                                int64_t v_head_stride, void* stream)
{
    return launch_rows(ctx, true, h_cache, h_batch, layer, d_k, d_v, dtype, k_token_stride, k_head_stride, v_token_stride, v_head_stride, stream);
}

extern "C" int32_t qp_kv_gather(qp_ctx* ctx, const qp_kv_cache_t* h_cache, const qp_kv_batch_t* h_batch, int layer, void* d_k, void* d_v,
                                int dtype, int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride,
                                void* stream)
{
    return launch_rows(ctx, false, h_cache, h_batch, layer, d_k, d_v, dtype, k_token_stride, k_head_stride, v_token_stride, v_head_stride, stream);
}
