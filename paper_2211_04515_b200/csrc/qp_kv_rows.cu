// Rows of the 4-bit cache of keys and values: new tokens quantized into its pages, and rows read back.
//
// A row x of D elements becomes lo = min x, scale = (max x - lo) / 15 and codes rint((x - lo) * 15 / (max x - lo)).
// min and max do not depend on the order they are taken in and every other step is one rounding, so the codes are
// those of the token-wise calls bit for bit.  (A clip from sums, ACIQ, would depend on the order of the sum.)
//
// Eight lanes take the K and the V row of one (token, head): the loads of both go out before anything else, min and max need
// three shuffles, and the four quotients of the two rows are one fp64 division, another one in every lane.  Rows without a NaN
// or an infinity (found by one fused operation to two elements) need no clamp.  Bound by the bytes, D elements in, D / 2 + 8
// bytes out, and by the instructions, about 12 to an element.  What keeps such a kernel from them is the chain of dependent loads batch -> position -> page -> row
// (with the divisions between them 3 us, in every warp: 21 us for 8246 tokens of 8 heads), so one warp looks up a block's
// tokens, a lane to a token, while the others' first rows are on their way.
// Measured for 8246 tokens of 8 heads of 128 in bf16: append 20 us by itself (34 MB in, 10 out; 49 % of the issue slots), gather 13 (48 %), both in
// a stream 30.
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

constexpr int TOKENS = 32;                       // of a block, at most
struct Places { int64_t at[TOKENS]; int row[TOKENS]; };

// Lane i < n: where token first + i's slice of head 0 begins and the row in it; -1 if nowhere (flag: the cache should have it).  The
// first token's sequence by a 32-way search, the others' by steps from there.
template <int D>
__device__ __forceinline__ void look_up(const RowArgs& a, int first, int n, Places& to, bool& flag)
{
    const int lane = threadIdx.x & 31, token = first + lane;
    const qp_kv_rows& r = a.rows;
    int lo = first, hi = r.batch;
    if (r.start) {
        lo = 0;                                                  // the last b with start[b] <= first, or 0
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) >> 5, at = lo + lane * step;
            const unsigned below = __ballot_sync(0xFFFFFFFFu, at < hi && (at == lo || qp_kv_start(r, at) <= first));
            const int last = 31 - __clz(below);
            hi = min(hi, lo + (last + 1) * step);
            lo += last * step;
        }
    }
    int64_t place = -1;
    int row = 0;
    if (lane < n) {
        int b = r.start ? lo : token, from = token;
        if (r.start) {
            from = qp_kv_start(r, b);
            for (int next; b < r.batch && (next = qp_kv_start(r, b + 1)) <= token; from = next) ++b;
        }
        const int pos = b < r.batch && from <= token ? qp_kv_ld(r.pos + b) : -1;
        if (pos >= 0) {
            const int64_t p = (int64_t)pos + (token - from);
            const int page = p < (1ll << 31) - 1 ? qp_kv_page(a.pages, qp_kv_slot(r, b), (int)p) : -1;
            if (page < 0) {
                flag = true;
            } else {
                const int in = (int)p % a.pages.page_size;
                row = in % QP_KV_SLICE;
                place = ((int64_t)page * a.heads * a.slices + in / QP_KV_SLICE) * qp_kv_slice<D>::BYTES;
            }
        }
    }
    to.at[lane] = place;
    to.row[lane] = row;
}

// A lane's elements of a row: pieces sub, sub + 8, ... of 16 bytes, so that the eight lanes of a row meet whole sectors.
template <typename T> constexpr int PIECE = 16 / sizeof(T);
template <typename T, int E>
__device__ __forceinline__ void load_run(const T* row, int sub, bool vec, float (&e)[E])
{
    constexpr int N = PIECE<T>;
#pragma unroll
    for (int i = 0; i < E / N; ++i) {
        const T* p = row + (sub + 8 * i) * N;
        if constexpr (sizeof(T) == 4) {
            if (vec) {
                const float4 x = __ldcs(reinterpret_cast<const float4*>(p));
                e[4 * i] = x.x; e[4 * i + 1] = x.y; e[4 * i + 2] = x.z; e[4 * i + 3] = x.w;
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) e[N * i + k] = __ldcs(p + k);
            }
        } else {
            if (vec) {
                const uint4 x = __ldcs(reinterpret_cast<const uint4*>(p));
                const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    e[8 * i + 2 * h] = __uint_as_float(w[h] << 16);
                    e[8 * i + 2 * h + 1] = __uint_as_float(w[h] & 0xFFFF0000u);
                }
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) e[N * i + k] = qp_bf16_to_f32(__ldcs(p + k));
            }
        }
    }
}

// Ends of a row from the E elements that each of eight lanes has; whether all are finite.
template <int E>
__device__ __forceinline__ bool ends_of(const float (&e)[E], float& mn, float& mx)
{
    const float inf = __int_as_float(0x7F800000);
    qp_f2 zero = qp_pack2(0.f, 0.f);                             // stays zero unless there is a NaN or an infinity
#pragma unroll
    for (int i = 0; i < E; i += 2) zero = qp_fma2(qp_pack2(e[i], e[i + 1]), qp_pack2(0.f, 0.f), zero);
    float z0, z1;
    qp_unpack2(zero, z0, z1);
    const bool fine = z0 == 0.f && z1 == 0.f;
    mn = e[0];
    mx = e[0];
    if (fine) {
#pragma unroll
        for (int i = 1; i + 1 < E; i += 2) { mn = qp_min3(mn, e[i], e[i + 1]); mx = qp_max3(mx, e[i], e[i + 1]); }
        mn = fminf(mn, e[E - 1]);
        mx = fmaxf(mx, e[E - 1]);
    } else {
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
    return fine;
}

// Quantizers of the two rows with the ends given: scale and inv_scale
__device__ __forceinline__ void quotients(float k_mn, float k_mx, float v_mn, float v_mx, int sub, float (&scale)[2], float (&inv)[2])
{
    const double width = sub & 2 ? (double)v_mx - (double)v_mn : (double)k_mx - (double)k_mn;
    const bool odd = sub & 1;
    const float mine = (float)((odd ? 15.0 : width) / (odd ? width : 15.0));          // lanes 0, 2: scales, lanes 1, 3: inv_scales
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        scale[h] = __shfl_sync(0xFFFFFFFFu, mine, 2 * h, 8);
        inv[h] = __shfl_sync(0xFFFFFFFFu, mine, 2 * h + 1, 8);
        if (!(inv[h] < __int_as_float(0x7F800000))) { scale[h] = 0.f; inv[h] = 0.f; }  // constant, or too narrow for inv_scale
    }
}

// the lane's codes, a quad of four to 16 bits
template <int E>
__device__ __forceinline__ void codes_of(float (&e)[E], bool fine, float mn, float mx, float inv, unsigned (&quads)[E / 4])
{
    float l = mn, h = mx;
    const bool wide = __fsub_rn(mx, mn) == __int_as_float(0x7F800000);                // the range passes fp32: halves
    if (wide) {
        l *= 0.5f; h *= 0.5f; inv *= 2.f;
#pragma unroll
        for (int i = 0; i < E; ++i) e[i] *= 0.5f;
    }
    if (__all_sync(0xFFFFFFFFu, fine)) {
        // qp_quad without its clamp: every element lies between the ends
        const qp_f2 nl = qp_pack2(-l, -l), inv2 = qp_pack2(inv, inv), magic = qp_pack2(QP_MAGIC, QP_MAGIC);
        constexpr unsigned offs = QP_MAGIC_BITS * 0x1111u;
#pragma unroll
        for (int i = 0; i < E / 4; ++i) {
            float a, b, c, d;
            qp_unpack2(qp_add2(qp_mul2(qp_add2(qp_pack2(e[4 * i], e[4 * i + 1]), nl), inv2), magic), a, b);
            qp_unpack2(qp_add2(qp_mul2(qp_add2(qp_pack2(e[4 * i + 2], e[4 * i + 3]), nl), inv2), magic), c, d);
            // (the sum of four shifted words, less the sum of the shifted constants)
            quads[i] = (__float_as_uint(a) + (__float_as_uint(b) << 4)) + ((__float_as_uint(c) << 8) + (__float_as_uint(d) << 12)) - offs;
        }
    } else {
#pragma unroll
        for (int i = 0; i < E / 4; ++i) quads[i] = qp_quad<4>(e + 4 * i, l, h, inv);
    }
}

// a lane's codes of a row, to and from the cache: pieces as load_run has them
template <typename T, int Q>
__device__ __forceinline__ void put_codes(char* row, int sub, const unsigned (&q)[Q])
{
#pragma unroll
    for (int i = 0; i < Q; i += PIECE<T> / 4) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<unsigned short*>(row + (sub + 8 * i) * 2) = (unsigned short)q[i];
        else *reinterpret_cast<unsigned*>(row + (sub + 4 * i) * 4) = q[i] | (q[i + 1] << 16);
    }
}
template <typename T, int Q>
__device__ __forceinline__ void get_codes(const char* row, int sub, unsigned (&q)[Q])
{
#pragma unroll
    for (int i = 0; i < Q; i += PIECE<T> / 4) {
        if constexpr (sizeof(T) == 4) {
            q[i] = *reinterpret_cast<const unsigned short*>(row + (sub + 8 * i) * 2);
        } else {
            const unsigned w = *reinterpret_cast<const unsigned*>(row + (sub + 4 * i) * 4);
            q[i] = w & 0xFFFFu;
            q[i + 1] = w >> 16;
        }
    }
}

constexpr int GROUPS = QP_THREADS / 8;

// a block's tokens: first = blockIdx.x * per_block, at most per_block of them
template <typename T, int D>
__global__ void __launch_bounds__(QP_THREADS) kv_append_kernel(const RowArgs a, int per_block, bool vec)
{
    constexpr int E = D / 8;
    using S = qp_kv_slice<D>;
    qp_kv_begin();
    __shared__ Places places;
    const int sub = threadIdx.x & 7, group = threadIdx.x >> 3;
    const int first = blockIdx.x * per_block, n = min(per_block, a.rows.tokens - first), pairs = n * a.heads;
    bool flag = false;
    for (int i0 = 0; i0 < pairs; i0 += GROUPS) {                 // whole groups of eight lanes take part in every round
        const int i = i0 + group, in = i / a.heads, head = i - in * a.heads;
        const int64_t token = first + in;
        float k[E], v[E];
        if (i < pairs) {
            load_run(static_cast<const T*>(a.k) + token * a.kt + head * a.kh, sub, vec, k);
            load_run(static_cast<const T*>(a.v) + token * a.vt + head * a.vh, sub, vec, v);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) k[e] = v[e] = 0.f;
        }
        if (i0 == 0) {
            if (threadIdx.x < 32) look_up<D>(a, first, n, places, flag);
            __syncthreads();
        }
        const int64_t place = i < pairs ? places.at[QP_CK(in, TOKENS)] : -1;
        const int row = i < pairs ? places.row[QP_CK(in, TOKENS)] : 0;
        char* s = a.pool + place + (int64_t)head * a.slices * S::BYTES;
        float k_mn, k_mx, v_mn, v_mx, scale[2], inv[2];
        const bool k_fine = ends_of(k, k_mn, k_mx), v_fine = ends_of(v, v_mn, v_mx);
        quotients(k_mn, k_mx, v_mn, v_mx, sub, scale, inv);
        unsigned kw[E / 4], vw[E / 4];
        codes_of(k, k_fine, k_mn, k_mx, inv[0], kw);
        codes_of(v, v_fine, v_mn, v_mx, inv[1], vw);
        if (place >= 0) {
            put_codes<T>(s + row * S::ROW, sub, kw);
            put_codes<T>(s + S::V + row * S::ROW, sub, vw);
            if (sub < 2) *reinterpret_cast<float2*>(s + (sub ? S::VQ : S::KQ) + row * 8) = make_float2(sub ? v_mn : k_mn, sub ? scale[1] : scale[0]);
        }
    }
    if (flag) atomicOr(a.status, QP_DEV_KV_RANGE);
}

template <typename T, int E>
__device__ __forceinline__ void store_run(T* row, int sub, bool vec, const float (&e)[E])
{
    constexpr int N = PIECE<T>;
#pragma unroll
    for (int i = 0; i < E / N; ++i) {
        T* p = row + (sub + 8 * i) * N;
        if constexpr (sizeof(T) == 4) {
            if (vec) {
                __stcs(reinterpret_cast<float4*>(p), make_float4(e[4 * i], e[4 * i + 1], e[4 * i + 2], e[4 * i + 3]));
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) p[k] = e[N * i + k];
            }
        } else {
            unsigned h[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(h[k]) : "f"(e[8 * i + 2 * k + 1]), "f"(e[8 * i + 2 * k]));
            if (vec) {
                __stcs(reinterpret_cast<uint4*>(p), make_uint4(h[0], h[1], h[2], h[3]));
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) p[k] = (unsigned short)(h[k / 2] >> (16 * (k & 1)));
            }
        }
    }
}

// A code under 128's exponent (at bits 16..19) or 2048's (at bits 12..15) is that number + code; less the number, exactly the code.
template <int E>
__device__ __forceinline__ void values_of(const unsigned (&q)[E / 4], float2 quant, float (&e)[E])
{
    const qp_f2 less = qp_pack2(-2048.f, -128.f), scale = qp_pack2(quant.y, quant.y), lo = qp_pack2(quant.x, quant.x);
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
        const unsigned a = q[i] << 12, b = q[i] << 4;            // codes 0, 1 and 2, 3 at bits 12..19
        qp_unpack2(qp_fma2(qp_add2(qp_pack2(__uint_as_float((a & 0xF000u) | 0x45000000u), __uint_as_float((a & 0xF0000u) | 0x43000000u)), less), scale, lo),
                   e[4 * i], e[4 * i + 1]);
        qp_unpack2(qp_fma2(qp_add2(qp_pack2(__uint_as_float((b & 0xF000u) | 0x45000000u), __uint_as_float((b & 0xF0000u) | 0x43000000u)), less), scale, lo),
                   e[4 * i + 2], e[4 * i + 3]);
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(QP_THREADS) kv_gather_kernel(const RowArgs a, int per_block, bool vec)
{
    constexpr int E = D / 8;
    using S = qp_kv_slice<D>;
    qp_kv_begin();
    __shared__ Places places;
    const int sub = threadIdx.x & 7, group = threadIdx.x >> 3;
    const int first = blockIdx.x * per_block, n = min(per_block, a.rows.tokens - first), pairs = n * a.heads;
    bool flag = false;
    if (threadIdx.x < 32) look_up<D>(a, first, n, places, flag);
    __syncthreads();
#pragma unroll 2
    for (int i = group; i < pairs; i += GROUPS) {
        const int in = i / a.heads, head = i - in * a.heads, row = places.row[QP_CK(in, TOKENS)];
        const int64_t token = first + in, place = places.at[QP_CK(in, TOKENS)];
        if (place < 0) continue;
        const char* s = a.pool + place + (int64_t)head * a.slices * S::BYTES;
        unsigned kw[E / 4], vw[E / 4];
        get_codes<T>(s + row * S::ROW, sub, kw);
        get_codes<T>(s + S::V + row * S::ROW, sub, vw);
        const float2 kq = *reinterpret_cast<const float2*>(s + S::KQ + row * 8), vq = *reinterpret_cast<const float2*>(s + S::VQ + row * 8);
        float e[E];
        if (a.k) {
            values_of(kw, kq, e);
            store_run(const_cast<T*>(static_cast<const T*>(a.k)) + token * a.kt + head * a.kh, sub, vec, e);
        }
        if (a.v) {
            values_of(vw, vq, e);
            store_run(const_cast<T*>(static_cast<const T*>(a.v)) + token * a.vt + head * a.vh, sub, vec, e);
        }
    }
    if (flag) atomicOr(a.status, QP_DEV_KV_RANGE);
}

typedef void (*RowKernel)(const RowArgs, int, bool);
template <typename T, int D> RowKernel kernel_of(bool append) { return append ? kv_append_kernel<T, D> : kv_gather_kernel<T, D>; }
template <typename T>
RowKernel pick(bool append, int d) { return d == 64 ? kernel_of<T, 64>(append) : d == 128 ? kernel_of<T, 128>(append) : kernel_of<T, 256>(append); }

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
    // Four rounds to a block at most (128 pairs of token and head; with more heads than that a token to a block, whose rounds are heads / 32), and
    // enough blocks for two on every SM where there are the tokens
    int per_block = 4 * GROUPS / c->heads, fill = (b->tokens + 2 * ctx->sm_count - 1) / (2 * ctx->sm_count);
    if (per_block > fill) per_block = fill;
    per_block = per_block < 1 ? 1 : per_block > TOKENS ? TOKENS : per_block;
    const RowKernel f = dtype == QP_F32 ? pick<float>(append, c->head_dim) : pick<unsigned short>(append, c->head_dim);
    qp_kv_launch(f, (unsigned)((b->tokens + per_block - 1) / per_block), QP_THREADS, 0, static_cast<cudaStream_t>(stream), a, per_block, vec);
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
