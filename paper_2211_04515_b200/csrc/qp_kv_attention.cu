// Attention over the 4-bit cache for few queries to a cached head (decoding, drafted tokens).
//
// With k_u = lo_u + scale_u * c_u and v_u = lo'_u + scale'_u * c'_u (c: 4-bit codes)
//     q . k_u        = scale_u * (q . c_u) + lo_u * sum(q)
//     sum_u p_u v_u  = sum_u (p_u scale'_u) c'_u + sum_u p_u lo'_u
// so the codes go into the matrix instructions as they are, and a row's quantizer costs a few operations per (token, query), not
// per element.  A nibble masked in place in a 16-bit lane is an fp16 subnormal, code * 2^-24 (or 2^-20, one nibble up): exact, no
// conversion, no offset.  One word of 8 codes becomes four operand registers with four ANDs and a shift.
//
// Bound by the cache's bytes: (D / 2 + 8) * 2 per (token, head).  What keeps an SM from that is issue slots: at 6.5 TB/s an SM
// has about 23 bytes a cycle to digest, 46 codes.  So the tokens lie along the M side (16) and the queries along the N side
// (8) of m16n8k16: the codes are the A operand in both products, no row is wasted where 8 queries share a head, and the accumulators
// of out^T need half the registers.  (Tensor memory and tcgen05 would need the codes written out as 16-bit operands in shared memory first,
// four times the bytes, for 8 queries.)  The probabilities turn from accumulator to operand by movmatrix.
//
//   - A warp takes slices of 16 tokens by itself: a ring of its own in shared memory, filled with 16-byte asynchronous
//     copies (a slice is contiguous), no barrier with other warps until its part of the sequence ends.
//   - Softmax with a reference instead of the running maximum: p = 2^(s - m) where m is only raised, by a vote, once a score
//     passes it by 8; the same for the scale of V, so that p * scale' fits fp16.
//   - The work of the whole batch, in units of 64 tokens of one (sequence, head, tile of queries), is cut into equal runs, one
//     for each resident block, whatever the lengths.  Where a cut falls inside an item, its blocks leave partial results,
//     and the last to finish (a counter per item; nobody waits) adds them up in the blocks' order, so the result does not depend on timing.
//   - fp32 queries (and probabilities) are split into two fp16 numbers, 22 bits together, with a product for each.  Two
//     things that 16 bits do not show cost bits there: the matrix unit lines its products up by the operands' exponents, so that a
//     subnormal's leading zeros are lost from the sum (1e-5 of the result), and it cuts sums off instead of rounding them.  So the codes
//     are made normal numbers there, and less 8 while at it (lo is then the value of code 8: smaller sums), and each slice's
//     sums start at zero and are added to the running ones by ordinary additions.
#include "qp_kv.cuh"
#include "qp_kv_attention.cuh"

QP_CK_UNIT

namespace {

constexpr int WARPS = 4, THREADS = WARPS * 32;
constexpr float M_NONE = -3.0e38f;               // reference before any score
constexpr float M_SLACK = 8.f;                   // a score may pass the reference by this (log2)
constexpr float V_SLACK = 64.f;                  // and a scale of V its norm by this: p * scale' <= 2^14 in fp16

template <int D, int NT, bool SPLIT> struct Cfg {
    static constexpr int ROWS = 8 * NT;
    static constexpr int SB = qp_kv_slice<D>::BYTES;
    static constexpr int STAGES = D == 256 ? 4 : D == 128 ? 5 : 6;
    static constexpr int RING = WARPS * STAGES * SB;
    static constexpr int MERGE = WARPS * ROWS * (D + 2) * 4;
    static constexpr int SMEM = RING > MERGE ? RING : MERGE;
    static constexpr int PER_SM = D == 256 ? 3 : NT == 2 || SPLIT ? 3 : 4;
};

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ void mma(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ unsigned half2_of(float lo, float hi)
{
    unsigned r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float half_lo(unsigned h)
{
    float r;
    asm("{.reg .b16 a, b; mov.b32 {a, b}, %1; cvt.f32.f16 %0, a;}" : "=f"(r) : "r"(h));
    return r;
}
__device__ __forceinline__ float half_hi(unsigned h)
{
    float r;
    asm("{.reg .b16 a, b; mov.b32 {a, b}, %1; cvt.f32.f16 %0, b;}" : "=f"(r) : "r"(h));
    return r;
}
// the codes under a mask as fp16: code * 2^-24 (16 times that under M1), or (NORMAL) code - 8 (16 times that): 1024 + code is
// code in the low bits of 1024's pattern, and the subtraction is exact
template <bool NORMAL>
__device__ __forceinline__ unsigned codes(unsigned x, unsigned mask)
{
    if constexpr (!NORMAL) return x & mask;
    x = (x & mask) | 0x64006400u;
    asm("sub.f16x2 %0, %0, %1;" : "+r"(x) : "r"(mask == 0x000F000Fu ? 0x64086408u : 0x64806480u));
    return x;
}
__device__ __forceinline__ unsigned transpose8(unsigned x)       // 8x8 16-bit matrix over the warp
{
    unsigned r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ void copy16(char* dst, const char* src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((unsigned)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int W>
__device__ __forceinline__ void lds_words(const char* p, unsigned (&w)[W])
{
    if constexpr (W == 1) w[0] = *reinterpret_cast<const unsigned*>(p);
    else if constexpr (W == 2) { const uint2 x = *reinterpret_cast<const uint2*>(p); w[0] = x.x; w[1] = x.y; }
    else {
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const uint4 x = *reinterpret_cast<const uint4*>(p + 16 * i);
            w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
        }
    }
}

// What the batch asks for: sequence b's part.
struct Seq {
    int pos, n, row0;                            // first position, tokens, row of the first
    int s0, s1;                                  // slices [s0, s1) hold the keys that some query sees
    int units, tiles;                            // units of 64 tokens, query tiles
    int64_t work;                                // units in all
};

template <int ROWS>
__device__ __forceinline__ Seq seq_of(const qp_kv_attn_args& a, int b)
{
    Seq q;
    q.row0 = qp_kv_start(a.rows, b);
    const int row1 = a.rows.start ? qp_kv_start(a.rows, b + 1) : (b < a.rows.tokens ? b + 1 : b);
    q.n = row1 - q.row0;
    if (q.n > a.max_new) q.n = a.max_new;
    q.pos = __ldg(a.rows.pos + b);
    if (q.n <= 0 || q.pos < 0) { q.work = 0; q.units = q.tiles = 0; q.s0 = q.s1 = 0; return q; }
    const int64_t most = (int64_t)a.pages.max_pages * a.pages.page_size;
    int64_t end = (int64_t)q.pos + q.n;
    if (end > most) end = most;
    int lo = a.window > 0 && q.pos >= a.window ? q.pos - a.window + 1 : 0;
    if (lo > end) lo = (int)end;
    q.s0 = lo / QP_KV_SLICE;
    q.s1 = (int)((end + QP_KV_SLICE - 1) / QP_KV_SLICE);
    q.units = (q.s1 - q.s0 + WARPS - 1) / WARPS;
    if (q.units < 1) q.units = 1;                                // an empty one still writes its rows
    q.tiles = (int)(((int64_t)q.n * a.group + ROWS - 1) / ROWS);
    q.work = (int64_t)q.units * q.tiles * a.heads;
    return q;
}

// Block-wide: total work, or the sequence that unit `find` falls in and the work in front of it.
template <int ROWS>
__device__ __forceinline__ int64_t batch_work(const qp_kv_attn_args& a, int64_t find, int& at_b, int64_t& at_base, int64_t* sh)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t carry = 0;
    for (int b0 = 0; b0 < a.rows.batch; b0 += THREADS) {
        const int b = b0 + threadIdx.x;
        const int64_t w = b < a.rows.batch ? seq_of<ROWS>(a, b).work : 0;
        int64_t x = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xFFFFFFFFu, x, o);
            if (lane >= o) x += y;
        }
        __syncthreads();
        if (lane == 31) sh[warp] = x;
        __syncthreads();
        int64_t total = 0, before = carry;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) {
            if (i == warp) before += total;
            total += sh[i];
        }
        before += x - w;
        if (find >= before && find < before + w) { sh[WARPS] = b; sh[WARPS + 1] = before; }
        carry += total;
        if (find >= 0 && find < carry) break;                    // uniform
    }
    __syncthreads();
    if (find >= 0) { at_b = (int)sh[WARPS]; at_base = sh[WARPS + 1]; }
    return carry;
}

// this lane's D / 4 elements of a query row
template <int N>
__device__ __forceinline__ void load_q(const unsigned short* p, bool vec, float (&e)[N])
{
    if (vec) {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            const uint4 x = __ldg(reinterpret_cast<const uint4*>(p) + i);
            const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int h = 0; h < 4; ++h) { e[8 * i + 2 * h] = __uint_as_float(w[h] << 16); e[8 * i + 2 * h + 1] = __uint_as_float(w[h] & 0xFFFF0000u); }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = qp_bf16_to_f32(__ldg(p + i));
    }
}
template <int N>
__device__ __forceinline__ void load_q(const float* p, bool vec, float (&e)[N])
{
    if (vec) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float4 x = __ldg(reinterpret_cast<const float4*>(p) + i);
            e[4 * i] = x.x; e[4 * i + 1] = x.y; e[4 * i + 2] = x.z; e[4 * i + 3] = x.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = __ldg(p + i);
    }
}
__device__ __forceinline__ void put_out(float* p, float v) { *p = v; }
__device__ __forceinline__ void put_out(unsigned short* p, float v) { *p = qp_f32_to_bf16(v); }

// out row and lse of query row r of a tile's sequence
template <typename T, int D>
__device__ __forceinline__ void put_row(const qp_kv_attn_args& a, const Seq& q, int head, int r, int d, float o, float m, float l)
{
    const int token = q.row0 + r / a.group, h = head * a.group + r % a.group;
    put_out(static_cast<T*>(a.out) + (int64_t)token * a.ot + (int64_t)h * a.oh + d, l == 0.f ? 0.f : o / l);
    if (a.lse && d == 0)
        a.lse[(int64_t)token * a.q_heads + h] = l == 0.f ? -__int_as_float(0x7F800000) : (m + log2f(l)) * 0.6931471805599453f;
}

template <int D, int NT, bool SPLIT>
__global__ void __launch_bounds__(THREADS, Cfg<D, NT, SPLIT>::PER_SM) kv_attn_kernel(const qp_kv_attn_args a)
{
    using C = Cfg<D, NT, SPLIT>;
    using S = qp_kv_slice<D>;
    using T = typename std::conditional<SPLIT, float, unsigned short>::type;
    constexpr int ROWS = C::ROWS, SB = C::SB, STAGES = C::STAGES;
    constexpr int KW = D / 32, VW = D / 64;                      // words of 8 codes a lane holds of a K row, of a V row
    constexpr int QB = 4 * KW;                                   // operand registers of a query tile
    constexpr unsigned M0 = 0x000F000Fu, M1 = 0x00F000F0u;
    extern __shared__ __align__(16) char smem[];
    __shared__ int64_t sh_work[WARPS + 2];
    __shared__ int sh_ok[WARPS][STAGES];
    __shared__ int sh_last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = lane >> 2, j = lane & 3;

    int b = 0;
    int64_t base = 0;
    const int64_t W = batch_work<ROWS>(a, -1, b, base, sh_work);
    int64_t blocks = gridDim.x;
    if (blocks > W) blocks = W;
    if ((int64_t)blockIdx.x >= blocks) return;
    const int64_t begin = blockIdx.x * W / blocks, end = (blockIdx.x + 1ll) * W / blocks;
    __syncthreads();
    batch_work<ROWS>(a, begin, b, base, sh_work);

    char* ring = smem + warp * (STAGES * SB);
    // rows of the slice behind operand row n: n and n + 8 with the middle pairs crossed, so that the four rows a quarter of the lanes
    // reads of V lie in both halves of the banks
    const int tok = n ^ ((n >> 1) & 1);
    const int v0 = (2 * j) ^ (j & 1), v1 = (2 * j + 1) ^ (j & 1);   // the same for rows 2j and 2j + 1
    bool flag = false;

    for (int64_t u = begin; u < end;) {
        Seq q = seq_of<ROWS>(a, b);
        while (u >= base + q.work) {                             // on to the next sequence with work
            base += q.work;
            q = seq_of<ROWS>(a, ++b);
        }
        const int64_t local = u - base, item = local / q.units;
        const int u0 = (int)(local - item * q.units);
        const int u1 = (int)(q.units - u0 < end - u ? q.units : u0 + (end - u));
        const int head = (int)(item / q.tiles), tile = (int)(item - (int64_t)head * q.tiles);
        const int rows = q.n * a.group - tile * ROWS < ROWS ? q.n * a.group - tile * ROWS : ROWS;   // of the tile
        const int slot = qp_kv_slot(a.rows, b);

        // ---- queries: operand registers and, per column, the factors of a score
        unsigned qb[NT][QB], ql[SPLIT ? NT : 1][SPLIT ? QB : 1];
        float kf[NT][2], qs[NT][2];
        int hi[NT][2];                                           // last key that the column's query sees
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float e[D / 4];
            const int r = tile * ROWS + 8 * t + n;
            const bool mine = 8 * t + n < rows;
            if (mine) {
                const int token = q.row0 + r / a.group, h = head * a.group + r % a.group;
                load_q(static_cast<const T*>(a.q) + (int64_t)token * a.qt + (int64_t)h * a.qh + j * (D / 4), a.vec, e);
            } else {
#pragma unroll
                for (int i = 0; i < D / 4; ++i) e[i] = 0.f;
            }
            float top = 0.f, sum = 0.f;
#pragma unroll
            for (int i = 0; i < D / 4; ++i) { top = fmaxf(top, fabsf(e[i])); sum += e[i]; }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            }
            const bool bad = !(top < __int_as_float(0x7F800000)) || !(fabsf(sum) < __int_as_float(0x7F800000));
            // the row's largest element to [2^11, 2^12): fp16 then holds what is down to 2^-25 of it whole
            int ex = 265 - (int)(__float_as_uint(top) >> 23);
            ex = top == 0.f ? 127 : ex > 254 ? 254 : ex;
            const float norm = __uint_as_float((unsigned)ex << 23);
#pragma unroll
            for (int i = 0; i < D / 4; ++i) e[i] = bad ? 0.f : e[i] * norm;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float* x = e + 8 * w;
#pragma unroll
                for (int i = 0; i < 4; ++i) {                    // nibbles i and i + 4; odd ones stand a factor 16 higher
                    const float f = i & 1 ? 0.0625f : 1.f;
                    qb[t][4 * w + i] = half2_of(x[i] * f, x[i + 4] * f);
                    if constexpr (SPLIT)
                        ql[t][4 * w + i] = half2_of(x[i] * f - half_lo(qb[t][4 * w + i]), x[i + 4] * f - half_hi(qb[t][4 * w + i]));
                }
            }
            const float my_kf = a.scale_log2 / norm * (SPLIT ? 1.f : 16777216.f), my_qs = bad ? __int_as_float(0x7FC00000) : sum * a.scale_log2;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                kf[t][c] = __shfl_sync(0xFFFFFFFFu, my_kf, 4 * (2 * j + c));
                qs[t][c] = __shfl_sync(0xFFFFFFFFu, my_qs, 4 * (2 * j + c));
                int rc = 8 * t + 2 * j + c;
                rc = rc < rows ? rc : rows - 1;
                hi[t][c] = q.pos + (tile * ROWS + rc) / a.group;
            }
        }
        // a slice inside [all_lo, all_hi) is seen whole by every query of the tile
        const int all_hi = q.pos + (tile * ROWS) / a.group + 1;
        const int last_i = (tile * ROWS + rows - 1) / a.group;
        const int all_lo = a.window > 0 ? q.pos + last_i - a.window + 1 : 0;
        const int held = q.pos + q.n;                            // tokens behind are not written yet

        float o[NT][4 * VW][4];
        float m[NT][2], l[NT][2], lv[NT][2], vn = 1.2676506e30f; // 2^100
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 4 * VW; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[t][i][c] = 0.f;
#pragma unroll
            for (int c = 0; c < 2; ++c) { m[t][c] = M_NONE; l[t][c] = lv[t][c] = 0.f; }
        }

        // ---- the warp's slices: first, first + 4, ...
        const int first = q.s0 + WARPS * u0 + warp;
        int count = (q.s1 - first + WARPS - 1) / WARPS;
        count = count < u1 - u0 ? count : u1 - u0;               // may be negative: none
        int64_t place = -1;                                      // lane i: where slice 32 * k + i of the warp lies
        auto look_up = [&](int k) {
            const int it = 32 * k + lane;
            place = -1;
            if (it < count) {
                const int s = first + WARPS * it, p = s / a.slices;
                const int page = qp_kv_page(a.pages, slot, p * a.pages.page_size);
                if (page >= 0) place = (((int64_t)page * a.heads + head) * a.slices + (s - p * a.slices)) * SB;
                else flag = true;
            }
        };
        auto issue = [&](int it) {
            if (it < count) {
                if ((it & 31) == 0) look_up(it >> 5);
                const int64_t from = __shfl_sync(0xFFFFFFFFu, place, it & 31);
                char* to = ring + (it % STAGES) * SB + lane * 16;
                if (lane == 0) sh_ok[warp][it % STAGES] = from >= 0;
                if (from >= 0) {
                    const char* src = a.pool + from + lane * 16;
#pragma unroll
                    for (int i = 0; i < SB / 512; ++i) copy16(to + 512 * i, src + 512 * i);
                    if (SB % 512 && lane < SB % 512 / 16) copy16(to + SB / 512 * 512, src + SB / 512 * 512);
                }
            }
            copies_close();
        };
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i) issue(i);
        for (int it = 0; it < count; ++it) {
            copies_wait<STAGES - 2>();
            __syncwarp();
            issue(it + STAGES - 1);                              // into the stage of the round before
            const int stage = it % STAGES;
            if (!sh_ok[warp][stage]) continue;
            const char* x = ring + stage * SB;
            const int t0 = (first + WARPS * it) * QP_KV_SLICE;

            float s[NT][4];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int c = 0; c < 4; ++c) s[t][c] = 0.f;
            {
                unsigned ka[KW], kb[KW];
                lds_words(x + tok * S::ROW + j * (D / 8), ka);
                lds_words(x + (8 + tok) * S::ROW + j * (D / 8), kb);
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    const unsigned c0 = codes<SPLIT>(ka[w], M0), c1 = codes<SPLIT>(kb[w], M0), c2 = codes<SPLIT>(ka[w], M1), c3 = codes<SPLIT>(kb[w], M1);
                    const unsigned e0 = codes<SPLIT>(ka[w] >> 8, M0), e1 = codes<SPLIT>(kb[w] >> 8, M0);
                    const unsigned e2 = codes<SPLIT>(ka[w] >> 8, M1), e3 = codes<SPLIT>(kb[w] >> 8, M1);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if constexpr (SPLIT) {
                            float x4[4] = {0.f, 0.f, 0.f, 0.f};
                            mma(x4, c0, c1, c2, c3, ql[t][4 * w], ql[t][4 * w + 1]);
                            mma(x4, e0, e1, e2, e3, ql[t][4 * w + 2], ql[t][4 * w + 3]);
                            mma(x4, c0, c1, c2, c3, qb[t][4 * w], qb[t][4 * w + 1]);
                            mma(x4, e0, e1, e2, e3, qb[t][4 * w + 2], qb[t][4 * w + 3]);
#pragma unroll
                            for (int c = 0; c < 4; ++c) s[t][c] += x4[c];
                        } else {
                            mma(s[t], c0, c1, c2, c3, qb[t][4 * w], qb[t][4 * w + 1]);
                            mma(s[t], e0, e1, e2, e3, qb[t][4 * w + 2], qb[t][4 * w + 3]);
                        }
                    }
                }
            }
            float2 kq[2], vq[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                kq[h] = *reinterpret_cast<const float2*>(x + S::KQ + (8 * h + tok) * 8);
                vq[h] = *reinterpret_cast<const float2*>(x + S::VQ + (8 * h + tok) * 8);
            }
            const bool whole = t0 >= all_lo && t0 + QP_KV_SLICE <= all_hi;
            if (!whole) {
#pragma unroll
                for (int h = 0; h < 2; ++h)                      // rows that were never written may hold anything
                    if (t0 + 8 * h + tok >= held) kq[h] = vq[h] = make_float2(0.f, 0.f);
            }
            if constexpr (SPLIT) {                               // the codes are less 8: lo is the value of code 8
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    kq[h].x = fmaf(8.f, kq[h].y, kq[h].x);
                    vq[h].x = fmaf(8.f, vq[h].y, vq[h].x);
                }
            }
            // scores, in log2
            bool raise = vq[0].y * vn > V_SLACK || vq[1].y * vn > V_SLACK;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    s[t][c] = fmaf(s[t][c] * kq[c >> 1].y, kf[t][c & 1], kq[c >> 1].x * qs[t][c & 1]);
            if (!whole) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int key = t0 + 8 * (c >> 1) + tok;
                        if (key > hi[t][c & 1] || (a.window > 0 && key <= hi[t][c & 1] - a.window)) s[t][c] = -__int_as_float(0x7F800000);
                    }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int c = 0; c < 4; ++c) raise = raise || s[t][c] > m[t][c & 1] + M_SLACK;
            if (__any_sync(0xFFFFFFFFu, raise)) {                // rare: new references
                float vmax = fmaxf(vq[0].y, vq[1].y), f[NT][2];
#pragma unroll
                for (int o2 = 4; o2 < 32; o2 <<= 1) vmax = fmaxf(vmax, __shfl_xor_sync(0xFFFFFFFFu, vmax, o2));
                float back = 1.f;
                if (vmax * vn > V_SLACK) {
                    int ex = 258 - (int)(__float_as_uint(vmax) >> 23);
                    ex = ex > 254 ? 254 : ex;                    // (at least 258 - 254)
                    const float next = __uint_as_float((unsigned)ex << 23);   // vmax * next in [16, 32)
                    back = next / vn;
                    vn = next;
                }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float top = fmaxf(s[t][c], s[t][c + 2]);
#pragma unroll
                        for (int o2 = 4; o2 < 32; o2 <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o2));
                        const float next = fmaxf(m[t][c], top);
                        f[t][c] = ex2(m[t][c] - next);
                        m[t][c] = next;
                        l[t][c] *= f[t][c];
                        lv[t][c] *= f[t][c];
                        f[t][c] *= back;
                    }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 4 * VW; ++i)
#pragma unroll
                        for (int c = 0; c < 4; ++c) o[t][i][c] *= f[t][c & 1];
            }
            // probabilities; times V's scale they are the second product's operand
            unsigned pb[NT][2], pl[SPLIT ? NT : 1][2];
            const float vs[2] = {vq[0].y * vn, vq[1].y * vn};
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float p0 = ex2(s[t][2 * h] - m[t][0]), p1 = ex2(s[t][2 * h + 1] - m[t][1]);
                    l[t][0] += p0;
                    l[t][1] += p1;
                    lv[t][0] = fmaf(p0, vq[h].x, lv[t][0]);
                    lv[t][1] = fmaf(p1, vq[h].x, lv[t][1]);
                    const float w0 = p0 * vs[h], w1 = p1 * vs[h];
                    const unsigned x2 = half2_of(w0, w1);
                    pb[t][h] = transpose8(x2);
                    if constexpr (SPLIT) pl[t][h] = transpose8(half2_of(w0 - half_lo(x2), w1 - half_hi(x2)));
                }
            // out^T += V^T P^T
            {
                unsigned w0[VW], w1[VW], w2[VW], w3[VW];
                const char* v = x + S::V + n * (D / 16);
                lds_words(v + v0 * S::ROW, w0);
                lds_words(v + v1 * S::ROW, w1);
                lds_words(v + (8 + v0) * S::ROW, w2);
                lds_words(v + (8 + v1) * S::ROW, w3);
#pragma unroll
                for (int w = 0; w < VW; ++w)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {                // codes 0..3, 4..7 of the word; both tokens of a pair in one register
                        const unsigned y = __byte_perm(w0[w], w1[w], h ? 0x7632 : 0x5410), z = __byte_perm(w2[w], w3[w], h ? 0x7632 : 0x5410);
                        const unsigned c0 = codes<SPLIT>(y, M0), c1 = codes<SPLIT>(y >> 8, M0), c2 = codes<SPLIT>(z, M0), c3 = codes<SPLIT>(z >> 8, M0);
                        const unsigned e0 = codes<SPLIT>(y, M1), e1 = codes<SPLIT>(y >> 8, M1), e2 = codes<SPLIT>(z, M1), e3 = codes<SPLIT>(z >> 8, M1);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            if constexpr (SPLIT) {
                                float x4[4] = {0.f, 0.f, 0.f, 0.f}, y4[4] = {0.f, 0.f, 0.f, 0.f};
                                mma(x4, c0, c1, c2, c3, pl[t][0], pl[t][1]);
                                mma(y4, e0, e1, e2, e3, pl[t][0], pl[t][1]);
                                mma(x4, c0, c1, c2, c3, pb[t][0], pb[t][1]);
                                mma(y4, e0, e1, e2, e3, pb[t][0], pb[t][1]);
#pragma unroll
                                for (int c = 0; c < 4; ++c) { o[t][4 * w + 2 * h][c] += x4[c]; o[t][4 * w + 2 * h + 1][c] += y4[c]; }
                            } else {
                                mma(o[t][4 * w + 2 * h], c0, c1, c2, c3, pb[t][0], pb[t][1]);
                                mma(o[t][4 * w + 2 * h + 1], e0, e1, e2, e3, pb[t][0], pb[t][1]);
                            }
                        }
                    }
            }
        }
        copies_wait<0>();
        __syncthreads();                                         // the ring is free: it takes the warps' results

        // ---- the block's result: O [warp][row][D], then m and l [warp][row]
        float* mo = reinterpret_cast<float*>(smem);
        float* mm = mo + WARPS * ROWS * D;
        float* ml = mm + WARPS * ROWS;
        const float un = 1.f / vn;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float sl = l[t][c], sv = lv[t][c];
#pragma unroll
                for (int o2 = 4; o2 < 32; o2 <<= 1) {
                    sl += __shfl_xor_sync(0xFFFFFFFFu, sl, o2);
                    sv += __shfl_xor_sync(0xFFFFFFFFu, sv, o2);
                }
                const int r = 8 * t + 2 * j + c;
                if (n == 0) { mm[warp * ROWS + r] = m[t][c]; ml[warp * ROWS + r] = sl; }
                float* row = mo + (warp * ROWS + r) * D + n * (D / 8);
#pragma unroll
                for (int i = 0; i < 4 * VW; ++i) {               // tile i: elements e and e + 2 of word i / 4
                    const float f = (i & 1 ? 0.0625f : 1.f) * (SPLIT ? 1.f : 16777216.f);
                    const int e = 8 * (i >> 2) + 4 * ((i >> 1) & 1) + (i & 1);
                    row[e] = fmaf(o[t][i][c] * un, f, sv);
                    row[e + 2] = fmaf(o[t][i][c + 2] * un, f, sv);
                }
            }
        __syncthreads();
        const bool split = u0 > 0 || u1 < q.units;
        float* part = a.part + ((int64_t)blockIdx.x * 2 + (u == begin ? 0 : 1)) * (ROWS * (D + 2));
        for (int i = threadIdx.x; i < rows * D; i += THREADS) {
            const int r = i / D, d = i % D;
            float top = mm[r];
#pragma unroll
            for (int w = 1; w < WARPS; ++w) top = fmaxf(top, mm[w * ROWS + r]);
            float so = 0.f, sl = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float f = ex2(mm[w * ROWS + r] - top);
                so = fmaf(mo[(w * ROWS + r) * D + d], f, so);
                sl = fmaf(ml[w * ROWS + r], f, sl);
            }
            if (!split) {
                put_row<T, D>(a, q, head, tile * ROWS + r, d, so, top, sl);
            } else {
                __stcg(part + r * D + d, so);
                if (d == 0) { __stcg(part + ROWS * D + r, top); __stcg(part + ROWS * D + ROWS + r, sl); }
            }
        }
        if (split) {
            // blocks of this item: those of units i0 and i0 + units - 1, and all between
            const int64_t i0 = base + item * q.units;
            const int c0 = (int)(((i0 + 1) * blocks - 1) / W), c1 = (int)(((i0 + q.units) * blocks - 1) / W);
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) {
                const unsigned done = atomicAdd(a.count + c0, 1u);
                sh_last = done == (unsigned)(c1 - c0);
                if (sh_last) a.count[c0] = 0u;
            }
            __syncthreads();
            if (sh_last) {
                __threadfence();
                for (int i = threadIdx.x; i < rows * D; i += THREADS) {
                    const int r = i / D, d = i % D;
                    // a block's part of this item is its first unless it began in front of the item
                    const float* p1 = a.part + ((int64_t)c0 * 2 + (c0 * W / blocks < i0 ? 1 : 0)) * (ROWS * (D + 2));
                    float top = __ldcg(p1 + ROWS * D + r);
                    for (int c = c0 + 1; c <= c1; ++c) top = fmaxf(top, __ldcg(a.part + (int64_t)c * 2 * (ROWS * (D + 2)) + ROWS * D + r));
                    float so = 0.f, sl = 0.f;
                    for (int c = c0; c <= c1; ++c) {
                        const float* p = c == c0 ? p1 : a.part + (int64_t)c * 2 * (ROWS * (D + 2));
                        const float f = ex2(__ldcg(p + ROWS * D + r) - top);
                        so = fmaf(__ldcg(p + r * D + d), f, so);
                        sl = fmaf(__ldcg(p + ROWS * D + ROWS + r), f, sl);
                    }
                    put_row<T, D>(a, q, head, tile * ROWS + r, d, so, top, sl);
                }
            }
        }
        __syncthreads();                                         // shared memory is free for the next part
        u += u1 - u0;
    }
    if (flag) atomicOr(a.status, QP_DEV_KV_RANGE);
}

struct Launch {
    const void* kernel;
    int smem, per_sm, rows;
    bool* ready;
};

template <int D, int NT, bool SPLIT>
Launch launch_of()
{
    static bool ready[QP_KV_MAX_DEVICES];
    using C = Cfg<D, NT, SPLIT>;
    return {reinterpret_cast<const void*>(kv_attn_kernel<D, NT, SPLIT>), C::SMEM, C::PER_SM, C::ROWS, ready};
}

// rows: queries to a cached head, at most
Launch choose(int dim, bool f32, int64_t rows)
{
    if (f32) return dim == 64 ? launch_of<64, 1, true>() : dim == 128 ? launch_of<128, 1, true>() : launch_of<256, 1, true>();
    if (dim == 256) return launch_of<256, 1, false>();
    // 16 queries to a pass where there are more than 8: the codes are taken apart once for both halves
    if (rows > 8) return dim == 64 ? launch_of<64, 2, false>() : launch_of<128, 2, false>();
    return dim == 64 ? launch_of<64, 1, false>() : launch_of<128, 1, false>();
}

constexpr int MAX_PER_SM = 4, MAX_ROWS = 16;

}  // namespace

extern "C" uint64_t qp_kv_attention_work_bytes(qp_ctx* ctx, const qp_kv_cache_t* h_cache)
{
    if (!ctx || !h_cache || !qp_kv_dim_ok(h_cache->head_dim)) return 0;
    const uint64_t blocks = (uint64_t)ctx->sm_count * MAX_PER_SM;
    return QP_KV_COUNTERS * 4 + blocks * 2 * MAX_ROWS * (uint64_t)(h_cache->head_dim + 2) * 4;
}

extern "C" int32_t qp_kv_attention(qp_ctx* ctx, const qp_kv_cache_t* h_cache, const qp_kv_batch_t* h_batch, const qp_kv_attention_t* h_plan,
                                   int layer, const void* d_q, int dtype, int64_t q_token_stride, int64_t q_head_stride, void* d_out,
                                   int64_t out_token_stride, int64_t out_head_stride, float* d_lse, void* stream)
{
    if (!ctx) return QP_ERR_INVALID_ARG;
    int32_t rc = qp_kv_check_cache(ctx, h_cache);
    if (!rc) rc = qp_kv_check_batch(ctx, h_batch);
    if (!rc) rc = qp_kv_check_layer(ctx, h_cache, layer);
    if (rc) return rc;
    if (!h_plan) return qp_fail(ctx, QP_ERR_INVALID_ARG, "null plan");
    if (dtype != QP_F32 && dtype != QP_BF16) return qp_fail(ctx, QP_ERR_UNSUPPORTED_DTYPE, "dtype must be QP_F32 or QP_BF16");
    const qp_kv_cache_t* c = h_cache;
    if (h_plan->q_heads < 1 || h_plan->q_heads % c->heads) return qp_fail(ctx, QP_ERR_INVALID_ARG, "q_heads must be a multiple of the cache's heads");
    if (h_plan->window < 0) return qp_fail(ctx, QP_ERR_INVALID_ARG, "window");
    if (!(h_plan->scale - h_plan->scale == 0.f)) return qp_fail(ctx, QP_ERR_INVALID_ARG, "scale must be finite");
    const int group = h_plan->q_heads / c->heads;
    if ((int64_t)h_batch->tokens * h_plan->q_heads >= (1ll << 31) - 4096) return qp_fail(ctx, QP_ERR_INVALID_ARG, "tokens * q_heads must be below 2^31 - 4096");
    if (h_batch->batch == 0 || h_batch->tokens == 0 || h_batch->max_new == 0) return QP_OK;
    if (!d_q || !d_out) return qp_fail(ctx, QP_ERR_INVALID_ARG, "null d_q or d_out");
    const int64_t es = dtype == QP_F32 ? 4 : 2;
    if ((((uintptr_t)d_q | (uintptr_t)d_out) & (uintptr_t)(es - 1)) || ((uintptr_t)d_lse & 3u)) return qp_fail(ctx, QP_ERR_ALIGNMENT, "d_q, d_out or d_lse");
    if (!h_plan->d_work || h_plan->work_bytes < qp_kv_attention_work_bytes(ctx, c)) return qp_fail(ctx, QP_ERR_BUFFER_TOO_SMALL, "the plan's workspace");
    if ((uintptr_t)h_plan->d_work & 15u) return qp_fail(ctx, QP_ERR_ALIGNMENT, "the plan's workspace");
    qp_device_guard guard(ctx->device);
    if (!guard.ok) return qp_fail(ctx, QP_ERR_CUDA, "cannot select device");

    qp_kv_attn_args a;
    a.rows = qp_kv_rows_of(h_batch);
    a.pages = qp_kv_pages_of(c);
    a.pool = static_cast<const char*>(c->d_pool) + (size_t)layer * c->layer_stride;
    a.heads = c->heads;
    a.slices = c->page_size / QP_KV_SLICE;
    a.q_heads = h_plan->q_heads;
    a.group = group;
    a.max_new = h_batch->max_new < h_batch->tokens ? h_batch->max_new : h_batch->tokens;
    a.window = h_plan->window;
    a.scale_log2 = (float)((double)h_plan->scale * 1.4426950408889634);
    a.q = d_q; a.qt = q_token_stride; a.qh = q_head_stride;
    a.out = d_out; a.ot = out_token_stride; a.oh = out_head_stride;
    a.lse = d_lse;
    a.vec = (((uintptr_t)d_q & 15u) | (uintptr_t)(((q_token_stride | q_head_stride) * es) & 15)) == 0;
    a.count = static_cast<unsigned*>(h_plan->d_work);
    a.part = reinterpret_cast<float*>(a.count + QP_KV_COUNTERS);
    a.status = ctx->d_status;
    const Launch f = choose(c->head_dim, dtype == QP_F32, (int64_t)a.max_new * group);
    const int grid = ctx->sm_count * f.per_sm;
    if (grid > QP_KV_COUNTERS) return qp_fail(ctx, QP_ERR_INVALID_ARG, "device with more SMs than the workspace has counters for");
    if (ctx->device >= QP_KV_MAX_DEVICES || !f.ready[ctx->device]) {
        if (cudaFuncSetAttribute(f.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, f.smem) != cudaSuccess)
            return qp_check_launch(ctx, "qp_kv_attention (shared memory)");
        if (ctx->device < QP_KV_MAX_DEVICES) f.ready[ctx->device] = true;
    }
    void* args[] = {&a};
    cudaLaunchKernel(f.kernel, dim3((unsigned)grid), dim3(THREADS), args, (size_t)f.smem, static_cast<cudaStream_t>(stream));
    ctx->launches += 1;
    return qp_check_launch(ctx, "qp_kv_attention");
}
