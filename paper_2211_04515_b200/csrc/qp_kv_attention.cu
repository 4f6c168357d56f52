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
//     passes it by 6.  The weights p * scale' have a norm of their own for each query, lowered where one of them would leave fp16 and then
//     so that the largest is at 2^7 or more: what fp16 drops (2^-25) is 2^-32 of the query's largest weight, and keys that it does not see,
//     or whose p is next to nothing, have no part in it however large their values are.
//   - The work of the whole batch, in units of 64 tokens of one item (sequence, head, tile of queries), is cut into equal runs, one
//     for each resident block, whatever the lengths; an item counts HEAD units more than it has, for what its beginning and end
//     cost.  Where a cut falls inside an item, its blocks leave partial results, and the last to finish (counters; nobody
//     waits) adds them up in the blocks' order, so the result does not depend on timing.  Many parts are added in two
//     levels, about the square root of them at a time.
//   - fp32 queries (and probabilities) are split into two fp16 numbers, 22 bits together, with a product for each.  Two
//     things that 16 bits do not show cost bits there: the matrix unit lines its products up by the operands' exponents, so that a
//     subnormal's leading zeros are lost from the sum (1e-5 of the result), and it cuts sums off instead of rounding them.  So the codes
//     are made normal numbers there, and less 8 while at it (lo is then the value of code 8: smaller sums), and each slice's
//     sums start at zero and are added to the running ones by ordinary additions.
//
// Measured in a stream: 64 sequences of 200 to 8191 tokens, 32 query heads on 8 of 128: 59 us (212 MB, 3.6 TB/s over the whole call and 5.2
// while codes are read; 50 % of the issue slots); 120001 and 131071 tokens, 64 query heads on 4: 59 us (143 MB, 2.4 TB/s: 16 queries to a
// code; 44 % of the issue slots, 28 % of the matrix unit: latencies); one sequence of 1021: 11.6 us; fp32, 24 sequences of 197 to 1500, 12 heads
// of 64: 18.7 us (15 MB).  A part of an item costs about 8 us beside
// its codes, in latencies: its lengths and first codes 4, the reduction over warps 2, arrival and sum 2.
#include "qp_kv.cuh"
#include "qp_kv_attention.cuh"

QP_CK_UNIT

namespace {

constexpr int WARPS = 4, THREADS = WARPS * 32;
constexpr float M_NONE = -3.0e38f;               // reference before any score
constexpr float M_SLACK = 6.f;                   // a score may pass the reference by this (log2), so p is at most 64;
constexpr float W_MOST = 64000.f;                // and p * scale' * norm at most this, in fp16; no need to look at p while
constexpr float V_MOST = 1000.f;                 // scale' * norm is at most this
constexpr float W_TOP = 256.f;                   // a norm that is lowered takes the largest weight to half of this or more
constexpr float NORM_MOST = 8.507059e37f;        // 2^126: the norm before any weight
constexpr int UNIT = 4;                          // slices
// What an item's beginning and end cost, in units: 3 / 6 / 9 / 12 took 62.2 / 58.8 / 58.6 / 60.9 us for 64 sequences of 200 to 8191 tokens, 35.3 /
// 33.0 / 32.2 / 33.7 for drafted tokens of 16 sequences, 19.0 / 18.2 / 19.4 / 20.1 for 24 short sequences in fp32.
constexpr int HEAD = 6;
// Units that are worth a block: 1 / 2 / 3 / 4 took 13.0 / 11.5 / 12.2 / 12.3 us for one sequence of 1021 tokens (16 parts to an item are
// added in two levels, 8 in one); with more work than blocks there is no difference.
constexpr int MIN_RUN = 2;
// Blocks that are free of work at least, for the rows that no sequence writes where these become 0 (always, so that a call's bits do not depend
// on it).
constexpr unsigned REST_BLOCKS = 2;
// Query rows of a sequence to a cached head from which on the tensor-memory kernel takes it.  This one against that, us, at 64 / 128 / 256
// rows: 38 / 58 / 99 against 57 / 60 / 70 for 4 sequences of 4000 tokens and 8 heads.  Where the two meet also depends on how many items of
// work there are, which a rule on rows does not know: at 128 rows 99 against 74 for 16 sequences of 4000 and 4 heads, 56 against 94 for one
// of 16000 and 8 heads.  The rows are what a sequence knows about itself, whatever else is in its batch.
constexpr int MANY = 160;

template <int D, int NT, bool SPLIT> struct Cfg {
    static constexpr int ROWS = 8 * NT;
    static constexpr int SB = qp_kv_slice<D>::BYTES;
    static constexpr int SL = NT == 1 && !SPLIT && D < 256 ? 2 : 1;        // adjacent slices a warp takes at a time
    static constexpr int STAGES = D == 256 ? 4 : D == 128 ? 5 : 8;         // slices in a warp's ring
    static constexpr int RING = WARPS * STAGES * SB;
    static constexpr int MERGE = WARPS * ROWS * (D + 2) * 4;
    static constexpr int SMEM = RING > MERGE ? RING : MERGE;
    static constexpr int PER_SM = D == 256 || NT == 2 || SPLIT ? 3 : 4;
    static constexpr int PART = ROWS * (D + 2);                            // floats of a partial result
};
constexpr int MAX_PER_SM = 4, MAX_ROWS = 16;

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

__device__ __forceinline__ qp_f2 mul2(qp_f2 a, qp_f2 b)
{
    qp_f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b)          // of non-negative numbers
{
    return (uint64_t)(a | b) >> 32 ? a / b : (int64_t)((unsigned)a / (unsigned)b);
}

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
    int pos, n, row0, slot;                      // first position, tokens, row of the first
    int s0, s1;                                  // slices [s0, s1) hold the keys that some query sees
    int units, tiles;                            // HEAD + units of 64 tokens, query tiles
    int64_t work;                                // units in all
};

__device__ __forceinline__ bool takes_part(const Seq& q) { return q.n > 0 && q.pos >= 0 && q.pos <= 0x7FFFFFFF - q.n; }
// what follows from pos, n, row0 and slot
template <int ROWS>
__device__ __forceinline__ void derive(const qp_kv_attn_args& a, Seq& q)
{
    if (!takes_part(q) || (int64_t)q.n * a.group >= a.many) { q.work = 0; q.units = q.tiles = 0; q.s0 = q.s1 = 0; return; }
    const unsigned most = (unsigned)a.pages.max_pages * (unsigned)a.pages.page_size;     // (below 2^31, as pos and n)
    const unsigned end0 = (unsigned)q.pos + (unsigned)q.n, end = end0 < most ? end0 : most;
    unsigned lo = a.window > 0 && q.pos >= a.window ? (unsigned)(q.pos - a.window + 1) : 0u;
    if (lo > end) lo = end;
    q.s0 = (int)(lo / QP_KV_SLICE);
    q.s1 = (int)((end + QP_KV_SLICE - 1) / QP_KV_SLICE);
    q.units = (q.s1 - q.s0 + UNIT - 1) / UNIT;
    q.units = (q.units < 1 ? 1 : q.units) + HEAD;                // (an empty one still writes its rows)
    q.tiles = (int)(((unsigned)q.n * (unsigned)a.group + ROWS - 1) / ROWS);
    q.work = (int64_t)q.units * q.tiles * a.heads;
}
// rest: set if there are rows in front of the sequence, in it or behind it that nobody writes
template <int ROWS>
__device__ __forceinline__ Seq seq_of(const qp_kv_attn_args& a, int b, bool* rest)
{
    Seq q;
    q.pos = qp_kv_ld(a.rows.pos + b);
    q.slot = qp_kv_slot(a.rows, b);
    q.row0 = qp_kv_start(a.rows, b);
    const int row1 = qp_kv_start(a.rows, b + 1);
    q.n = row1 - q.row0;
    if (rest) *rest |= (b == 0 && q.row0 > 0) || (b == a.rows.batch - 1 && row1 < a.rows.tokens) || q.n < 0 || q.n > a.max_new;
    if (q.n > a.max_new) {                                       // (every block comes here for every sequence; one says so)
        if (blockIdx.x == 0) atomicOr(a.status, QP_DEV_KV_RANGE);
        q.n = a.max_new;
    }
    derive<ROWS>(a, q);
    if (rest) *rest |= q.n > 0 && !takes_part(q);
    // tokens behind the last page that the table has room for: counted as masked (the same for sequences that qp_kv_chunk.cu takes)
    const int most = a.pages.max_pages * a.pages.page_size;      // (below 2^31 - 4096)
    if (blockIdx.x == 0 && takes_part(q) && q.pos + q.n > most) atomicOr(a.status, QP_DEV_KV_RANGE);
    return q;
}

// Sequences b0 .. b0 + THREADS - 1 into shared memory, with the work in front of each (base: in front of b0); returns the work
// up to the last.
struct Chunk {
    int64_t before[THREADS + 1];
    int4 seq[THREADS];                           // pos, n, row0, slot
    int64_t sum[WARPS];
};
// A part of an item: the run of units that one block has of it.
struct Part {
    Seq q;
    int64_t u, next;                             // first unit and the one behind the last, counted with the items' heads
    int g0, u0, u1;                              // the first in the item, with its head; units without it
    int head, tile, rows;
};
// The part that begins with unit u of the chunk in shared memory; a warp does this by itself.
template <int ROWS>
__device__ __forceinline__ void find_part(const qp_kv_attn_args& a, const Chunk& sh, int64_t u, int64_t end, Part& to)
{
    const int lane = threadIdx.x & 31;
    unsigned hit = 0;
    int at = 0;
#pragma unroll
    for (int k = 0; k < THREADS / 32; ++k) {
        const unsigned in = __ballot_sync(0xFFFFFFFFu, u >= sh.before[32 * k + lane] && u < sh.before[32 * k + lane + 1]);
        if (in) { hit = in; at = 32 * k; }
    }
    at += __ffs(hit) - 1;
    const int4 x = sh.seq[QP_CK(at, THREADS)];
    Part p;
    p.q.pos = x.x; p.q.n = x.y; p.q.row0 = x.z; p.q.slot = x.w;
    derive<ROWS>(a, p.q);
    const int64_t local = u - sh.before[at], item = quotient(local, p.q.units);
    p.g0 = (int)(local - item * p.q.units);
    const int g1 = (int)(p.q.units - p.g0 < end - u ? p.q.units : p.g0 + (end - u));
    p.u = u;
    p.next = u + (g1 - p.g0);
    p.u0 = p.g0 > HEAD ? p.g0 - HEAD : 0;
    p.u1 = g1 - HEAD;
    p.head = (int)quotient(item, p.q.tiles);
    p.tile = (int)(item - (int64_t)p.head * p.q.tiles);
    const int all = p.q.n * a.group - p.tile * ROWS;
    p.rows = all < ROWS ? all : ROWS;
    if (lane == 0) to = p;
}
template <int ROWS>
__device__ __forceinline__ int64_t load_chunk(const qp_kv_attn_args& a, int b0, int64_t base, Chunk& sh, bool* rest = nullptr)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = b0 + threadIdx.x;
    Seq q = {-1, 0, 0, 0, 0, 0, 0, 0, 0};
    if (b < a.rows.batch) q = seq_of<ROWS>(a, b, rest);
    int64_t x = q.work;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();                                             // nobody reads the chunk before this any more
    if (lane == 31) sh.sum[warp] = x;
    sh.seq[threadIdx.x] = make_int4(q.pos, q.n, q.row0, q.slot);
    __syncthreads();
    int64_t front = base;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
        if (i < warp) front += sh.sum[i];
        base += sh.sum[i];
    }
    sh.before[threadIdx.x + 1] = front + x;
    if (threadIdx.x == 0) sh.before[0] = front;
    return base;
}

// this lane's D / 4 elements of a query row
template <int N>
__device__ __forceinline__ void load_q(const unsigned short* p, bool vec, float (&e)[N])
{
    if (vec) {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            const uint4 x = qp_kv_ld(reinterpret_cast<const uint4*>(p) + i);
            const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int h = 0; h < 4; ++h) { e[8 * i + 2 * h] = __uint_as_float(w[h] << 16); e[8 * i + 2 * h + 1] = __uint_as_float(w[h] & 0xFFFF0000u); }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = qp_bf16_to_f32(qp_kv_ld(p + i));
    }
}
template <int N>
__device__ __forceinline__ void load_q(const float* p, bool vec, float (&e)[N])
{
    if (vec) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float4 x = qp_kv_ld(reinterpret_cast<const float4*>(p) + i);
            e[4 * i] = x.x; e[4 * i + 1] = x.y; e[4 * i + 2] = x.z; e[4 * i + 3] = x.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = qp_kv_ld(p + i);
    }
}
__device__ __forceinline__ void put_out(float* p, bool vec, const float (&v)[4])
{
    if (vec) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = v[i];
}
__device__ __forceinline__ void put_out(unsigned short* p, bool vec, const float (&v)[4])
{
    unsigned short h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = qp_f32_to_bf16(v[i]);
    if (vec) *reinterpret_cast<uint2*>(p) = make_uint2(h[0] | ((unsigned)h[1] << 16), h[2] | ((unsigned)h[3] << 16));
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = h[i];
}

// Rows that no sequence writes become 0: the n blocks without a part of the work look at the whole batch for each row (uncommon: a padded
// batch, sequences that take no part; in the other blocks the code for it costs registers, 1 to 3 us a call).
template <typename T, int D>
__device__ __forceinline__ void zero_rows(const qp_kv_attn_args& a, int first, int n)
{
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
    for (int row = first; row < a.rows.tokens; row += n) {
        bool mine = false;
        for (int b = threadIdx.x; b < a.rows.batch && !mine; b += THREADS) {
            Seq q;
            q.pos = qp_kv_ld(a.rows.pos + b);
            q.row0 = qp_kv_start(a.rows, b);
            q.n = min(qp_kv_start(a.rows, b + 1) - q.row0, a.max_new);
            mine = takes_part(q) && row >= q.row0 && row - q.row0 < q.n;
        }
        if (__syncthreads_or(mine)) continue;
        for (int64_t i = threadIdx.x; i < (int64_t)a.q_heads * (D / 4); i += THREADS)
            put_out(static_cast<T*>(a.out) + row * a.ot + i / (D / 4) * a.oh + 4 * (i % (D / 4)), a.out_vec, zero);
    }
}

// What a tile's rows need at the end, worked out once by a thread each: where a row of out begins, and 1 over the sum of its weights (0 for
// a row that saw nothing; NaN stays NaN).  Writes lse.
struct RowEnds { int64_t at[16]; float over[16]; };
template <typename T>
__device__ __forceinline__ void end_row(const qp_kv_attn_args& a, const Seq& q, int head, int r, float m, float l, int64_t& at, float& over)
{
    const int token = q.row0 + r / a.group, h = head * a.group + r % a.group;
    at = (int64_t)token * a.ot + (int64_t)h * a.oh;
    over = l == 0.f ? 0.f : 1.f / l;
    if (a.lse) a.lse[(int64_t)token * a.q_heads + h] = l == 0.f ? -__int_as_float(0x7F800000) : (m + log2f(l)) * 0.6931471805599453f;
}
// four elements of a row, from their weighted sum
template <typename T>
__device__ __forceinline__ void put_row(const qp_kv_attn_args& a, int64_t at, float over, int d, float4 o)
{
    const float v[4] = {o.x * over, o.y * over, o.z * over, o.w * over};
    put_out(static_cast<T*>(a.out) + at + d, a.out_vec, v);
}

// Whether this block is the last of n to come here (the counter is at zero again then).  What the others wrote before is visible.
__device__ __forceinline__ bool arrived(unsigned* count, int n, int& sh)
{
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();                                         // (for the whole block's writes: the barrier put them in front)
        sh = atomicAdd(count, 1u) == (unsigned)(n - 1);
        if (sh) *count = 0u;
        __threadfence();
    }
    __syncthreads();
    return sh != 0;
}

// Adds n partial results: the first at place `at`, part i > 0 at place even + 2 * step * i; in that order.  Into `sum`, a partial
// result again (it may be the first), or (null) into out.
template <typename T, int D, int ROWS>
__device__ __forceinline__ void add_parts(const qp_kv_attn_args& a, const Seq& q, int head, int tile, int rows, int at, int even,
                                          int step, int n, float* sum, char* smem, RowEnds& ends)
{
    constexpr int PART = ROWS * (D + 2);
    auto part = [&](int i) { return a.part + (int64_t)QP_CK(i ? even + 2 * step * i : at, 2 * gridDim.x) * PART; };
    float* f = reinterpret_cast<float*>(smem);                   // [n][2 ROWS] references, then factors, and sums; [ROWS] of the whole
    float* tops = f + n * 2 * ROWS;
    __syncthreads();                                             // shared memory is free
    for (int i = threadIdx.x; i < n * 2 * ROWS; i += THREADS) f[QP_CK(i, WARPS * ROWS * (D + 2) - 2 * ROWS)] = __ldcg(part(i / (2 * ROWS)) + ROWS * D + i % (2 * ROWS));
    __syncthreads();
    if (threadIdx.x < (unsigned)rows) {
        const int r = threadIdx.x;
        float top = M_NONE, l = 0.f;
        for (int p = 0; p < n; ++p) top = fmaxf(top, f[p * 2 * ROWS + r]);
        for (int p = 0; p < n; ++p) {
            const float w = ex2(f[p * 2 * ROWS + r] - top);
            f[p * 2 * ROWS + r] = w;
            l = fmaf(w, f[p * 2 * ROWS + ROWS + r], l);
        }
        tops[r] = top;
        tops[ROWS + r] = l;
        if (!sum) end_row<T>(a, q, head, tile * ROWS + r, top, l, ends.at[r], ends.over[r]);
    }
    __syncthreads();
    // all of a thread's elements of some parts are asked for at once: what this costs is the trips to L2
    constexpr int MINE = ROWS * (D / 4) / THREADS, AT_ONCE = 8 / MINE > 0 ? 8 / MINE : 1;
    float4 so[MINE];
#pragma unroll
    for (int k = 0; k < MINE; ++k) so[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    const int last = rows * (D / 4) - 1;
#pragma unroll 1
    for (int p0 = 0; p0 < n; p0 += AT_ONCE) {
        float4 y[AT_ONCE][MINE];
#pragma unroll
        for (int p = 0; p < AT_ONCE; ++p)
#pragma unroll
            for (int k = 0; k < MINE; ++k) {                     // (past the end: again the last, with no weight)
                const int i = threadIdx.x + k * THREADS;
                y[p][k] = __ldcg(reinterpret_cast<const float4*>(part(p0 + p < n ? p0 + p : n - 1)) + (i < last ? i : last));
            }
#pragma unroll
        for (int p = 0; p < AT_ONCE; ++p)
#pragma unroll
            for (int k = 0; k < MINE; ++k) {
                const int i = threadIdx.x + k * THREADS;
                const float w = p0 + p < n ? f[(p0 + p) * 2 * ROWS + (i < last ? i : last) / (D / 4)] : 0.f;
                const float4 x = p0 + p < n ? y[p][k] : make_float4(0.f, 0.f, 0.f, 0.f);
                so[k].x = fmaf(x.x, w, so[k].x); so[k].y = fmaf(x.y, w, so[k].y);
                so[k].z = fmaf(x.z, w, so[k].z); so[k].w = fmaf(x.w, w, so[k].w);
            }
    }
#pragma unroll
    for (int k = 0; k < MINE; ++k) {
        const int i = threadIdx.x + k * THREADS, r = i / (D / 4), d = 4 * (i % (D / 4));
        if (r >= rows) continue;
        if (!sum) {
            put_row<T>(a, ends.at[r], ends.over[r], d, so[k]);
        } else {
            __stcg(reinterpret_cast<float4*>(sum + r * D + d), so[k]);
            if (d == 0) { __stcg(sum + ROWS * D + r, tops[r]); __stcg(sum + ROWS * D + ROWS + r, tops[ROWS + r]); }
        }
    }
}

template <int D, int NT, bool SPLIT>
__global__ void __launch_bounds__(THREADS, Cfg<D, NT, SPLIT>::PER_SM) kv_attn_kernel(const qp_kv_attn_args a)
{
    using C = Cfg<D, NT, SPLIT>;
    using S = qp_kv_slice<D>;
    using T = typename std::conditional<SPLIT, float, unsigned short>::type;
    constexpr int ROWS = C::ROWS, SB = C::SB, STAGES = C::STAGES, SL = C::SL;
    constexpr int KW = D / 32, VW = D / 64;                      // words of 8 codes a lane holds of a K row, of a V row
    constexpr int QB = 4 * KW;                                   // operand registers of a query tile
    constexpr unsigned M0 = 0x000F000Fu, M1 = 0x00F000F0u;
    extern __shared__ __align__(16) char smem[];
    qp_kv_begin();
    __shared__ Chunk chunk;
    __shared__ Part part[2];
    __shared__ int sh_ok[WARPS][STAGES], sh_hi[WARPS][ROWS];    // slices that are there; last key that a query sees
    __shared__ int sh_last;
    __shared__ RowEnds ends;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = lane >> 2, j = lane & 3;

    int b0 = 0;
    bool rest = a.rows.batch == 0;
    int64_t base = 0, upto = load_chunk<ROWS>(a, 0, 0, chunk, &rest), W = upto;
    for (int c = THREADS; c < a.rows.batch; c += THREADS) W = load_chunk<ROWS>(a, c, W, chunk, &rest);
    const int64_t most = gridDim.x - REST_BLOCKS, blocks = most * MIN_RUN < W ? most : (W + MIN_RUN - 1) / MIN_RUN;
    if ((int64_t)blockIdx.x >= blocks) {
        if (a.zero_rest && __syncthreads_or(rest)) zero_rows<T, D>(a, blockIdx.x - (int)blocks, gridDim.x - (int)blocks);
        return;
    }
    const int64_t begin = quotient(blockIdx.x * W, blocks), end = quotient((blockIdx.x + 1ll) * W, blocks);
    if (a.rows.batch > THREADS) {                                // back to the chunk that the run begins in
        upto = load_chunk<ROWS>(a, 0, 0, chunk);
        while (upto <= begin) { base = upto; upto = load_chunk<ROWS>(a, b0 += THREADS, base, chunk); }
    }

    char* ring = smem + warp * (STAGES * SB);
    // rows of the slice behind operand row n: n and n + 8 with the middle pairs crossed, so that the four rows a quarter of the lanes
    // reads of V lie in both halves of the banks
    const int tok = n ^ ((n >> 1) & 1);
    const int v0 = (2 * j) ^ (j & 1), v1 = (2 * j + 1) ^ (j & 1);   // the same for rows 2j and 2j + 1
    bool flag = false;

    // Lane i: the warp's slice number 32 * k + i of a part, and where it lies (-1: nowhere) by the table's entry.  The first entries of
    // a part are asked for while the one before it is finished.
    auto slice_of = [&](const Part& p, int k) {
        return p.q.s0 + UNIT * p.u0 + SL * warp + SL * WARPS * ((32 * k + lane) / SL) + (SL == 2 ? lane & 1 : 0);
    };
    auto stop_of = [&](const Part& p) { const int s = p.q.s0 + UNIT * p.u1; return s < p.q.s1 ? s : p.q.s1; };
    auto ask = [&](const Part& p, int k) {
        const int s = slice_of(p, k), i = s / a.slices;
        const bool in = s < stop_of(p) && (unsigned)p.q.slot < (unsigned)a.pages.max_seqs && i < a.pages.max_pages;
        return in ? qp_kv_ld(a.pages.table + (size_t)p.q.slot * a.pages.max_pages + i) : -1;
    };
    auto place_of = [&](const Part& p, int k, int page) {
        const int s = slice_of(p, k);
        if (s >= stop_of(p)) return (int64_t)-1;
        const bool in = page >= 0 && page < a.pages.num_pages;
        flag |= !in;
        return in ? (((int64_t)page * a.heads + p.head) * a.slices + s % a.slices) * SB : (int64_t)-1;
    };

    __syncthreads();
    if (warp == 0) find_part<ROWS>(a, chunk, begin, end, part[0]);
    __syncthreads();
    int entry = ask(part[0], 0);
    for (int turn = 0;; turn ^= 1) {
        const Part& p = part[turn];
        const int u0 = p.u0, u1 = p.u1, rows = p.rows, tile = p.tile, head = p.head;
        const int64_t next = p.next;
        const Seq& q = p.q;
        // (the next part's description is there behind the part's last barriers)
        auto look_ahead = [&]() {
            while (next >= upto) { base = upto; upto = load_chunk<ROWS>(a, b0 += THREADS, base, chunk); }
            __syncthreads();
            if (warp == 0) find_part<ROWS>(a, chunk, next, end, part[turn ^ 1]);
            __syncthreads();
            entry = ask(part[turn ^ 1], 0);
        };
        if (u1 <= u0) {                                          // nothing but the item's head
            if (next >= end) break;
            look_ahead();
            continue;
        }
        if (warp == 0 && next < end && next < upto) find_part<ROWS>(a, chunk, next, end, part[turn ^ 1]);

        // ---- the warp's slices, SL adjacent ones at a time: first + SL * WARPS * k + h
        const int first = q.s0 + UNIT * u0 + SL * warp, stop = stop_of(p);
        const int count = first < stop ? (stop - first + SL * WARPS - 1) / (SL * WARPS) : 0;
        int64_t place = place_of(p, 0, entry);
        int put = 0, take = 0;                                   // places in the ring
        auto issue = [&](int i) {                                // the warp's slice number i
            if (i < count * SL) {
                if ((i & 31) == 0 && i > 0) place = place_of(p, i >> 5, ask(p, i >> 5));
                const int64_t from = __shfl_sync(0xFFFFFFFFu, place, i & 31);
                if (lane == 0) sh_ok[warp][QP_CK(put, STAGES)] = from >= 0;
                if (from >= 0) {
                    char* to = ring + QP_CK(put, STAGES) * SB + lane * 16;
                    const char* src = a.pool + from + lane * 16;
#pragma unroll
                    for (int c = 0; c < SB / 512; ++c) copy16(to + 512 * c, src + 512 * c);
                    if (SB % 512 && lane < SB % 512 / 16) copy16(to + SB / 512 * 512, src + SB / 512 * 512);
                }
                put = put + 1 == STAGES ? 0 : put + 1;
            }
            copies_close();
        };
        // (the queries are asked for, the copies go out, then the queries are looked at)
        float e[NT][D / 4];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int r = tile * ROWS + 8 * t + n;
            if (8 * t + n < rows) {
                const int token = q.row0 + r / a.group, h = head * a.group + r % a.group;
                load_q(static_cast<const T*>(a.q) + (int64_t)token * a.qt + (int64_t)h * a.qh + j * (D / 4), a.vec, e[t]);
            } else {
#pragma unroll
                for (int i = 0; i < D / 4; ++i) e[t][i] = 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < STAGES; ++i) issue(i);

        // ---- queries: operand registers and, per column, the factors of a score
        unsigned qb[NT][QB], ql[SPLIT ? NT : 1][SPLIT ? QB : 1];
        qp_f2 kf[NT], qs[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float top = 0.f, sum = 0.f;
#pragma unroll
            for (int i = 0; i < D / 4; ++i) top = fmaxf(top, fabsf(e[t][i]));
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            // the row's largest element to [2^11, 2^12): fp16 then holds what is down to 2^-25 of it whole
            int ex = 265 - (int)(__float_as_uint(top) >> 23);
            ex = top == 0.f ? 127 : ex > 254 ? 254 : ex;
            const float norm = __uint_as_float((unsigned)ex << 23);
#pragma unroll
            for (int i = 0; i < D / 4; ++i) { e[t][i] *= norm; sum += e[t][i]; }      // (at most 2^20; NaN where an element is not finite,
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            if (!(top < __int_as_float(0x7F800000))) sum = __int_as_float(0x7FC00000);   // or taken so; products stay in the query's column)
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float* x = e[t] + 8 * w;
#pragma unroll
                for (int i = 0; i < 4; ++i) {                    // nibbles i and i + 4; odd ones stand a factor 16 higher
                    const float f = i & 1 ? 0.0625f : 1.f;
                    qb[t][4 * w + i] = half2_of(x[i] * f, x[i + 4] * f);
                    if constexpr (SPLIT)
                        ql[t][4 * w + i] = half2_of(x[i] * f - half_lo(qb[t][4 * w + i]), x[i + 4] * f - half_hi(qb[t][4 * w + i]));
                }
            }
            const float back = a.scale_log2 / norm, my_kf = back * (SPLIT ? 1.f : 16777216.f), my_qs = sum * back;
            kf[t] = qp_pack2(__shfl_sync(0xFFFFFFFFu, my_kf, 8 * j), __shfl_sync(0xFFFFFFFFu, my_kf, 8 * j + 4));
            qs[t] = qp_pack2(__shfl_sync(0xFFFFFFFFu, my_qs, 8 * j), __shfl_sync(0xFFFFFFFFu, my_qs, 8 * j + 4));
        }
        if (lane < ROWS) sh_hi[warp][lane] = q.pos + (tile * ROWS + (lane < rows ? lane : rows - 1)) / a.group;
        // a slice inside [all_lo, all_hi) is seen whole by every query of the tile
        const int all_hi = q.pos + (tile * ROWS) / a.group + 1;
        const int last_i = (tile * ROWS + rows - 1) / a.group;
        const int all_lo = a.window > 0 ? q.pos + last_i - a.window + 1 : 0;

        float o[NT][4 * VW][4];
        qp_f2 mn[NT], l[NT], lv[NT], wn[NT];                     // the reference, negated; sums of p and of p * lo'; norm of the weights
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 4 * VW; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[t][i][c] = 0.f;
            mn[t] = qp_pack2(-M_NONE, -M_NONE);
            l[t] = lv[t] = qp_pack2(0.f, 0.f);
            wn[t] = qp_pack2(NORM_MOST, NORM_MOST);
        }

        for (int it = 0; it < count; ++it) {
            copies_wait<STAGES - SL>();
            __syncwarp();
            const int t0 = (first + SL * WARPS * it) * QP_KV_SLICE;
            const char* at[SL];
            bool ok[SL], all = t0 >= all_lo && t0 + SL * QP_KV_SLICE <= all_hi;
#pragma unroll
            for (int i = 0; i < SL; ++i) {
                at[i] = ring + QP_CK(take, STAGES) * SB;
                ok[i] = sh_ok[warp][take] != 0;
                all = all && ok[i];
                take = take + 1 == STAGES ? 0 : take + 1;
            }

            qp_f2 s[SL][NT][2];                                  // scores, in log2: of operand rows n and n + 8, two queries each
            float2 vq[SL][2];
#pragma unroll
            for (int i = 0; i < SL; ++i) {
                const char* x = at[i];
                float raw[NT][4];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int c = 0; c < 4; ++c) raw[t][c] = 0.f;
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
                            for (int c = 0; c < 4; ++c) raw[t][c] += x4[c];
                        } else {
                            mma(raw[t], c0, c1, c2, c3, qb[t][4 * w], qb[t][4 * w + 1]);
                            mma(raw[t], e0, e1, e2, e3, qb[t][4 * w + 2], qb[t][4 * w + 3]);
                        }
                    }
                }
                float2 kq[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    kq[h] = *reinterpret_cast<const float2*>(x + S::KQ + (8 * h + tok) * 8);
                    vq[i][h] = *reinterpret_cast<const float2*>(x + S::VQ + (8 * h + tok) * 8);
                    // rows that were never written, or not copied, may hold anything
                    if (!all && (!ok[i] || t0 + 16 * i + 8 * h + tok >= p.q.pos + p.q.n)) kq[h] = vq[i][h] = make_float2(0.f, 0.f);
                    if constexpr (SPLIT) {                       // the codes are less 8: lo is the value of code 8
                        kq[h].x = fmaf(8.f, kq[h].y, kq[h].x);
                        vq[i][h].x = fmaf(8.f, vq[i][h].y, vq[i][h].x);
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        s[i][t][h] = qp_fma2(mul2(qp_pack2(raw[t][2 * h], raw[t][2 * h + 1]), qp_pack2(kq[h].y, kq[h].y)), kf[t],
                                             mul2(qp_pack2(kq[h].x, kq[h].x), qs[t]));
                }
            }
            if (!all) {
#pragma unroll
                for (int i = 0; i < SL; ++i)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float y[2];
                            qp_unpack2(s[i][t][h], y[0], y[1]);
                            const int key = t0 + 16 * i + 8 * h + tok;
#pragma unroll
                            for (int c = 0; c < 2; ++c)
                            {
                                const int hi = sh_hi[warp][8 * t + 2 * j + c];
                                if (!ok[i] || key > hi || (a.window > 0 && key <= hi - a.window)) y[c] = -__int_as_float(0x7F800000);
                            }
                            s[i][t][h] = qp_pack2(y[0], y[1]);
                        }
            }
            float over = -1.f, vmax = 0.f, nmax = 0.f;           // how far the scores pass their references; the largest scale of V and norm
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float y0, y1;
                qp_unpack2(wn[t], y0, y1);
                nmax = qp_max3(nmax, y0, y1);
            }
#pragma unroll
            for (int i = 0; i < SL; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    vmax = fmaxf(vmax, vq[i][h].y);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        float y0, y1;
                        qp_unpack2(qp_add2(s[i][t][h], mn[t]), y0, y1);
                        over = qp_max3(over, y0, y1);
                    }
                }
            if (__any_sync(0xFFFFFFFFu, over > M_SLACK || vmax * nmax > V_MOST)) {     // uncommon: look at the weights themselves
                float most = 0.f;
#pragma unroll
                for (int i = 0; i < SL; ++i)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float y0, y1, n0, n1;
                            qp_unpack2(qp_add2(s[i][t][h], mn[t]), y0, y1);
                            qp_unpack2(wn[t], n0, n1);
                            most = qp_max3(most, ex2(y0) * vq[i][h].y * n0, ex2(y1) * vq[i][h].y * n1);
                        }
                if (__any_sync(0xFFFFFFFFu, over > M_SLACK || most > W_MOST)) {        // rare: new references
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        float top[2] = {M_NONE, M_NONE}, w[2] = {0.f, 0.f}, old[2], norm[2], f[2], back[2];
                        qp_unpack2(mn[t], old[0], old[1]);
                        qp_unpack2(wn[t], norm[0], norm[1]);
#pragma unroll
                        for (int i = 0; i < SL; ++i)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                float y0, y1;
                                qp_unpack2(s[i][t][h], y0, y1);
                                top[0] = fmaxf(top[0], y0);
                                top[1] = fmaxf(top[1], y1);
                            }
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
#pragma unroll
                            for (int o2 = 4; o2 < 32; o2 <<= 1) top[c] = fmaxf(top[c], __shfl_xor_sync(0xFFFFFFFFu, top[c], o2));
                            top[c] = fmaxf(-old[c], top[c]);
                            f[c] = ex2(-old[c] - top[c]);
                        }
                        mn[t] = qp_pack2(-top[0], -top[1]);
#pragma unroll
                        for (int i = 0; i < SL; ++i)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                float y0, y1;
                                qp_unpack2(s[i][t][h], y0, y1);
                                w[0] = fmaxf(w[0], ex2(y0 - top[0]) * vq[i][h].y);
                                w[1] = fmaxf(w[1], ex2(y1 - top[1]) * vq[i][h].y);
                            }
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
#pragma unroll
                            for (int o2 = 4; o2 < 32; o2 <<= 1) w[c] = fmaxf(w[c], __shfl_xor_sync(0xFFFFFFFFu, w[c], o2));
                            // the p so far are f times as large: the norm takes that up where it can, so that what out holds may stay
                            float next = f[c] > 0.f ? fminf(norm[c] / f[c], NORM_MOST) : NORM_MOST;
                            if (w[c] * next > W_TOP) {
                                const int ex = 261 - (int)(__float_as_uint(w[c]) >> 23);          // w * next in [2^7, 2^8)
                                next = __uint_as_float((unsigned)(ex > 253 ? 253 : ex < 1 ? 1 : ex) << 23);
                            }
                            back[c] = f[c] > 0.f ? f[c] * (next / norm[c]) : 0.f;
                            norm[c] = next;
                        }
                        wn[t] = qp_pack2(norm[0], norm[1]);
                        l[t] = mul2(l[t], qp_pack2(f[0], f[1]));
                        lv[t] = mul2(lv[t], qp_pack2(f[0], f[1]));
#pragma unroll
                        for (int i = 0; i < 4 * VW; ++i)
#pragma unroll
                            for (int c = 0; c < 4; ++c) o[t][i][c] *= back[c & 1];
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < SL; ++i) {
                // probabilities; times V's scale and the norm they are the second product's operand
                unsigned pb[NT][2], pl[SPLIT ? NT : 1][2];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float p0, p1, w0, w1;
                        qp_unpack2(qp_add2(s[i][t][h], mn[t]), p0, p1);
                        const qp_f2 p = qp_pack2(ex2(p0), ex2(p1));
                        l[t] = qp_add2(l[t], p);
                        lv[t] = qp_fma2(p, qp_pack2(vq[i][h].x, vq[i][h].x), lv[t]);
                        qp_unpack2(mul2(mul2(p, qp_pack2(vq[i][h].y, vq[i][h].y)), wn[t]), w0, w1);
                        const unsigned x2 = half2_of(w0, w1);
                        pb[t][h] = transpose8(x2);
                        if constexpr (SPLIT) pl[t][h] = transpose8(half2_of(w0 - half_lo(x2), w1 - half_hi(x2)));
                    }
                // out^T += V^T P^T
                unsigned w0[VW], w1[VW], w2[VW], w3[VW];
                const char* v = at[i] + S::V + n * (D / 16);
                lds_words(v + v0 * S::ROW, w0);
                lds_words(v + v1 * S::ROW, w1);
                lds_words(v + (8 + v0) * S::ROW, w2);
                lds_words(v + (8 + v1) * S::ROW, w3);
#pragma unroll
                for (int w = 0; w < VW; ++w)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {                // codes 0..3, 4..7 of the word; both tokens of a pair in one register
                        const unsigned y = __byte_perm(w0[w], w1[w], h ? 0x7632 : 0x5410), z = __byte_perm(w2[w], w3[w], h ? 0x7632 : 0x5410);
                        unsigned c0, c1, c2, c3, e0, e1, e2, e3;
                        if constexpr (SPLIT) {
                            c0 = codes<true>(y, M0); c1 = codes<true>(y >> 8, M0); c2 = codes<true>(z, M0); c3 = codes<true>(z >> 8, M0);
                            e0 = codes<true>(y, M1); e1 = codes<true>(y >> 8, M1); e2 = codes<true>(z, M1); e3 = codes<true>(z >> 8, M1);
                        } else {                                 // the odd code's sum comes with the even one's in a whole byte: one operation less
                            e0 = y & 0x00FF00FFu; e1 = __byte_perm(y, 0u, 0x4341); e2 = z & 0x00FF00FFu; e3 = __byte_perm(z, 0u, 0x4341);
                            c0 = y & M0; c1 = e1 & M0; c2 = z & M0; c3 = e3 & M0;
                        }
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
            __syncwarp();                                        // all lanes have read: the places are filled again
#pragma unroll
            for (int i = 0; i < SL; ++i) issue(SL * it + STAGES + i);
        }
        copies_wait<0>();
        __syncthreads();                                         // the ring is free: it takes the warps' results
        if (next < end && next < upto) entry = ask(part[turn ^ 1], 0);

        // ---- the block's result: O [warp][row][D], then m and l [warp][row]
        float* mo = reinterpret_cast<float*>(smem);
        float* mm = mo + WARPS * ROWS * D;
        float* ml = mm + WARPS * ROWS;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float sl[2], sv[2], mc[2], norm0, norm1;
            qp_unpack2(wn[t], norm0, norm1);
            qp_unpack2(l[t], sl[0], sl[1]);
            qp_unpack2(lv[t], sv[0], sv[1]);
            qp_unpack2(mn[t], mc[0], mc[1]);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int o2 = 4; o2 < 32; o2 <<= 1) {
                    sl[c] += __shfl_xor_sync(0xFFFFFFFFu, sl[c], o2);
                    sv[c] += __shfl_xor_sync(0xFFFFFFFFu, sv[c], o2);
                }
                const int r = 8 * t + 2 * j + c;
                if (n == 0) { mm[warp * ROWS + r] = -mc[c]; ml[warp * ROWS + r] = sl[c]; }
                float* row = mo + (warp * ROWS + r) * D + n * (D / 8);
                // (codes as subnormals: 2^24 in two steps, so that neither leaves fp32)
                constexpr float f = SPLIT ? 1.f : 4096.f, less = SPLIT ? 0.f : 1.f;
                const float un = f / (c ? norm1 : norm0);
#pragma unroll
                for (int i = 0; i < 4 * VW; i += 2) {            // tiles i and i + 1: elements e, e + 2 and e + 1, e + 3 of word i / 4
                    *reinterpret_cast<float4*>(row + 8 * (i >> 2) + 4 * ((i >> 1) & 1)) =
                        make_float4(fmaf(o[t][i][c] * un, f, sv[c]), fmaf((o[t][i + 1][c] - less * o[t][i][c]) * un, f * 0.0625f, sv[c]),
                                    fmaf(o[t][i][c + 2] * un, f, sv[c]), fmaf((o[t][i + 1][c + 2] - less * o[t][i][c + 2]) * un, f * 0.0625f, sv[c]));
                }
            }
        }
        __syncthreads();
        const bool split = u0 > 0 || u1 < q.units - HEAD;
        const int64_t i0 = p.u - p.g0;                           // the item's first unit; its blocks:
        int c0 = 0, c1 = 0, at = 0;
        if (split) {
            c0 = (int)quotient((i0 + HEAD + 1) * blocks - 1, W);
            c1 = (int)quotient((i0 + q.units) * blocks - 1, W);
            // a block's part of an item is its first if the item began in front of it or with it
            at = 2 * (int)blockIdx.x + (p.u == begin ? 0 : 1);
        }
        float* mine_at = a.part + (int64_t)QP_CK(at, 2 * gridDim.x) * C::PART;
        if (threadIdx.x < (unsigned)rows) {                      // the warps' references become factors
            const int r = threadIdx.x;
            float top = mm[r], sl = 0.f;
#pragma unroll
            for (int w = 1; w < WARPS; ++w) top = fmaxf(top, mm[w * ROWS + r]);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float f = ex2(mm[w * ROWS + r] - top);
                sl = fmaf(ml[w * ROWS + r], f, sl);
                mm[w * ROWS + r] = f;
            }
            if (split) { __stcg(mine_at + ROWS * D + r, top); __stcg(mine_at + ROWS * D + ROWS + r, sl); }
            else end_row<T>(a, q, head, tile * ROWS + r, top, sl, ends.at[r], ends.over[r]);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < rows * (D / 4); i += THREADS) {
            const int r = i / (D / 4), d = 4 * (i % (D / 4));
            float4 so = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float f = mm[w * ROWS + r];
                const float4 y = *reinterpret_cast<const float4*>(mo + (w * ROWS + r) * D + d);
                so.x = fmaf(y.x, f, so.x); so.y = fmaf(y.y, f, so.y); so.z = fmaf(y.z, f, so.z); so.w = fmaf(y.w, f, so.w);
            }
            if (split) __stcg(reinterpret_cast<float4*>(mine_at + r * D + d), so);
            else put_row<T>(a, ends.at[r], ends.over[r], d, so);
        }
        if (split) {
            // the parts of blocks c0 .. c1, `step` of them to a group; the group's sum takes the place of its first part
            const int parts = c1 - c0 + 1, first_at = 2 * c0 + (quotient(c0 * W, blocks) < i0 ? 1 : 0);
            int step = parts;
            if (parts > 8) {
                step = 4;
                while (step * step < parts) ++step;
            }
            const int group = ((int)blockIdx.x - c0) / step, groups = (parts + step - 1) / step;
            const int gc = c0 + group * step, gn = parts - group * step < step ? parts - group * step : step;
            const int g_at = group ? 2 * gc : first_at;
            float* sum = a.part + (int64_t)QP_CK(g_at, 2 * gridDim.x) * C::PART;
            bool mine = arrived(a.count + QP_CK(g_at, QP_KV_COUNTERS / 2), gn, sh_last);
            if (mine && groups == 1) {
                add_parts<T, D, ROWS>(a, q, head, tile, rows, first_at, 2 * c0, 1, parts, nullptr, smem, ends);
            } else if (mine) {
                add_parts<T, D, ROWS>(a, q, head, tile, rows, g_at, 2 * gc, 1, gn, sum, smem, ends);
                mine = arrived(a.count + QP_KV_COUNTERS / 2 + QP_CK(first_at, QP_KV_COUNTERS / 2), groups, sh_last);
                if (mine) add_parts<T, D, ROWS>(a, q, head, tile, rows, first_at, 2 * c0, step, groups, nullptr, smem, ends);
            }
        }
        if (next >= end) break;
        if (next >= upto) look_ahead();
        else __syncthreads();                                    // shared memory is free for the next part
    }
    if (flag) atomicOr(a.status, QP_DEV_KV_RANGE);
}

struct Launch {
    void (*kernel)(const qp_kv_attn_args);
    int smem, per_sm, rows;
    bool* ready;
};

template <int D, int NT, bool SPLIT>
Launch launch_of()
{
    static bool ready[QP_KV_MAX_DEVICES];
    using C = Cfg<D, NT, SPLIT>;
    return {kv_attn_kernel<D, NT, SPLIT>, C::SMEM, C::PER_SM, C::ROWS, ready};
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

}  // namespace

extern "C" uint64_t qp_kv_attention_work_bytes(qp_ctx* ctx, const qp_kv_cache_t* h_cache)
{
    if (!ctx || !h_cache || !qp_kv_dim_ok(h_cache->head_dim)) return 0;
    const uint64_t blocks = (uint64_t)ctx->sm_count * MAX_PER_SM;
    const uint64_t few = blocks * 2 * MAX_ROWS * (uint64_t)(h_cache->head_dim + 2) * 4, many = qp_kv_chunk_part_bytes(h_cache->head_dim, ctx->sm_count);
    return QP_KV_COUNTERS * 4 + (few > many ? few : many);
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
    if (h_plan->flags & ~QP_KV_ZERO_REST) return qp_fail(ctx, QP_ERR_INVALID_ARG, "flags");
    const bool zero_rest = (h_plan->flags & QP_KV_ZERO_REST) != 0;
    if (h_batch->tokens == 0 || (!zero_rest && (h_batch->batch == 0 || h_batch->max_new == 0))) return QP_OK;
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
    a.out_vec = (((uintptr_t)d_out & (uintptr_t)(4 * es - 1)) | (uintptr_t)(((out_token_stride | out_head_stride) * es) & (4 * es - 1))) == 0;
    a.count = static_cast<unsigned*>(h_plan->d_work);
    a.part = reinterpret_cast<float*>(a.count + QP_KV_COUNTERS);
    a.zero_rest = zero_rest;
    a.status = ctx->d_status;
    a.many = 0x7FFFFFFF;
    a.wait_cycles = ctx->wait_cycles;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == QP_BF16 && c->head_dim <= 128 && (int64_t)a.max_new * group >= MANY) {
        a.many = MANY;
        rc = qp_kv_chunk_launch(ctx, a, c->head_dim, s);
        if (rc) return rc;
    }
    const Launch f = choose(c->head_dim, dtype == QP_F32, a.many < 0x7FFFFFFF ? a.many - 1 : (int64_t)a.max_new * group);
    const int grid = ctx->sm_count * f.per_sm;
    if (2 * grid > QP_KV_COUNTERS / 2) return qp_fail(ctx, QP_ERR_INVALID_ARG, "device with more SMs than the workspace has counters for");
    if (ctx->device >= QP_KV_MAX_DEVICES || !f.ready[ctx->device]) {
        if (cudaFuncSetAttribute(f.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, f.smem) != cudaSuccess)
            return qp_check_launch(ctx, "qp_kv_attention (shared memory)");
        if (ctx->device < QP_KV_MAX_DEVICES) f.ready[ctx->device] = true;
    }
    qp_kv_launch(f.kernel, (unsigned)grid, THREADS, (size_t)f.smem, s, a);
    ctx->launches += 1;
    return qp_check_launch(ctx, "qp_kv_attention");
}
