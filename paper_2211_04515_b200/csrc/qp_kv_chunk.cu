// Attention over the 4-bit cache for many queries to a cached head (chunks of a prompt), bf16, on tcgen05.
//
// An item is 256 query rows of one cached head (row = token * group + query head of the group: all of them read the same
// keys) as two tiles of 128, against the keys they see in tiles of 128, taken in halves of 64.  Per half and query tile
//     S = Q K^T    128 x 64 x D, both operands in shared memory, S in tensor memory
//     P = 2^(S f - X)   a thread to a row
//     O += P V     P from tensor memory (over S), V in shared memory, O in tensor memory
//
// Roles: warps 0-3 and 4-7 are the rows of query tiles 0 and 1; warps 8-11 turn the cache's codes into fp16 operands; warp 12
// issues the products.  The two query tiles take turns: one's softmax runs while the other's products do.
//
// What it has to do: 4 * 256 * 128 * D operations of the products (2048 cycles at D = 128 and the nominal rate) and as many cycles for
// the 32768 exponentials (16 a cycle).  So a softmax element gets three more operations and no more: the codes are not multiplied
// as they are, as for few queries (their quantizers would cost two operations and shared-memory reads on every score and weight), but
// as their values in fp16: a nibble under 1024's exponent is 1024 + code (or + 16 * code), less 1032 it is code - 8, and a fused
// operation takes two of them to (lo + 8 scale) + scale * (code - 8): 13 operations to 8 codes.  (In fp32 first, rounded once: 20, and the whole
// kernel 14 % slower.  The nibbles as subnormals, without the subtraction: 10, but the range left for values is 2^20 within a tile.)
// The result, scale and the value of code 8 are each rounded to 11 bits, an eighth of what bf16 would lose.  (About code 0 instead: lo is
// several times the middle of a row, and its rounding moves a whole row of scores; the result was 1.6 times as far off.)  fp16's range: each tile of K and of V is scaled by a power of two that takes its largest
// value to [2^10, 2^11); queries are scaled by row.  K's power goes into the factor of the scores, V's into the exponent of
// the weights (both are one number a tile).  A tile whose rows are of very different sizes has a power for each of them, which goes into
// each score, or each weight's exponent.  Elements lie in the order 0 4 1 5 2 6 3 7 of each eight, in the operands and in O.
//
//   - Softmax reference raised only when a score passes it by 8 (log2).  O has another, of the scores plus V's powers: raised likewise, and then O
//     is read from tensor memory, scaled and put back.
//   - The work, in key tiles, is cut into equal runs for the SMs; an item that a cut falls into leaves partial results
//     and the last block to finish adds them (as for few queries).
//   - Registers: 128 a thread at launch; the softmax warps go to 160 (a row's 64 scores stay in registers), the issuing warp's group
//     to 64 (2 * 160 + 128 + 64 = 4 * 128).  One copy of each hot loop: unrolled for each role they did not fit the instruction
//     cache (1161 us against 936 for the case below).
//   - Measured: 2048 tokens over 9001 and 16384, 32 query heads on 8 of 128: 952 us, 736 TFLOP/s, with the GPU at its power limit.
//     52 % of the issue slots, tcgen05 43 % of the time: neither is full.  The scores' products take 6 KB of operands
//     for 32 cycles at the nominal rate, more than the 128 bytes a cycle that shared memory gives; that this bounds them is not shown.
//   - Every wait has a limit: a block that gives up raises QP_DEV_STREAM_TIMEOUT, its roles leave, the products in flight are
//     waited for, tensor memory is freed.
#include "qp_kv.cuh"
#include "qp_kv_attention.cuh"
#include "qp_stream.cuh"

QP_CK_UNIT

namespace {

constexpr int THREADS = 512, TILE = 128, ROWS = 2 * TILE;
constexpr int HALF = 64;                         // keys of a step of softmax and products
constexpr int HEAD = 2;                          // what an item costs beside its key tiles, in key tiles
constexpr int MIN_RUN = 4;                       // key tiles that are worth a block
constexpr int SEGS = 32;                         // parts of items that are listed at a time
constexpr float M_NONE = -3.0e38f, M_SLACK = 8.f;
constexpr int P_SHIFT = 5;                       // weights are 2^5 higher: up to 2^13 in fp16
// A tile whose rows of V have largest values further apart than this (log2) has a power of two for each row.  2048 tokens over 9001 and 16384
// take 1743 us if every tile does, 956 if none does.  (Rows 2^7 apart under one power lose 7 of the 39 powers of two that
// fp16 has below 2^13.)
constexpr int V_SPREAD = 7;
// The same for rows of K: a row's largest value stands at 2^-2 or above, so that what fp16 drops is 2^-23 of it.
constexpr int K_SPREAD = 12;

template <int D> struct Cfg {
    static constexpr int OPERAND = TILE * D * 2;                 // bytes of Q, K, V tiles
    static constexpr int SMEM = 1024 + 6 * OPERAND;
    static constexpr int PART = TILE * (D + 2);                  // floats of a query tile's partial result
    static constexpr int SB = qp_kv_slice<D>::BYTES;
    static constexpr int LOADS = TILE * (D / 2) / 16 / 128;      // 16-byte loads of a thread for K's codes of a tile
};

// ---------------------------------------------------------------------------- tcgen05

__device__ __forceinline__ uint32_t smem_of(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// operand in shared memory: rows of 128 bytes, 16-byte pieces exchanged within 8 rows (128-byte swizzle).  K-major: the row is the
// M or N index, eight rows 1024 bytes on; MN-major: the row is the K index, 64 elements of M or N to a panel, panels `lead` bytes apart
__device__ __forceinline__ uint64_t operand_at(uint32_t addr, uint32_t lead)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// fp16 x fp16 -> fp32, M = 128
__host__ __device__ constexpr uint32_t shape_of(int n, bool b_mn_major)
{
    return 1u << 4 | (b_mn_major ? 1u << 16 : 0u) | (uint32_t)(n / 8) << 17 | (uint32_t)(128 / 16) << 24;
}
// (called by a whole warp, issued by one lane: what the instructions take in uniform registers stays uniform)
__device__ __forceinline__ bool leader()
{
    uint32_t e;
    asm volatile("{.reg .pred p; elect.sync _|p, 0xFFFFFFFF; selp.b32 %0, 1, 0, p;}" : "=r"(e));
    return e != 0u;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add)
{
    if (leader())
        asm volatile("{.reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;}" ::"r"(d), "l"(a), "l"(b),
                     "r"(shape), "r"((uint32_t)add)
                     : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t shape, bool add)
{
    if (leader())
        asm volatile("{.reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;}" ::"r"(d), "r"(a), "l"(b),
                     "r"(shape), "r"((uint32_t)add)
                     : "memory");
}
__device__ __forceinline__ void commit(uint64_t* bar)
{
    if (leader()) asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_of(bar)) : "memory");
}
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
// the loads into x are there: nothing that uses x may move in front of this
template <int N>
__device__ __forceinline__ void wait_ld(float (&x)[N])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+f"(x[i]));
}
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_operands() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 32 columns of a warp's 32 rows, a row to a lane
__device__ __forceinline__ void tmem_ld32(uint32_t at, float* x)
{
    uint32_t* r = reinterpret_cast<uint32_t*>(x);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,"
        "%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(at));
}
__device__ __forceinline__ void tmem_st32(uint32_t at, const float* x)
{
    const uint32_t* r = reinterpret_cast<const uint32_t*>(x);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,"
        "%26,%27,%28,%29,%30,%31,%32};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t* r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                 "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}

__device__ __forceinline__ void tmem_ld16(uint32_t at, float* x)
{
    uint32_t* r = reinterpret_cast<uint32_t*>(x);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_st8(uint32_t at, const uint32_t* r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ unsigned half2_of(float lo, float hi)
{
    unsigned r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ unsigned mul_h2(unsigned a, unsigned b)
{
    unsigned r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ unsigned fma_h2(unsigned a, unsigned b, unsigned c)
{
    unsigned r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
// codes less 8 (16 times that under the higher mask): 1024 + x has x in its low bits
template <unsigned MASK>
__device__ __forceinline__ unsigned nibbles(unsigned w)
{
    unsigned r = (w & MASK) | 0x64006400u;
    asm("sub.f16x2 %0, %0, %1;" : "+r"(r) : "r"(MASK == 0x000F000Fu ? 0x64086408u : 0x64806480u));
    return r;
}
// a warp's arrival, for all that its lanes did before
__device__ __forceinline__ void arrive(uint64_t* bar)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_of(bar)) : "memory");
}
template <int ID> __device__ __forceinline__ void group_sync() { asm volatile("bar.sync %0, 128;" ::"n"(ID) : "memory"); }
__device__ __forceinline__ void group_sync(int id) { asm volatile("bar.sync %0, 128;" ::"r"(id) : "memory"); }
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((unsigned)(e < -126 ? 1 : e > 127 ? 254 : e + 127) << 23); }

// 2^e for e <= 0, to the smallest subnormal; 0 below
__device__ __forceinline__ float pow2_down(int e) { return e >= -126 ? pow2(e) : e >= -149 ? __uint_as_float(1u << (149 + e)) : 0.f; }

// ---------------------------------------------------------------------------- work

// a part of an item: key tiles [u0, u1) of query rows tile * ROWS ..
struct Seg {
    int pos, n, row0, slot, head, tile, u0, u1;
    int s0;                                      // slice that key tile 0 begins with
    int split, c0, c1, first_at, at;             // parts of the item: blocks c0 .. c1, places of the first and of this one
};

struct Shared {
    uint64_t q_full[2], kv_full[2], kv_empty[2], s_full[2][2], p_full[2][2], pv_done[2][2], all_done;
    uint32_t tmem, give_up;
    int n_segs, more;
    // per stage: what takes K's scaled values back (bits of a float), the power of two that V's were divided by, and per 32 keys which
    // are there
    int2 about[2];
    uint4 valid[2];
    float2 quant[2][2][TILE];                    // K's and V's quantizers of a tile
    // where rows are scaled one by one (spread: 1 V's, 2 K's): a row of V's power of two less the tile's; 2 to that for a row of K
    alignas(16) float row_power[2][TILE], row_scale[2][TILE];
    int spread[2];
    unsigned amax[2][2][4];                      // per 32 keys the largest value of K and of V (bits of a float),
    int amin[2][2][4];                           // and the smallest power of a row
    int last[2];
    Seg segs[SEGS];
};

struct Seq { int pos, n, row0, slot, tiles; };

__device__ __forceinline__ Seq seq_of(const qp_kv_attn_args& a, int b)
{
    Seq q;
    q.pos = qp_kv_ld(a.rows.pos + b);
    q.slot = qp_kv_slot(a.rows, b);
    q.row0 = qp_kv_start(a.rows, b);
    q.n = qp_kv_start(a.rows, b + 1) - q.row0;
    if (q.n > a.max_new) q.n = a.max_new;
    const int64_t rows = (int64_t)q.n * a.group;
    q.tiles = q.n <= 0 || q.pos < 0 || q.pos > 0x7FFFFFFF - q.n || rows < a.many ? 0 : (int)((rows + ROWS - 1) / ROWS);
    return q;
}
// slices [first, first + 8 * returned) hold the keys that rows tile * ROWS .. see (counts of rows and of keys fit 32 bits)
__device__ __forceinline__ int tiles_of(const qp_kv_attn_args& a, const Seq& q, int tile, int& first)
{
    const unsigned most = (unsigned)a.pages.max_pages * (unsigned)a.pages.page_size, group = (unsigned)a.group;
    const unsigned r0 = (unsigned)tile * ROWS, all = (unsigned)q.n * group, r1 = r0 + ROWS < all ? r0 + ROWS : all;
    const unsigned end0 = (unsigned)q.pos + (r1 - 1) / group + 1u, end = end0 < most ? end0 : most;
    unsigned lo = 0u;
    if (a.window > 0) {
        const unsigned at = (unsigned)q.pos + r0 / group + 1u;
        lo = at > (unsigned)a.window ? at - (unsigned)a.window : 0u;
        if (lo > end) lo = end;
    }
    first = (int)(lo / QP_KV_SLICE);
    const int slices = (int)((end + QP_KV_SLICE - 1) / QP_KV_SLICE) - first;
    return slices < 1 ? 1 : (slices + TILE / QP_KV_SLICE - 1) / (TILE / QP_KV_SLICE);
}
__device__ __forceinline__ int64_t work_of(const qp_kv_attn_args& a, const Seq& q)      // of one head
{
    int64_t w = 0;
    int first;
    for (int t = 0; t < q.tiles; ++t) w += HEAD + tiles_of(a, q, t, first);
    return w;
}

// lists the block's next parts, from unit u on; warp 0.  b: the sequence, base: work in front of it
__device__ __forceinline__ void list_parts(const qp_kv_attn_args& a, Shared& sh, int64_t& u, int64_t end, int64_t begin, int64_t W,
                                           int64_t blocks, int& b, int64_t& base)
{
    int n = 0;
    while (u < end && n < SEGS) {
        Seq q = seq_of(a, b);
        int64_t one = work_of(a, q);
        while (u >= base + one * a.heads) {
            base += one * a.heads;
            q = seq_of(a, ++b);
            one = work_of(a, q);
        }
        int head = (int)((u - base) / one);
        int64_t i0 = base + head * one;
        while (u < end && head < a.heads && n < SEGS) {
            int tile = 0, first, units = HEAD + tiles_of(a, q, 0, first);
            while (u >= i0 + units) { i0 += units; units = HEAD + tiles_of(a, q, ++tile, first); }
            for (; tile < q.tiles && u < end && n < SEGS; ++tile) {
                units = HEAD + tiles_of(a, q, tile, first);
                const int g0 = (int)(u - i0), g1 = units - g0 < end - u ? units : g0 + (int)(end - u);
                const int u0 = g0 > HEAD ? g0 - HEAD : 0, u1 = g1 - HEAD;
                if (u1 > u0) {
                    Seg s;
                    s.pos = q.pos; s.n = q.n; s.row0 = q.row0; s.slot = q.slot; s.head = head; s.tile = tile;
                    s.u0 = u0; s.u1 = u1; s.s0 = first;
                    s.split = u0 > 0 || u1 < units - HEAD;
                    s.c0 = s.c1 = s.first_at = s.at = 0;
                    if (s.split) {
                        s.c0 = (int)(((i0 + HEAD + 1) * blocks - 1) / W);
                        s.c1 = (int)(((i0 + units) * blocks - 1) / W);
                        s.first_at = 2 * s.c0 + ((int64_t)s.c0 * W / blocks < i0 ? 1 : 0);
                        s.at = 2 * (int)blockIdx.x + (u == begin ? 0 : 1);
                    }
                    if ((threadIdx.x & 31) == 0) sh.segs[QP_CK(n, SEGS)] = s;
                    ++n;
                }
                u += g1 - g0;
                i0 += units;
            }
            ++head;
        }
    }
    if ((threadIdx.x & 31) == 0) { sh.n_segs = n; sh.more = u < end; }
}

// A wait with a limit.  Once one has run out none waits any more: every role goes on to the end of its loops, so that no barrier is
// left with a part of its threads, and nothing more is written out.
__device__ __forceinline__ bool given_up(const Shared& sh) { return *(const volatile uint32_t*)&sh.give_up != 0u; }
__device__ __forceinline__ void wait_on(Shared& sh, uint64_t* bar, unsigned parity, long long limit)
{
    const long long since = clock64();
    while (!qp_stream::mbar_try_wait(bar, parity)) {
        if (given_up(sh)) return;
        if (clock64() - since > limit) {
            *(volatile uint32_t*)&sh.give_up = 1u;
            return;
        }
    }
}
__device__ __forceinline__ void wait(Shared& sh, uint64_t* bar, unsigned parity, long long limit)
{
    if (!qp_stream::mbar_try_wait(bar, parity)) wait_on(sh, bar, parity, limit);
}

// ---------------------------------------------------------------------------- the cache's codes into operands

template <int D>
__device__ __forceinline__ void produce(const qp_kv_attn_args& a, Shared& sh, char* stages, int& g)
{
    using C = Cfg<D>;
    using S = qp_kv_slice<D>;
    constexpr int L = C::LOADS, PER = 16 * (D / 32);             // 16-byte pieces of a slice's K (or V) codes
    const int p = threadIdx.x & 127, lane = p & 31;
    // this thread's piece of a slice: row and 32 elements; eight lanes take eight rows, so that their stores meet all banks
    const int in = p & (PER - 1), row = (in & 7) + 8 * ((in >> 3) & (D == 128 ? 0 : 1)) + (D == 128 ? 8 * (in >> 5) : 0);
    const int piece = D == 128 ? (in >> 3) & 3 : in >> 4;
    for (int i = 0; i < sh.n_segs; ++i) {
        const Seg& s = sh.segs[i];
        const int held = s.pos + s.n, units = s.u1 - s.u0;
        // keys that some row of the item sees: the others must not count where a power of two is chosen for a tile
        const int row0 = s.tile * ROWS, row1 = min(row0 + ROWS, s.n * a.group);
        const int seen0 = a.window > 0 ? s.pos + row0 / a.group - a.window + 1 : 0, seen1 = s.pos + (row1 - 1) / a.group + 1;
        // what a tile needs from memory, in registers: asked for one tile ahead, its places two
        struct Raw { uint4 k[L], v[L]; float4 quant; unsigned there; } now, next;
        int64_t place = -1;
        auto look_up = [&](int u) {                              // lane i < 8 of each warp: slice i
            const int sl = s.s0 + 8 * u + lane, pg = sl / a.slices;
            place = -1;
            if (lane < 8 && u < s.u1 && (int64_t)sl * QP_KV_SLICE < held) {
                const int page = qp_kv_page(a.pages, s.slot, pg * a.pages.page_size);
                if (page >= 0) place = (((int64_t)page * a.heads + s.head) * a.slices + (sl - pg * a.slices)) * C::SB;
                else atomicOr(a.status, QP_DEV_KV_RANGE);
            }
        };
        auto load = [&](Raw& x, int u) {
#pragma unroll
            for (int l = 0; l < L; ++l) {
                const int64_t at = __shfl_sync(0xFFFFFFFFu, place, (l * 128 + p) / PER);
                const char* from = a.pool + at + row * S::ROW + piece * 16;
                x.k[l] = at >= 0 ? qp_kv_ld(reinterpret_cast<const uint4*>(from)) : make_uint4(0, 0, 0, 0);
                x.v[l] = at >= 0 ? qp_kv_ld(reinterpret_cast<const uint4*>(from + S::V)) : make_uint4(0, 0, 0, 0);
            }
            const int64_t mine = __shfl_sync(0xFFFFFFFFu, place, p / QP_KV_SLICE);
            x.quant = make_float4(0.f, 0.f, 0.f, 0.f);
            const int key = (s.s0 + 8 * u) * QP_KV_SLICE + p;
            const bool there = mine >= 0 && key >= seen0 && key < seen1;
            if (there) {
                const float2 kq = qp_kv_ld(reinterpret_cast<const float2*>(a.pool + mine + S::KQ + p % QP_KV_SLICE * 8));
                const float2 vq = qp_kv_ld(reinterpret_cast<const float2*>(a.pool + mine + S::VQ + p % QP_KV_SLICE * 8));
                x.quant = make_float4(kq.x, kq.y, vq.x, vq.y);
            }
            x.there = __ballot_sync(0xFFFFFFFFu, there);
        };
        auto convert = [&](Raw& x) {
            const int st = g & 1;
            const float4 quant = x.quant;
            // powers of two for the tile, which take its largest value to [2^10, 2^11) (not below -100: nothing to gain)
            const unsigned k_bits = __float_as_uint(fmaxf(fabsf(quant.x), fabsf(fmaf(15.f, quant.y, quant.x))));
            const unsigned v_bits = __float_as_uint(fmaxf(fabsf(quant.z), fabsf(fmaf(15.f, quant.w, quant.z))));
            const int k_own = max((int)(k_bits >> 23) - 137, -100), v_own = max((int)(v_bits >> 23) - 137, -100);
            const unsigned ka = __reduce_max_sync(0xFFFFFFFFu, k_bits), va = __reduce_max_sync(0xFFFFFFFFu, v_bits);
            // (a row of zeros is one however it is scaled; of V it may have all the weight, and then the others must not lose theirs)
            const int kmin = __reduce_min_sync(0xFFFFFFFFu, k_bits ? k_own : 1000);
            const int vmin = __reduce_min_sync(0xFFFFFFFFu, x.there >> lane & 1u ? v_own : 1000);
            if (lane == 0) {
                sh.amax[st][0][p >> 5] = ka; sh.amax[st][1][p >> 5] = va;
                sh.amin[st][0][p >> 5] = kmin; sh.amin[st][1][p >> 5] = vmin;
            }
            sh.quant[st][0][p] = make_float2(quant.x, quant.y);
            sh.quant[st][1][p] = make_float2(quant.z, quant.w);
            group_sync<1>();
            unsigned kb = 0, vb = 0;
            int k_least = 1000, v_least = 1000;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                kb = max(kb, sh.amax[st][0][w]); vb = max(vb, sh.amax[st][1][w]);
                k_least = min(k_least, sh.amin[st][0][w]); v_least = min(v_least, sh.amin[st][1][w]);
            }
            const int ke = max((int)(kb >> 23) - 137, -100), ve = max((int)(vb >> 23) - 137, -100);
            const int spread = (ve - v_least > V_SPREAD ? 1 : 0) | (ke - k_least > K_SPREAD ? 2 : 0);      // (the same in all threads)
            const float kf = spread & 2 ? 1.f : pow2(-ke), vf = spread & 1 ? 1.f : pow2(-ve);
            if (g >= 2) wait(sh, &sh.kv_empty[st], ((g >> 1) + 1) & 1, a.wait_cycles);
            __syncwarp();
            if (spread) {
                const float k_f = pow2(-k_own), v_f = pow2(-v_own);
                if (spread & 2) sh.quant[st][0][p] = make_float2(quant.x * k_f, quant.y * k_f);
                if (spread & 1) sh.quant[st][1][p] = make_float2(quant.z * v_f, quant.w * v_f);
                sh.row_scale[st][p] = spread & 2 ? pow2_down(k_own - ke) : 1.f;
                sh.row_power[st][p] = spread & 1 ? (float)(v_own - ve) : 0.f;
                group_sync<1>();
            }
            char* to = stages + st * (2 * C::OPERAND);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {                        // K, then V
                const float f = h ? vf : kf;
#pragma unroll
                for (int l = 0; l < L; ++l) {
                    const int sl = (l * 128 + p) / PER, key = sl * QP_KV_SLICE + row;
                    const float2 q = sh.quant[st][h][QP_CK(key, TILE)];
                    const float sc = q.y * f;
                    const unsigned m1 = half2_of(sc, sc), m16 = mul_h2(m1, 0x2C002C00u);         // (times 2^-4)
                    const float mid = fmaf(8.f, sc, q.x * f);
                    const unsigned base = half2_of(mid, mid);
                    const uint4 codes = x.k[l];
                    const unsigned w4[4] = {codes.x, codes.y, codes.z, codes.w};
                    char* panel = to + h * C::OPERAND + (D == 128 ? (piece >> 1) * (TILE * 128) : 0) + key * 128;
                    const int c0 = D == 128 ? 4 * (piece & 1) : 4 * piece;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const unsigned high = w4[w] >> 8;        // codes 0 4, 1 5 and 2 6, 3 7 at bits 0..3, 4..7 of each half
                        const uint4 out = make_uint4(fma_h2(nibbles<0x000F000Fu>(w4[w]), m1, base), fma_h2(nibbles<0x00F000F0u>(w4[w]), m16, base),
                                                     fma_h2(nibbles<0x000F000Fu>(high), m1, base), fma_h2(nibbles<0x00F000F0u>(high), m16, base));
                        *reinterpret_cast<uint4*>(panel + (((c0 + w) ^ (key & 7)) << 4)) = out;
                    }
                }
#pragma unroll
                for (int l = 0; l < L; ++l) x.k[l] = x.v[l];
            }
            if (p == 0) { sh.about[st] = make_int2(__float_as_int(pow2(ke)), ve); sh.spread[st] = spread; }
            if (lane == 0) (&sh.valid[st].x)[p >> 5] = x.there;
            fence_operands();
            arrive(&sh.kv_full[st]);
            ++g;
        };
        look_up(s.u0);
        load(now, s.u0);
        look_up(s.u0 + 1);
#pragma unroll 1
        for (int u = 0; u < units; ++u) {
            load(next, s.u0 + u + 1);                            // (behind the last: nothing)
            look_up(s.u0 + u + 2);
            convert(now);
            now = next;
        }
    }
}

// ---------------------------------------------------------------------------- products

template <int D>
__device__ __forceinline__ void multiply(const qp_kv_attn_args& a, Shared& sh, char* q_at, char* stages, int& g, int& items)
{
    using C = Cfg<D>;
    constexpr uint32_t S_SHAPE = shape_of(HALF, false), O_SHAPE = shape_of(D, true);
    const uint32_t tm = sh.tmem;
    // descriptors move on by 16-byte units of the address
    const uint64_t q_desc = operand_at(smem_of(q_at), 16), k_desc = operand_at(smem_of(stages), 16),
                   v_desc = operand_at(smem_of(stages) + C::OPERAND, TILE * 128);
    for (int i = 0; i < sh.n_segs; ++i, ++items) {
        const int halves = 2 * (sh.segs[i].u1 - sh.segs[i].u0);
        // weights of half k, then scores of half k + 2 in their place; each stands once in the code, which all roles share a cache for
#pragma unroll 1
        for (int k = -2; k < halves; ++k) {
            const int h = k & 1, now = g + (k >> 1), st = now & 1;       // (k = -2, -1: tile g - 1, which there is none of)
            if (k >= 0) {
#pragma unroll 1
                for (int t = 0; t < 2; ++t) {
                    wait(sh, &sh.p_full[t][h], now & 1, a.wait_cycles);
                    fence_after();
                    const uint64_t v = v_desc + (uint32_t)(st * (2 * C::OPERAND / 16) + h * (HALF * 128 / 16));
                    const uint32_t to = tm + 2 * TILE + t * TILE, from = tm + t * TILE + h * HALF;
#pragma unroll
                    for (int s = 0; s < HALF / 16; ++s) mma_ts(to, from + s * 8, v + (uint32_t)(s * (2048 / 16)), O_SHAPE, k > 0 || s > 0);
                    commit(&sh.pv_done[t][h]);
                }
                if (h == 1) commit(&sh.kv_empty[st]);
            }
            if (k + 2 < halves) {
                if (h == 0) wait(sh, &sh.kv_full[st ^ 1], ((now + 1) >> 1) & 1, a.wait_cycles);
#pragma unroll 1
                for (int t = 0; t < 2; ++t) {
                    if (k == -2) wait(sh, &sh.q_full[t], items & 1, a.wait_cycles);
                    if (k >= 0) wait(sh, &sh.pv_done[t][h], now & 1, a.wait_cycles);
                    fence_after();
                    const uint64_t q = q_desc + (uint32_t)(t * (C::OPERAND / 16)), kk = k_desc + (uint32_t)((st ^ 1) * (2 * C::OPERAND / 16) + h * (HALF * 128 / 16));
                    const uint32_t to = tm + t * TILE + h * HALF;
#pragma unroll
                    for (int s = 0; s < D / 16; ++s) {
                        const uint32_t in = (uint32_t)(s >> 2) * (TILE * 128 / 16) + (uint32_t)(s & 3) * 2;
                        mma_ss(to, q + in, kk + in, S_SHAPE, s > 0);
                    }
                    commit(&sh.s_full[t][h]);
                }
            }
        }
        g += halves / 2;
    }
}

// ---------------------------------------------------------------------------- softmax

// N elements of a row of out
template <int N>
__device__ __forceinline__ void put_out(unsigned short* to, bool vec, const float* v, float f, bool bad)
{
    unsigned w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const float x = bad ? __int_as_float(0x7FC00000) : v[2 * i] * f, y = bad ? __int_as_float(0x7FC00000) : v[2 * i + 1] * f;
        w[i] = qp_f32_to_bf16(x) | ((unsigned)qp_f32_to_bf16(y) << 16);
    }
    if (vec) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) *reinterpret_cast<uint2*>(to + 4 * i) = make_uint2(w[2 * i], w[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) { to[2 * i] = (unsigned short)w[i]; to[2 * i + 1] = (unsigned short)(w[i] >> 16); }
    }
}
__device__ __forceinline__ void put_lse(const qp_kv_attn_args& a, int token, int head, float m, float l, bool bad)
{
    if (a.lse)
        a.lse[(int64_t)token * a.q_heads + head] =
            bad ? __int_as_float(0x7FC00000) : l == 0.f ? -__int_as_float(0x7F800000) : (m + log2f(l)) * 0.6931471805599453f;
}

template <int D>
__device__ __forceinline__ void softmax(const qp_kv_attn_args& a, Shared& sh, char* q_at, int& g)
{
    using C = Cfg<D>;
    const int t = threadIdx.x >> 7, row = threadIdx.x & 127, lane = threadIdx.x & 31;
    const uint32_t lanes = (uint32_t)(row & ~31) << 16;
    const uint32_t s_at = sh.tmem + t * TILE + lanes, o_at = sh.tmem + 2 * TILE + t * TILE + lanes;
    const float inf = __int_as_float(0x7F800000);
    for (int i = 0; i < sh.n_segs; ++i) {
        const Seg& s = sh.segs[i];
        const int r = s.tile * ROWS + t * TILE + row, all = s.n * a.group;       // (tokens * q_heads is below 2^31 - 4096)
        const bool mine = r < all;
        // ---- the query row, scaled, into shared memory
        float kf;
        bool bad;
        {
            uint4 x[D / 8];
            const unsigned short* from = static_cast<const unsigned short*>(a.q);
            if (mine) from += (int64_t)(s.row0 + r / a.group) * a.qt + (int64_t)(s.head * a.group + r % a.group) * a.qh;
            if (!mine) {
#pragma unroll
                for (int c = 0; c < D / 8; ++c) x[c] = make_uint4(0, 0, 0, 0);
            } else if (a.vec) {
#pragma unroll
                for (int c = 0; c < D / 8; ++c) x[c] = qp_kv_ld(reinterpret_cast<const uint4*>(from) + c);
            } else {
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    unsigned w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = qp_kv_ld(from + 8 * c + 2 * e) | ((unsigned)qp_kv_ld(from + 8 * c + 2 * e + 1) << 16);
                    x[c] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            float top = 0.f;
            bool nan = false;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                const unsigned w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y0 = fabsf(__uint_as_float(w[e] << 16)), y1 = fabsf(__uint_as_float(w[e] & 0xFFFF0000u));
                    nan |= !(y0 < inf) || !(y1 < inf);
                    top = qp_max3(top, y0, y1);
                }
            }
            bad = nan;
            int ex = 265 - (int)(__float_as_uint(top) >> 23);    // the row's largest element to [2^11, 2^12)
            ex = top == 0.f || bad ? 127 : ex > 254 ? 254 : ex;
            float norm = __uint_as_float((unsigned)ex << 23);
            kf = fabsf(a.scale_log2) / norm;
            norm = bad ? 0.f : a.scale_log2 < 0.f ? -norm : norm;
            char* to = q_at + t * C::OPERAND + row * 128;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                const unsigned w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
                unsigned h[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {                    // elements e and e + 4
                    const float y0 = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
                    const float y1 = __uint_as_float(e & 1 ? w[e / 2 + 2] & 0xFFFF0000u : w[e / 2 + 2] << 16);
                    h[e] = bad ? 0u : half2_of(y0 * norm, y1 * norm);
                }
                *reinterpret_cast<uint4*>(to + (c >> 3) * (TILE * 128) + (((c & 7) ^ (row & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
            }
            fence_operands();
            arrive(&sh.q_full[t]);
        }
        // last key that the row sees; keys in front of all_hi and from all_lo on are seen by every row of the tile (a key's position
        // fits 32 bits; past the end of the range nothing is seen)
        const int row0 = s.tile * ROWS + t * TILE, last_row = row0 + TILE <= all ? row0 + TILE - 1 : all - 1;
        const int hi = (int)min((int64_t)s.pos + (mine ? r : all - 1) / a.group, (int64_t)0x7FFFFFFF);
        const int all_hi = (int)min((int64_t)s.pos + row0 / a.group, (int64_t)0x7FFFFFFE) + 1;
        const int all_lo = a.window > 0 ? (int)min((int64_t)s.pos + last_row / a.group - a.window, (int64_t)0x7FFFFFFE) + 1 : 0;
        // p = 2^(s - m) in l; O holds sums of 2^(s + P_SHIFT - X) * v.  X follows the largest s + (power of two of the tile's V), of keys that the
        // row sees, as a whole number (so that it adds to V's powers and to m without rounding): weights of 2^13 at most in fp16, and none lost that
        // counts, whatever the other rows and tiles hold.
        float m = M_NONE, X = M_NONE, l = 0.f;
        const int first_key = s.s0 * QP_KV_SLICE, u0 = s.u0, u1 = s.u1;
        for (int u = u0; u < u1; ++u, ++g) {
            const int st = g & 1;
            wait(sh, &sh.kv_full[st], (g >> 1) & 1, a.wait_cycles);      // (long there: for what the producers say of the tile)
            const int2 about = sh.about[st];
            const uint4 v4 = sh.valid[st];
            const float f = fmaxf(kf * __int_as_float(about.x), 1e-37f);         // (positive, so that -inf stays)
            const float ve = (float)about.y;
            const bool spread = sh.spread[st] != 0;
            const int key0 = first_key + u * TILE;
            const bool whole = (v4.x & v4.y & v4.z & v4.w) == 0xFFFFFFFFu && key0 >= all_lo && key0 + TILE <= all_hi;
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const int t0 = key0 + h * HALF;
                wait(sh, &sh.s_full[t][h], g & 1, a.wait_cycles);
                __syncwarp();
                fence_after();
                // which of 32 keys the row sees
                auto seen_of = [&](int c) {
                    if (whole) return 0xFFFFFFFFu;
                    const int up = hi - t0 - 32 * c, down = a.window > 0 ? hi - a.window - t0 - 32 * c : -1;   // keys (down, up]
                    unsigned seen = h ? (c ? v4.w : v4.z) : (c ? v4.y : v4.x);
                    seen &= up < 0 ? 0u : up >= 31 ? 0xFFFFFFFFu : (2u << up) - 1u;
                    return seen & (down < 0 ? 0xFFFFFFFFu : down >= 31 ? 0u : ~((2u << down) - 1u));
                };
                // rows scaled one by one (uncommon): 16 keys at a time, read again for the weights, so that this code is short
                const float *scale = sh.row_scale[st] + h * HALF, *power = sh.row_power[st] + h * HALF;
                auto piece = [&](int c, float (&y)[16], float (&pw)[16]) {
                    tmem_ld16(s_at + h * HALF + 16 * c, y);
                    const unsigned seen = seen_of(c >> 1) >> (16 * (c & 1));
                    float sc[16];
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const float4 r = *reinterpret_cast<const float4*>(scale + 16 * c + e), w = *reinterpret_cast<const float4*>(power + 16 * c + e);
                        sc[e] = r.x; sc[e + 1] = r.y; sc[e + 2] = r.z; sc[e + 3] = r.w;
                        pw[e] = w.x; pw[e + 1] = w.y; pw[e + 2] = w.z; pw[e + 3] = w.w;
                    }
                    wait_ld(y);
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[e] = seen >> e & 1u ? y[e] * sc[e] : -inf;
                };
                // new references where a score, or a score plus V's power, has passed them by too much (rare)
                auto refer = [&](float top, float most) {
                    if (__any_sync(0xFFFFFFFFu, top > m + M_SLACK || most > X + M_SLACK)) {     // rare: new references
                        const float next = fmaxf(m, top), to = fmaxf(X, floorf(most)), back = ex2(X - to);
                        l *= ex2(m - next);
                        m = next;
                        X = to;
                        if (u > u0 || h > 0) {
                            wait(sh, &sh.pv_done[t][h ^ 1], (h ? g : g - 1) & 1, a.wait_cycles);      // of the half before
                            __syncwarp();
                            fence_after();
#pragma unroll 1
                            for (int c = 0; c < D / 32; ++c) {
                                float y[32];
                                tmem_ld32(o_at + 32 * c, y);
                                wait_ld(y);
#pragma unroll
                                for (int e = 0; e < 32; ++e) y[e] *= back;
                                tmem_st32(o_at + 32 * c, y);
                            }
                            wait_st();
                        }
                    }
                };
                if (!spread) {
                    float x[HALF];
                    tmem_ld32(s_at + h * HALF, x);
                    tmem_ld32(s_at + h * HALF + 32, x + 32);
                    wait_ld(x);
                    if (!whole) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const unsigned seen = seen_of(c);
#pragma unroll
                            for (int e = 0; e < 32; ++e) x[32 * c + e] = seen >> e & 1u ? x[32 * c + e] : -inf;
                        }
                    }
                    float top4[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
                    for (int c = 4; c < HALF; c += 8)
#pragma unroll
                        for (int e = 0; e < 4; ++e) top4[e] = c + 4 + e < HALF ? qp_max3(top4[e], x[c + e], x[c + 4 + e]) : fmaxf(top4[e], x[c + e]);
                    const float top = fmaxf(qp_max3(top4[0], top4[1], top4[2]), top4[3]) * f;
                    refer(top, top + ve);
                    // (where V is so small against what O holds that its weights leave fp16, they must not leave fp32, for the sum's sake)
                    const float sub = fmaxf((float)P_SHIFT + ve - X, (float)(P_SHIFT - 90) - m);
                    const qp_f2 f2 = qp_pack2(f, f), sub2 = qp_pack2(sub, sub);
                    qp_f2 sum = qp_pack2(0.f, 0.f), sum1 = sum;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t w[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float y0, y1;
                            qp_unpack2(qp_fma2(qp_pack2(x[32 * c + 2 * e], x[32 * c + 2 * e + 1]), f2, sub2), y0, y1);
                            y0 = ex2(y0);
                            y1 = ex2(y1);
                            if (e & 1) sum1 = qp_add2(sum1, qp_pack2(y0, y1));
                            else sum = qp_add2(sum, qp_pack2(y0, y1));
                            w[e] = half2_of(y0, y1);
                        }
                        tmem_st16(s_at + h * HALF + 16 * c, w);
                    }
                    float s0, s1;
                    qp_unpack2(qp_add2(sum, sum1), s0, s1);
                    l = fmaf(s0 + s1, ex2(-m - sub), l);
                } else {
                    float top = -inf, most = -inf;
#pragma unroll 1
                    for (int c = 0; c < HALF / 16; ++c) {
                        float y[16], pw[16];
                        piece(c, y, pw);
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            top = qp_max3(top, y[e], y[e + 1]);
                            most = qp_max3(most, fmaf(y[e], f, pw[e]), fmaf(y[e + 1], f, pw[e + 1]));
                        }
                    }
                    refer(top * f, most + ve);
                    const float sub = (float)P_SHIFT + ve - X;
                    float sum = 0.f;
#pragma unroll 1
                    for (int c = 0; c < HALF / 16; ++c) {        // (a piece's weights lie over scores that were read before)
                        float y[16], pw[16];
                        uint32_t w[8];
                        piece(c, y, pw);
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            sum += ex2(fmaf(y[e], f, -m)) + ex2(fmaf(y[e + 1], f, -m));
                            w[e / 2] = half2_of(ex2(fmaf(y[e], f, pw[e]) + sub), ex2(fmaf(y[e + 1], f, pw[e + 1]) + sub));
                        }
                        tmem_st8(s_at + h * HALF + 8 * c, w);
                    }
                    l += sum;
                }
                wait_st();
                fence_before();
                arrive(&sh.p_full[t][h]);
            }
        }
        // ---- the row's result
        wait(sh, &sh.pv_done[t][1], (g - 1) & 1, a.wait_cycles);
        __syncwarp();
        fence_after();
        const bool out = mine && !given_up(sh);
        bad = bad && l != 0.f;                                   // (a row that sees nothing is 0, whatever its query)
        float* part = a.part + ((int64_t)QP_CK(s.at, 2 * gridDim.x) * 2 + t) * C::PART;
        const int token = s.row0 + r / a.group, head = s.head * a.group + r % a.group;      // (of a row that is there)
        unsigned short* to = static_cast<unsigned short*>(a.out) + (int64_t)token * a.ot + (int64_t)head * a.oh;
        const float un = ex2(X - m - (float)P_SHIFT), over = s.split ? 1.f : l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
            float y[32];
            tmem_ld32(o_at + 32 * c, y);
            wait_ld(y);
            if (out) {
#pragma unroll
                for (int e = 0; e < 32; ++e) y[e] *= un;
                float z[32];                                     // in the elements' own order
#pragma unroll
                for (int e = 0; e < 32; ++e) z[(e & ~7) + ((e & 7) >> 1) + 4 * (e & 1)] = y[e];
                if (!s.split) put_out<32>(to + 32 * c, a.out_vec, z, over, bad);
                else
#pragma unroll
                    for (int e = 0; e < 32; e += 4) __stcg(reinterpret_cast<float4*>(part + row * D + 32 * c + e), make_float4(z[e], z[e + 1], z[e + 2], z[e + 3]));
            }
        }
        if (out && !s.split) put_lse(a, token, head, m, l, bad);
        if (s.split) {
            if (out) {
                __stcg(part + TILE * D + row, bad ? __int_as_float(0x7FC00000) : m);
                __stcg(part + TILE * D + TILE + row, l);
            }
            const int parts = s.c1 - s.c0 + 1;
            __threadfence();
            group_sync(2 + t);
            if (row == 0) {
                unsigned* count = a.count + QP_CK(s.first_at * 2 + t, QP_KV_COUNTERS);
                sh.last[t] = atomicAdd(count, 1u) == (unsigned)(parts - 1);
                if (sh.last[t]) *count = 0u;
            }
            group_sync(2 + t);
            if (__all_sync(0xFFFFFFFFu, sh.last[t] != 0 && !given_up(sh))) {
                __threadfence();
                auto at = [&](int p) { return a.part + ((int64_t)QP_CK(p ? 2 * (s.c0 + p) : s.first_at, 2 * gridDim.x) * 2 + t) * C::PART; };
                const int warp_row = row & ~31, base_row = s.tile * ROWS + t * TILE;
                // a lane's row: the parts' weights, and the sum of their sums
                float best = M_NONE, sl = 0.f;
                bool nan = false;
                for (int p = 0; p < parts; ++p) {
                    const float y = __ldcg(at(p) + TILE * D + row);
                    nan |= !(y == y);
                    best = fmaxf(best, y);
                }
                for (int p = 0; p < parts; ++p) {
                    const float* x = at(p) + TILE * D + row;
                    sl = fmaf(ex2(__ldcg(x) - best), __ldcg(x + TILE), sl);
                }
                // then 16 rows at a time, four elements to a lane
                constexpr int LANES = D / 4, AT_ONCE = 16, STEP = 32 / LANES;
#pragma unroll 1
                for (int k0 = 0; k0 < 32; k0 += AT_ONCE * STEP) {
                    float4 so[AT_ONCE];
#pragma unroll
                    for (int k = 0; k < AT_ONCE; ++k) so[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                    const int mine0 = warp_row + k0 + lane / LANES, d = 4 * (lane % LANES);
                    for (int p = 0; p < parts; ++p) {
                        const float* x = at(p);
                        const float wt = ex2(__ldcg(x + TILE * D + row) - best);
#pragma unroll
                        for (int k = 0; k < AT_ONCE; ++k) {
                            const int w = mine0 + k * STEP;
                            const float4 y = base_row + w < all ? __ldcg(reinterpret_cast<const float4*>(x + w * D + d)) : make_float4(0.f, 0.f, 0.f, 0.f);
                            const float f = __shfl_sync(0xFFFFFFFFu, wt, w & 31);
                            so[k].x = fmaf(f, y.x, so[k].x); so[k].y = fmaf(f, y.y, so[k].y);
                            so[k].z = fmaf(f, y.z, so[k].z); so[k].w = fmaf(f, y.w, so[k].w);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < AT_ONCE; ++k) {
                        const int w = mine0 + k * STEP;
                        const float f = __shfl_sync(0xFFFFFFFFu, sl == 0.f ? 0.f : 1.f / sl, w & 31);
                        const int fn = __shfl_sync(0xFFFFFFFFu, (int)nan, w & 31);
                        const int64_t at_row = __shfl_sync(0xFFFFFFFFu, (int64_t)token * a.ot + (int64_t)head * a.oh, w & 31);
                        const float y[4] = {so[k].x, so[k].y, so[k].z, so[k].w};
                        if (base_row + w < all) put_out<4>(static_cast<unsigned short*>(a.out) + at_row + d, a.out_vec, y, f, fn != 0);
                    }
                }
                if (mine) put_lse(a, token, head, best, sl, nan);
            }
        }
        fence_before();
    }
}

__device__ __forceinline__ void block_sync() { asm volatile("bar.sync 0;" ::: "memory"); }
// behind a list of parts: whether there is another, once nobody reads this one any more
__device__ __forceinline__ bool more_parts(const Shared& sh)
{
    __syncwarp();
    const bool more = *(const volatile int*)&sh.more != 0;
    block_sync();
    return more;
}

template <int D>
__global__ void __launch_bounds__(THREADS, 1) kv_chunk_kernel(const qp_kv_attn_args a)
{
    using C = Cfg<D>;
    extern __shared__ char raw[];
    qp_kv_begin();
    __shared__ Shared sh;
    char* smem = raw + ((1024u - (smem_of(raw) & 1023u)) & 1023u);
    char* stages = smem + 2 * C::OPERAND;
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    // ---- the work, and this block's run of it (every warp for itself)
    int64_t W = 0;
    for (int b = lane; b < a.rows.batch; b += 32) W += work_of(a, seq_of(a, b)) * a.heads;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) W += __shfl_xor_sync(0xFFFFFFFFu, W, o);
    int64_t blocks = W / (MIN_RUN + HEAD);
    blocks = blocks < 1 ? 1 : blocks < (int64_t)gridDim.x ? blocks : (int64_t)gridDim.x;
    if (W == 0 || (int64_t)blockIdx.x >= blocks) return;
    const int64_t begin = blockIdx.x * W / blocks, end = (blockIdx.x + 1ll) * W / blocks;

    if (threadIdx.x == 0) {
        for (int t = 0; t < 2; ++t) {
            qp_stream::mbar_init(&sh.q_full[t], 4);
            qp_stream::mbar_init(&sh.kv_full[t], 4);
            qp_stream::mbar_init(&sh.kv_empty[t], 1);
            for (int h = 0; h < 2; ++h) {
                qp_stream::mbar_init(&sh.s_full[t][h], 1);
                qp_stream::mbar_init(&sh.p_full[t][h], 4);
                qp_stream::mbar_init(&sh.pv_done[t][h], 1);
            }
        }
        qp_stream::mbar_init(&sh.all_done, 1);
        sh.give_up = a.wait_cycles <= 0 ? 1u : 0u;               // (a limit of nothing has run out: test only)
        qp_stream::fence_barrier_init();
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_of(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    int64_t u = begin, base = 0;
    int b = 0;
    if (warp == 0) {                                             // the sequence that the run begins in
        for (int64_t front = 0; ; b += 32) {
            const int64_t mine = b + lane < a.rows.batch ? work_of(a, seq_of(a, b + lane)) * a.heads : 0;
            int64_t x = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t y = __shfl_up_sync(0xFFFFFFFFu, x, o);
                if (lane >= o) x += y;
            }
            const unsigned hit = __ballot_sync(0xFFFFFFFFu, begin >= front + x - mine && begin < front + x);
            if (hit) {
                const int at = __ffs(hit) - 1;
                base = front + __shfl_sync(0xFFFFFFFFu, x - mine, at);
                b += at;
                break;
            }
            front += __shfl_sync(0xFFFFFFFFu, x, 31);
            if (b + 32 >= a.rows.batch) break;                   // (never: begin < W)
        }
    }
    fence_before();
    __syncthreads();
    fence_after();

    // Registers by role: 2 * 128 * 160 + 128 * 128 + 128 * 64 are the block's 512 * 128.  (A loop for each role, so that each
    // is compiled for its own number.)
    int g = 0;
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
        do {
            if (warp == 0) list_parts(a, sh, u, end, begin, W, blocks, b, base);
            block_sync();
            softmax<D>(a, sh, smem, g);
        } while (more_parts(sh));
    } else if (warp < 12) {
        do {
            block_sync();
            produce<D>(a, sh, stages, g);
        } while (more_parts(sh));
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        int items = 0;
        do {
            block_sync();
            if (warp == 12) multiply<D>(a, sh, smem, stages, g, items);
        } while (more_parts(sh));
    }
    // all products have to be done before tensor memory goes back
    if (warp == 12) {
        commit(&sh.all_done);
        for (long long since = clock64(); !qp_stream::mbar_try_wait(&sh.all_done, 0u) && clock64() - since < QP_STREAM_TIMEOUT_CYCLES;) {}
    }
    if (threadIdx.x == 0 && given_up(sh)) atomicOr(a.status, QP_DEV_STREAM_TIMEOUT);
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(sh.tmem) : "memory");
}

}  // namespace

uint64_t qp_kv_chunk_part_bytes(int head_dim, int sm_count)
{
    return head_dim <= 128 ? (uint64_t)sm_count * 2 * 2 * TILE * (uint64_t)(head_dim + 2) * 4 : 0;
}

int32_t qp_kv_chunk_launch(qp_ctx* ctx, const qp_kv_attn_args& a, int head_dim, cudaStream_t s)
{
    static bool ready[2][QP_KV_MAX_DEVICES];
    void (*f)(const qp_kv_attn_args) = head_dim == 64 ? kv_chunk_kernel<64> : kv_chunk_kernel<128>;
    const int smem = head_dim == 64 ? Cfg<64>::SMEM : Cfg<128>::SMEM;
    bool* done = ctx->device < QP_KV_MAX_DEVICES ? &ready[head_dim == 128][ctx->device] : nullptr;
    if (!done || !*done) {
        if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
            return qp_check_launch(ctx, "qp_kv_attention (shared memory)");
        if (done) *done = true;
    }
    qp_kv_launch(f, (unsigned)ctx->sm_count, THREADS, (size_t)smem, s, a);
    ctx->launches += 1;
    return qp_check_launch(ctx, "qp_kv_attention");
}
