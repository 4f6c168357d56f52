"""The 4-bit cache of keys and values: rows in and out, attention, pages, and a run of them together."""
import ctypes as C

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2211_04515_b200 as qp

BF16, F32 = torch.bfloat16, torch.float32


# ------------------------------------------------------------------------------------------------ without a GPU

@pytest.fixture(scope="module")
def lib():
    from paper_2211_04515_b200 import build
    build.build()
    return qp.load()


def test_sizes(lib):
    assert [qp.qp_kv_slice_bytes(d) for d in (64, 128, 256)] == [16 * (d + 16) for d in (64, 128, 256)]
    assert [qp.qp_kv_slice_bytes(d) for d in (0, -64, 32, 96, 512)] == [0] * 5
    assert lib.qp_kv_work_ints(10, 3) == 64 + 30 + 9 and lib.qp_kv_work_ints(0, 3) == 0 and lib.qp_kv_work_ints(5, -1) == 0
    b = qp.binding
    assert [C.sizeof(t) for t in (b.KVCacheDesc, b.KVBatchDesc, b.KVAttentionDesc)] == [80, 40, 32]


def test_no_context_is_an_error(lib):
    b = qp.binding
    c, t, p = b.KVCacheDesc(), b.KVBatchDesc(), b.KVAttentionDesc()
    assert lib.qp_kv_extend(None, C.byref(c), C.byref(t), None) == qp.QP_ERR_INVALID_ARG
    assert lib.qp_kv_append(None, C.byref(c), C.byref(t), 0, None, None, 0, 0, 0, 0, 0, None) == qp.QP_ERR_INVALID_ARG
    assert lib.qp_kv_gather(None, C.byref(c), C.byref(t), 0, None, None, 0, 0, 0, 0, 0, None) == qp.QP_ERR_INVALID_ARG
    assert lib.qp_kv_attention(None, C.byref(c), C.byref(t), C.byref(p), 0, None, 0, 0, 0, None, 0, 0, None, None) == qp.QP_ERR_INVALID_ARG
    assert lib.qp_kv_attention_work_bytes(None, C.byref(c)) == 0
    for f in (lib.qp_kv_fork, lib.qp_kv_copy_pages):
        assert f(None, C.byref(c), None, None, 1, None) == qp.QP_ERR_INVALID_ARG
    assert lib.qp_kv_free(None, C.byref(c), None, 1, None) == qp.QP_ERR_INVALID_ARG
    assert lib.qp_kv_compact(None, C.byref(c), None, None) == qp.QP_ERR_INVALID_ARG


def test_python_refuses_what_is_not_a_cache(lib):
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(qp.QuantPipeError):
        qp.KVCache(torch.zeros(1, 2, 1, 1, 1280, dtype=torch.uint8), i.view(2, 2), i[:2], i[:2], 64)    # not on a GPU
    with pytest.raises(qp.QuantPipeError):
        qp.KVCache(torch.zeros(1, 2, 1, 1, 1280, dtype=torch.uint8), i.view(2, 2), i[:2], i[:2], 80)
    with pytest.raises(qp.QuantPipeError):
        qp.KVBatch(i)
    for bad in (dict(head_dim=96), dict(page_size=24), dict(pages=0), dict(page_size=0)):
        with pytest.raises(qp.QuantPipeError):
            qp.KVCache.empty(**(dict(pages=4, heads=1, head_dim=64, slots=2, max_pages=2) | bad))


def test_reference_rows():
    """The reference against hand-made rows: ties, a constant row, infinities, ranges beyond fp32."""
    x = np.arange(16, dtype=np.float32)
    assert ref.quantize_row(x)[0].tolist() == list(range(16))
    c, lo, s = ref.quantize_row([3.0] * 8)
    assert c.tolist() == [0] * 8 and lo == 3 and s == 0
    c, lo, s = ref.quantize_row([np.nan, np.inf, -np.inf, 0, 15] + [0] * 3)
    assert c.tolist() == [0, 15, 0, 0, 15, 0, 0, 0] and lo == 0 and s == 1
    c, lo, s = ref.quantize_row(np.array([-3e38, 3e38, 0, 0], np.float32))
    assert c.tolist()[:2] == [0, 15] and c[2] in (7, 8)
    assert ref.quantize_row(np.array([0, 1e-39], np.float32))[2] == 0
    assert ref.quantize_row([np.nan] * 4)[1] == 0


def test_reference_book():
    b = ref.Book(6, 4, 4, 16)
    assert b.extend([0, 1, 0, 9], [17, 16, 1, 1]) == ([0, 0, -1, -1], True, False)
    assert b.table[0][:2] == [0, 1] and b.table[1][0] == 2
    assert b.fork([0, 1, 0], [2, 3, 2]) == ([(1, 3)], True, False)
    assert b.refs == [2, 1, 2, 1, 0, 0] and b.lens == [17, 16, 17, 16]
    assert b.extend([0], [50]) == ([-1], True, False)
    assert b.extend([0, 1], [40, 20]) == ([-1, -1], False, True)
    assert not b.free([0, 0])
    assert b.refs == [1, 0, 2, 1, 0, 0]
    assert b.compact() == ([(3, 1)], 3) and b.table[2][:2] == [0, 1]
    assert b.copies([0, 1, 4, 5, 4], [3, 4, 3, 5, 9]) == ([(0, 3), (1, 4), (5, 5)], True)


# ------------------------------------------------------------------------------------------------ on a GPU

@pytest.fixture(scope="module")
def ctx(lib):
    c = qp.Context(0)
    yield c
    c.close()


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def make(rng, lens, heads, dim, page, layers=1, spare=2, max_pages=None, slots=None):
    """A cache whose slots 0 .. hold `lens` tokens on pages of a random order; every byte of the pool is random, quantizers
    included (NaN and infinities among them): rows that were never written may hold anything."""
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    max_pages = max_pages or max(need + [1]) + 1
    slots = slots or len(lens)
    cache = qp.KVCache.empty(pages, heads, dim, slots, max_pages, page, layers)
    cache.pool.copy_(torch.from_numpy(rng.integers(0, 256, cache.pool.shape, dtype=np.uint8)))
    order = rng.permutation(pages)
    table = np.full((slots, max_pages), -1, np.int32)
    refs = np.zeros(pages, np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        refs[order[at:at + n]] = 1
        at += n
    cache.table.copy_(torch.from_numpy(table))
    cache.refs.copy_(torch.from_numpy(refs))
    cache.lens.copy_(ints(list(lens) + [0] * (slots - len(lens))))
    return cache


def fill(ctx, rng, cache, lens, layer=0, dtype=F32):
    """Writes keys and values of every token of slots 0 .. through the library; returns them."""
    start = np.concatenate(([0], np.cumsum(lens)))
    total = int(start[-1])
    shape = (max(total, 1), cache.heads, cache.head_dim)
    k = torch.from_numpy((rng.standard_normal(shape) * 1.3 + 0.4).astype(np.float32)).cuda().to(dtype)
    v = torch.from_numpy((rng.standard_normal(shape) * rng.uniform(0.05, 3, (shape[0], 1, 1))).astype(np.float32)).cuda().to(dtype)
    batch = qp.KVBatch(ints([0] * len(lens)), start=ints(start), tokens=total, max_new=max(list(lens) + [1]))
    ctx.qp_kv_append(cache, batch, k, v, layer)
    return k, v


def strided(t, how):
    """A tensor of t's values: contiguous, with heads outermost, or cut out of a wider one at an odd offset."""
    if how == "heads_first":
        return t.transpose(0, 1).contiguous().transpose(0, 1)
    if how == "odd":
        wide = torch.zeros(t.shape[0], t.shape[1], t.shape[2] + 3, dtype=t.dtype, device=t.device)
        wide[..., 1:-2] = t
        return wide[..., 1:-2]
    return t.contiguous()


@pytest.mark.gpu
@pytest.mark.parametrize("dim,dtype,page,how", [(64, F32, 16, "plain"), (64, BF16, 48, "odd"), (128, BF16, 64, "plain"),
                                                (128, F32, 32, "heads_first"), (256, BF16, 16, "heads_first"),
                                                (256, F32, 128, "odd"), (128, BF16, 1024, "heads_first")])
def test_append_and_gather(ctx, dim, dtype, page, how):
    rng = np.random.default_rng(dim + page)
    heads, layers, lens = 3, 2, [0, 1, 15, 16, 17, 70, 131]
    pos = [0, 0, 9, 16, 3, 0, 130]                                  # of the first new token
    new = [n - p for n, p in zip(lens, pos)]
    cache = make(rng, lens, heads, dim, page, layers)
    before = cache.pool.cpu().numpy().copy()
    start = np.concatenate(([0], np.cumsum(new)))
    total = int(start[-1])
    x = rng.standard_normal((2, total + 2, heads, dim)).astype(np.float32) * 2 + 0.3
    x[0, 1, 0, :] = 1.25                                            # constant
    x[0, 2, 1, 5:9] = [np.nan, np.inf, -np.inf, 4.0]
    x[1, 3, 2, :] = np.nan
    x[0, 4, 0, :2] = [3e38, -3e38]
    x[1, 5, 1, :] = 0
    x[1, 5, 1, 3] = 1e-39
    k, v = (strided(torch.from_numpy(t).cuda().to(dtype), how) for t in x)
    batch = qp.KVBatch(ints(pos), start=ints(start), tokens=total, max_new=max(new))
    ctx.qp_kv_append(cache, batch, k, v, layer=1)
    after = cache.pool.cpu().numpy()
    want = before.copy()
    xk, xv = k.float().cpu().numpy(), v.float().cpu().numpy()
    table = cache.table.cpu().numpy()
    for s in range(len(lens)):
        for i in range(new[s]):
            p, row = pos[s] + i, int(start[s]) + i
            for h in range(heads):
                sl = want[1, table[s, p // page], h, p % page // 16]
                for at, r in ((0, xk[row, h]), (8 * dim + 128, xv[row, h])):
                    c, lo, scale = ref.quantize_row(r)
                    o = at + p % 16 * (dim // 2)
                    sl[o:o + dim // 2] = ref.pack_row(c)
                    sl[at + 8 * dim + p % 16 * 8:][:8] = np.array([lo, scale], np.float32).view(np.uint8)
    # (a zero may carry either sign: compared as numbers)
    assert np.array_equal(after[0], want[0])
    for got, exp in zip(ref.parts(after[1], dim), ref.parts(want[1], dim)):
        if got.shape[-1] == 8:
            got, exp = got.view(np.uint32).copy(), exp.view(np.uint32).copy()
            got[got == 0x80000000] = 0
            exp[exp == 0x80000000] = 0
        assert np.array_equal(got, exp)
    assert ctx.qp_get_status() == 0
    # back again, in both types; rows behind the last sequence stay
    for out_dtype in (F32, BF16):
        ko, vo = (strided(torch.full((total + 2, heads, dim), 7.0, dtype=out_dtype, device="cuda"), how) for _ in range(2))
        ctx.qp_kv_gather(cache, batch, ko, vo, layer=1)
        half = torch.finfo(out_dtype).eps / 2
        for got, which in ((ko, 0), (vo, 1)):
            got = got.double().cpu().numpy()
            assert (got[total:] == 7).all()
            for s in range(len(lens)):
                for h in range(heads):
                    val = ref.sequence(after[1], table[s], h, lens[s], page, dim)[which][0][pos[s]:]
                    if val.size:
                        g = got[start[s]:start[s + 1], h]
                        big = np.abs(val) < 3.38e38                  # the end of bf16's range rounds to infinity
                        # fma rounds once to fp32 (2^-24) and the result to its type
                        assert (np.abs(g - val) <= (half + 2.0 ** -24) * np.abs(val) + 1e-45)[big].all()
    only = torch.zeros(total, heads, dim, device="cuda")
    ctx.qp_kv_gather(cache, batch, None, only, layer=1)
    kz, vz = ctx.qp_kv_gather(cache, batch, layer=1)
    assert torch.equal(only, vz) and ctx.qp_get_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dim,dtype", [(64, F32), (128, BF16), (256, BF16)])
def test_rows_are_those_of_the_token_calls(ctx, dim, dtype):
    """Codes and quantizers are bit for bit those of the token-wise calls under the min/max clip at 4 bits."""
    rng = np.random.default_rng(5)
    cache = make(rng, [160], 1, dim, 16)
    k, _ = fill(ctx, rng, cache, [160], dtype=dtype)
    d_stats = ctx.qp_stats_tokens(k, dim)
    d_qp = ctx.qp_clip_qparams_tokens_device(d_stats, 160, 4, qp.QP_CLIP_MINMAX)
    packed = ctx.qp_quantize_pack_tokens(k, dim, 4, d_qp).cpu().numpy().reshape(160, dim // 2)
    quant = d_qp.cpu().numpy().view(np.float32).reshape(160, 6)
    kc, kq, _, _ = ref.parts(cache.pool[0].cpu().numpy()[cache.table[0, :10].cpu().numpy(), 0, 0], dim)
    assert np.array_equal(kc.reshape(160, -1), packed)
    assert np.array_equal(kq.reshape(160, 8).copy().view(np.float32), quant[:, [0, 2]])


def halves(dtype, dim, rows):
    """Whether these query rows to a cached head go through the kernel that takes K and V in fp16."""
    return dtype == BF16 and dim <= 128 and rows >= 160


def check_attention(ctx, cache, lens_k, slots, pos, start, q, window, got, lse, scale, rows_left=None):
    pool, table = cache.pool[0].cpu().numpy(), cache.table.cpu().numpy()
    group = q.shape[1] // cache.heads
    qn, gn, ln = q.double().cpu().numpy(), got.double().cpu().numpy(), lse.double().cpu().numpy()
    bf = q.dtype == BF16
    worst = 0.0
    for b, s in enumerate(slots):
        if pos[b] < 0:
            continue
        n = int(start[b + 1] - start[b])
        if n == 0:
            continue
        for h in range(cache.heads):
            k, v = ref.sequence(pool, table[s], h, pos[b] + n, cache.page_size, cache.head_dim)
            u = np.arange(pos[b] + n)
            for i in range(n):
                seen = u <= pos[b] + i
                if window:
                    seen &= u > pos[b] + i - window
                for g in range(group):
                    row, hq = int(start[b]) + i, h * group + g
                    out, e, bound, lb = ref.attention_row(qn[row, hq], k, v, seen, scale, 2.0 ** -11 if bf else 2.0 ** -21,
                                                          torch.finfo(q.dtype).eps / 2, halves(q.dtype, cache.head_dim, n * group))
                    off = np.abs(gn[row, hq] - out)
                    assert (off <= bound).all(), (b, i, h, g, float((off / bound).max()))
                    worst = max(worst, float((off / bound).max()))
                    assert ln[row, hq] == e or abs(ln[row, hq] - e) <= lb
    return worst


CASES = [
    # dim, dtype, heads, group, page, lens, new, window
    (128, BF16, 2, 1, 64, [1, 2, 16, 17, 63, 64, 65, 700], 1, 0),
    (128, BF16, 2, 4, 64, [900, 3, 129, 1], 1, 0),
    (128, BF16, 1, 8, 16, [5000, 31], 1, 0),
    (128, BF16, 2, 16, 48, [333, 1, 16], 1, 0),
    (128, BF16, 1, 20, 32, [257, 65], 1, 0),
    (64, BF16, 3, 2, 16, [100, 1, 33, 2000], 1, 0),
    (64, BF16, 1, 12, 128, [513, 12], 1, 0),
    (256, BF16, 2, 3, 32, [400, 1, 90], 1, 0),
    (256, BF16, 1, 16, 64, [130], 1, 0),
    (64, F32, 2, 1, 32, [197, 1, 50], 1, 0),
    (128, F32, 2, 5, 64, [300, 16, 1200], 1, 0),
    (256, F32, 1, 8, 16, [200, 7], 1, 0),
    (128, BF16, 2, 4, 64, [40, 5, 700], 5, 0),
    (128, BF16, 1, 8, 16, [300, 64, 21], 7, 33),
    (64, F32, 2, 3, 16, [90, 11], 11, 16),
    (128, BF16, 1, 4, 32, [100, 60], 60, 0),
    (128, BF16, 2, 2, 64, [300], 130, 50),
    (128, BF16, 1, 1, 16, [600, 129], 1, 1),
    (128, BF16, 1, 1, 64, [600, 129, 20], 1, 20),
    (64, BF16, 2, 2, 64, [257], 257, 0),
    (128, BF16, 2, 4, 64, [700, 333], 300, 0),
    (128, BF16, 1, 3, 16, [411], 222, 100),
    (128, BF16, 2, 8, 32, [260, 90], 64, 0),
    (64, BF16, 1, 7, 16, [511, 333], 150, 0),
    (256, BF16, 1, 2, 64, [150], 100, 0),
    (128, F32, 1, 2, 64, [150], 100, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=str)
def test_attention(ctx, case):
    dim, dtype, heads, group, page, lens, new, window = case
    rng = np.random.default_rng(dim + page + new)
    cache = make(rng, lens, heads, dim, page)
    fill(ctx, rng, cache, lens)
    slots = rng.permutation(len(lens))
    pos = [lens[s] - min(new, lens[s]) for s in slots]
    counts = [lens[s] - p for s, p in zip(slots, pos)]
    start = np.concatenate(([0], np.cumsum(counts)))
    total = int(start[-1])
    q = torch.from_numpy(rng.standard_normal((total + 3, heads * group, dim)).astype(np.float32) * 1.7).cuda().to(dtype)
    batch = qp.KVBatch(ints(pos), slots=ints(slots), start=ints(start), tokens=total, max_new=max(counts))
    plan = ctx.qp_kv_attention_plan(cache, heads * group, window)
    out = torch.full_like(q, 5.0)
    lse = torch.full((total + 3, heads * group), 5.0, device="cuda")
    ctx.qp_kv_attention(cache, batch, q, plan, out=out, lse=lse)
    assert ctx.qp_get_status() == 0
    assert (out[total:] == 5).all() and (lse[total:] == 5).all()
    check_attention(ctx, cache, lens, slots, pos, start, q, window, out, lse, dim ** -0.5)
    again, lse2 = torch.empty_like(q), torch.empty_like(lse)
    ctx.qp_kv_attention(cache, batch, q, plan, out=again, lse=lse2)
    assert torch.equal(again[:total], out[:total]) and torch.equal(lse2[:total], lse[:total])    # the work is cut the same way: the same bits
    if max(counts) == 1:                                            # without start: row b is sequence b's
        one = qp.KVBatch(ints(pos), slots=ints(slots))
        got = ctx.qp_kv_attention(cache, one, q, plan)
        assert torch.equal(got[:total], out[:total])
    for how in ("heads_first", "odd"):
        qs, os = strided(q, how), strided(torch.zeros_like(q), how)
        ctx.qp_kv_attention(cache, batch, qs, plan, out=os)
        assert torch.equal(os[:total], out[:total])
    assert int(plan.work[:4096 * 4].count_nonzero()) == 0           # the counters are back at zero


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 80])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_of_odd_batches(ctx, dtype, new):
    """Sequences that take no part, without tokens, at position 0, on pages that the table does not name, in slots out of range."""
    rng = np.random.default_rng(3)
    lens, heads, group, dim, page = [300, 180, 90, 400, 222], 2, 4, 128, 16
    cache = make(rng, lens, heads, dim, page)
    fill(ctx, rng, cache, lens)
    table = cache.table.cpu().numpy()
    slots = [0, 1, 2, 3, 4, 99, -1]
    pos = [300 - new, -1, 0, 400 - new, 222 - new, 5, 5]
    counts = [new, new, new, 0, new, new, new]
    start = np.concatenate(([0], np.cumsum(counts)))
    total = int(start[-1])
    # a hole in slot 4: tokens 32..47 lie on no page
    cache.table[4, 2] = -1 if new == 1 else 10 ** 6
    q = torch.from_numpy(rng.standard_normal((total, heads * group, dim)).astype(np.float32)).cuda().to(dtype)
    batch = qp.KVBatch(ints(pos), slots=ints(slots), start=ints(start), tokens=total, max_new=new)
    plan = ctx.qp_kv_attention_plan(cache, heads * group)
    out, lse = torch.full_like(q, 5.0), torch.full((total, heads * group), 5.0, device="cuda")
    ctx.qp_kv_attention(cache, batch, q, plan, out=out, lse=lse)
    assert ctx.qp_get_status() == qp.QP_DEV_KV_RANGE
    cache.table[4, 2] = int(table[4, 2])
    check_attention(ctx, cache, lens, [0, 1, 2, 3], pos[:4], start[:5], q, 0, out, lse, dim ** -0.5)
    a, b = start[1], start[2]
    assert (out[a:b] == 5).all() and (lse[a:b] == 5).all()          # position -1: untouched
    for i in (5, 6):                                                # no such slot: nothing is seen
        a, b = start[i], start[i + 1]
        assert (out[a:b] == 0).all() and (lse[a:b] == -np.inf).all()
    # the hole counts as masked
    pool = cache.pool[0].cpu().numpy()
    qn, gn = q.double().cpu().numpy(), out.double().cpu().numpy()
    for h in range(heads):
        k, v = ref.sequence(pool, table[4], h, 222, page, dim)
        for i in (0, new - 1):
            seen = (np.arange(222) <= pos[4] + i) & ((np.arange(222) < 32) | (np.arange(222) >= 48))
            r, hq = int(start[4]) + i, h * group + 1
            o, e, bound, _ = ref.attention_row(qn[r, hq], k, v, seen, dim ** -0.5, 2.0 ** -11, torch.finfo(dtype).eps / 2,
                                               halves(dtype, dim, new * group))
            assert (np.abs(gn[r, hq] - o) <= bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 70])
def test_attention_of_extreme_values(ctx, new):
    """Non-finite queries poison their own rows only; large scores, tiny and huge quantizers, scales that grow along the
    sequence."""
    rng = np.random.default_rng(8)
    dim, heads, group, page, n = 128, 1, 4, 16, 500
    cache = make(rng, [n, n], heads, dim, page)
    shape = (2 * n, heads, dim)
    k = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda()
    v = torch.from_numpy((rng.standard_normal(shape) * np.tile(np.exp(np.linspace(-40, 40, n)), 2)[:, None, None]).astype(np.float32)).cuda()
    v[n:] = v[n:].flip(0)                                           # rising in slot 0, falling in slot 1
    k[:n] *= torch.linspace(0.1, 30, n, device="cuda")[:, None, None]
    start = ints([0, n, 2 * n])
    ctx.qp_kv_append(cache, qp.KVBatch(ints([0, 0]), start=start, tokens=2 * n, max_new=n), k, v)
    q = torch.from_numpy(rng.standard_normal((2 * new, group, dim)).astype(np.float32)).cuda().to(BF16)
    q[0, 1] *= 1e-30
    q[0, 2] = 0
    q[new, 3, 7] = float("nan")
    q[new, 0, 9] = float("inf")
    pos = [n - new, n - new]
    batch = qp.KVBatch(ints(pos), start=ints([0, new, 2 * new]), tokens=2 * new, max_new=new)
    plan = ctx.qp_kv_attention_plan(cache, group)
    out, lse = torch.empty_like(q), torch.empty(2 * new, group, device="cuda")
    ctx.qp_kv_attention(cache, batch, q, plan, out=out, lse=lse)
    assert out[new, [0, 3]].isnan().all() and lse[new, [0, 3]].isnan().all()
    assert not out[:new].isnan().any() and not out[new, 1:3].isnan().any() and not out[new + 1:].isnan().any()
    q[new, [0, 3]] = 0
    ctx.qp_kv_attention(cache, batch, q, plan, out=out, lse=lse)
    check_attention(ctx, cache, [n, n], [0, 1], pos, [0, new, 2 * new], q, 0, out, lse, dim ** -0.5)


@pytest.mark.gpu
def test_attention_of_a_long_sequence(ctx):
    """A few long sequences among short ones, so that the work is cut inside items; a chosen scale."""
    rng = np.random.default_rng(4)
    lens, heads, group, dim = [9, 40000, 1, 12345, 3, 17], 2, 8, 128
    cache = make(rng, lens, heads, dim, 64)
    fill(ctx, rng, cache, lens, dtype=BF16)
    q = torch.from_numpy(rng.standard_normal((6, heads * group, dim)).astype(np.float32)).cuda().to(BF16)
    pos = [n - 1 for n in lens]
    batch = qp.KVBatch(ints(pos))
    plan = ctx.qp_kv_attention_plan(cache, heads * group, scale=0.05)
    lse = torch.empty(6, heads * group, device="cuda")
    out = ctx.qp_kv_attention(cache, batch, q, plan, lse=lse)
    check_attention(ctx, cache, lens, range(6), pos, np.arange(7), q, 0, out, lse, plan.scale)


@pytest.mark.gpu
@pytest.mark.parametrize("dim,group,window", [(128, 4, 0), (64, 2, 0), (128, 3, 700)])
def test_attention_of_mixed_batches(ctx, dim, group, window):
    """Chunks of prompts, drafts and single tokens in one batch; chunks whose work is cut between many blocks."""
    rng = np.random.default_rng(12)
    lens, new, heads = [3000, 900, 64, 2000, 1, 777], [500, 1, 64, 5, 1, 130], 2
    cache = make(rng, lens, heads, dim, 32)
    fill(ctx, rng, cache, lens, dtype=BF16)
    start = np.concatenate(([0], np.cumsum(new)))
    total = int(start[-1])
    q = torch.from_numpy(rng.standard_normal((total, heads * group, dim)).astype(np.float32)).cuda().to(BF16)
    pos = [n - m for n, m in zip(lens, new)]
    batch = qp.KVBatch(ints(pos), start=ints(start), tokens=total, max_new=500)
    plan = ctx.qp_kv_attention_plan(cache, heads * group, window, scale=-0.07)
    lse = torch.empty(total, heads * group, device="cuda")
    out = ctx.qp_kv_attention(cache, batch, q, plan, lse=lse)
    assert ctx.qp_get_status() == 0
    check_attention(ctx, cache, lens, range(6), pos, start, q, window, out, lse, plan.scale)
    zero = qp.KVAttention(plan.work, heads * group, window, 0.0)     # all keys alike
    ctx.qp_kv_attention(cache, batch, q, zero, out=out, lse=lse)
    check_attention(ctx, cache, lens, range(6), pos, start, q, window, out, lse, 0.0)


@pytest.mark.gpu
def test_a_wait_that_runs_out(ctx):
    """The chunk kernel's waits are bounded: one that gives up reports it, and the context and the plan stay usable."""
    rng = np.random.default_rng(13)
    lens, heads, group, dim = [2500, 1300], 2, 4, 128
    cache = make(rng, lens, heads, dim, 16)
    fill(ctx, rng, cache, lens, dtype=BF16)
    q = torch.from_numpy(rng.standard_normal((800, heads * group, dim)).astype(np.float32)).cuda().to(BF16)
    batch = qp.KVBatch(ints([2000, 1000]), start=ints([0, 500, 800]), tokens=800, max_new=500)
    plan = ctx.qp_kv_attention_plan(cache, heads * group)
    good = ctx.qp_kv_attention(cache, batch, q, plan)
    assert ctx.qp_get_status() == 0
    ctx.qp_set_wait_limit_for_testing(tile_wait_cycles=0)
    try:
        ctx.qp_kv_attention(cache, batch, q, plan)
        with pytest.raises(qp.QuantPipeError) as e:
            ctx.qp_get_status()
        assert e.value.status == qp.QP_ERR_TIMEOUT
    finally:
        ctx.qp_set_wait_limit_for_testing()
    assert ctx.qp_get_status() == 0 and int(plan.work[:4096 * 4].count_nonzero()) == 0
    assert torch.equal(ctx.qp_kv_attention(cache, batch, q, plan), good)
    assert ctx.qp_get_status() == 0


@pytest.mark.gpu
def test_offsets_beyond_32_bits(ctx):
    """Pages and layers further than 4 GB into the pool."""
    rng = np.random.default_rng(6)
    heads, dim, page, layers = 8, 128, 64, 2
    pages = 36000                                                   # 73728 bytes each, 2.65 GB a layer
    cache = qp.KVCache.empty(pages, heads, dim, 2, 40, page, layers)
    ids = [pages - 1 - 3 * i for i in range(40)]
    cache.table[1] = ints(ids)
    n = 40 * page - 5
    k = torch.from_numpy(rng.standard_normal((n, heads, dim)).astype(np.float32)).cuda().to(BF16)
    batch = qp.KVBatch(ints([0]), slots=ints([1]), start=ints([0, n]), tokens=n, max_new=n)
    ctx.qp_kv_append(cache, batch, k, k.flip(0), layer=1)
    q = torch.from_numpy(rng.standard_normal((1, 16, dim)).astype(np.float32)).cuda().to(BF16)
    lse = torch.empty(1, 16, device="cuda")
    one = qp.KVBatch(ints([n - 1]), slots=ints([1]))
    plan = ctx.qp_kv_attention_plan(cache, 16)
    out = ctx.qp_kv_attention(cache, one, q, plan, layer=1, lse=lse)
    small = make(rng, [n], heads, dim, page)
    small.pool[0, small.table[0, :40].long()] = cache.pool[1, ids]
    check_attention(ctx, small, [n], [0], [n - 1], [0, 1], q, 0, out, lse, dim ** -0.5)
    src, dst = ints(ids[:7]), ints([5, 9, 11, 6, 30000, 1, 0])
    ctx.qp_kv_copy_pages(cache, src, dst)
    assert torch.equal(cache.pool[1, dst.long()], cache.pool[1, src.long()])
    assert ctx.qp_get_status() == 0


def same(cache, book):
    assert cache.refs.tolist() == book.refs
    assert cache.lens.tolist() == book.lens
    assert cache.table.tolist() == book.table


@pytest.mark.gpu
@pytest.mark.parametrize("pages,slots,page,heads,layers,seed", [(40, 7, 16, 1, 1, 0), (300, 33, 16, 3, 2, 1), (9000, 300, 64, 1, 1, 2),
                                                                (20000, 5000, 16, 1, 1, 3), (64, 16, 1024, 2, 3, 4)])
def test_pages_against_the_book(ctx, pages, slots, page, heads, layers, seed):
    """Random calls, good and bad ones, against the plain bookkeeping; the pool's bytes follow the pages."""
    rng = np.random.default_rng(seed)
    max_pages = max(2, min(60, 3 * pages // slots))
    cache = qp.KVCache.empty(pages, heads, 64, slots, max_pages, page, layers)
    cache.pool.random_(0, 256)
    pool = cache.pool.clone()
    book = ref.Book(pages, slots, max_pages, page)
    kinds = set()
    for step in range(60):
        kind = rng.choice(["extend", "extend", "free", "fork", "compact", "copy"])
        flags = 0
        if kind == "extend":
            n = int(rng.integers(1, slots + 1))
            ids = rng.permutation(slots)[:n].tolist()
            if step % 5 == 4:
                ids[-1] = int(rng.choice([-1, slots, ids[0]]))
            new = rng.integers(0, max(2, max_pages * page // 4), n).tolist() if step % 3 else [1] * n
            start = np.concatenate(([0], np.cumsum(new)))
            batch = qp.KVBatch(ints([7] * n), slots=ints(ids), start=ints(start), tokens=int(start[-1]), max_new=max(new))
            pos, r, x = book.extend(ids, new)
            assert ctx.qp_kv_extend(cache, batch).tolist() == pos
            flags = (qp.QP_DEV_KV_RANGE if r and not x else 0) | (qp.QP_DEV_KV_EXHAUSTED if x else 0)
            got = ctx.qp_get_status()
            assert got == flags or (x and got & ~qp.QP_DEV_KV_RANGE == flags)
            flags = None
            kinds.add((kind, x))
        elif kind == "free":
            ids = rng.integers(0, slots, max(1, slots // 3)).tolist() + ([slots] if step % 4 == 0 else [])
            flags = qp.QP_DEV_KV_RANGE if book.free(ids) else 0
            ctx.qp_kv_free(cache, ints(ids))
        elif kind == "fork":
            n = int(rng.integers(1, slots + 1))
            src = rng.integers(0, slots, n).tolist()
            empty = [s for s in range(slots) if book.lens[s] == 0]
            dst = (empty + [0, -1])[:n] if step % 2 else empty[:n]
            src = src[:len(dst)]
            moves, r, x = book.fork(src, dst)
            flags = (qp.QP_DEV_KV_RANGE if r else 0) | (qp.QP_DEV_KV_EXHAUSTED if x else 0)
            ctx.qp_kv_fork(cache, ints(src), ints(dst))
            for a, b in moves:
                pool[:, b] = pool[:, a]
            kinds.add((kind, bool(moves)))
        elif kind == "copy":
            n = int(rng.integers(0, pages // 3))
            perm = rng.permutation(pages)
            src, dst = perm[:n].tolist(), perm[n:2 * n].tolist()
            if n > 5 and step % 2:
                src[1], dst[2], dst[3], src[4], dst[4] = dst[0], dst[0], -1, 3, 3
            moves, r = book.copies(src, dst)
            flags = qp.QP_DEV_KV_RANGE if r else 0
            ctx.qp_kv_copy_pages(cache, ints(src), ints(dst))
            if moves:
                f, t = (torch.tensor(z, device="cuda") for z in zip(*moves))
                pool[:, t] = pool[:, f]
        else:
            moves, live = book.compact()
            out = ints([-1])
            ctx.qp_kv_compact(cache, out)
            assert out.item() == live
            for a, b in moves:
                pool[:, b] = pool[:, a]
            kinds.add((kind, bool(moves)))
        if flags is not None:
            assert ctx.qp_get_status() == flags, kind
        same(cache, book)
        assert torch.equal(cache.pool, pool), kind
    assert ("extend", False) in kinds and ("fork", True) in kinds and ("compact", True) in kinds


@pytest.mark.gpu
def test_exhausted_pool_changes_nothing(ctx):
    cache = qp.KVCache.empty(4, 1, 64, 5, 4, 16)
    batch = qp.KVBatch(ints([0, 0]), start=ints([0, 20, 53]), tokens=53, max_new=33)      # 2 + 3 pages
    assert ctx.qp_kv_extend(cache, batch).tolist() == [-1, -1]
    assert ctx.qp_get_status() == qp.QP_DEV_KV_EXHAUSTED
    assert cache.lens.tolist() == [0] * 5 and int(cache.refs.sum()) == 0 and (cache.table == -1).all()
    batch = qp.KVBatch(ints([0, 0]), start=ints([0, 20, 40]), tokens=40, max_new=30)
    assert ctx.qp_kv_extend(cache, batch).tolist() == [0, 0]
    ctx.qp_kv_fork(cache, ints([0, 1]), ints([2, 3]))
    assert ctx.qp_get_status() == qp.QP_DEV_KV_EXHAUSTED and cache.lens.tolist() == [20, 20, 0, 0, 0]
    # sequences longer than max_new, or beyond the rows, are refused
    batch = qp.KVBatch(ints([0, 0]), start=ints([0, 3, 4]), tokens=3, max_new=2)
    assert ctx.qp_kv_extend(cache, batch).tolist() == [-1, -1] and ctx.qp_get_status() == qp.QP_DEV_KV_RANGE


@pytest.mark.gpu
def test_sums_of_pages_beyond_31_bits(ctx):
    """17 of 33 sequences want 2^27 - 257 pages each, 2^31 + 2^27 - 4369 together, from starts that go up and down."""
    most, n = 2**27 - 257, 33
    i32 = dict(dtype=torch.int32, device="cuda:0")
    pool = torch.empty(1, 4, 1, 1, qp.qp_kv_slice_bytes(64), dtype=torch.uint8, device="cuda:0")
    cache = qp.KVCache(pool, torch.empty(n, most, **i32), torch.zeros(n, **i32), torch.zeros(4, **i32), 64)
    tokens = 16 * most
    batch = qp.KVBatch(torch.zeros(n, **i32), start=ints([0, tokens] * 17), tokens=tokens, max_new=tokens)
    assert ctx.qp_kv_extend(cache, batch).tolist() == [-1] * n
    assert ctx.qp_get_status() & qp.QP_DEV_KV_EXHAUSTED
    assert cache.lens.tolist() == [0] * n and cache.refs.tolist() == [0] * 4
    batch = qp.KVBatch(torch.zeros(n, **i32), start=ints([0] * 5 + [40] * 29), tokens=tokens, max_new=tokens)
    assert ctx.qp_kv_extend(cache, batch).tolist() == [0] * n and ctx.qp_get_status() == 0
    assert cache.lens.tolist() == [0] * 4 + [40] + [0] * 28 and cache.refs.tolist() == [1, 1, 1, 0]
    assert cache.table[4, :3].tolist() == [0, 1, 2]
    del cache
    torch.cuda.empty_cache()


def dense(ks, vs, q, dim, group):
    """Attention of q [q_heads, dim] over the fp64 rows ks, vs [heads, n, dim]."""
    out = []
    for h in range(q.shape[0]):
        s = ks[h // group] @ q[h] * dim ** -0.5
        p = torch.softmax(s, 0)
        out.append(p @ vs[h // group])
    return torch.stack(out)


def step_of(ctx, cache, batch, plan, k, v, q, out, layer=0):
    ctx.qp_kv_extend(cache, batch)
    ctx.qp_kv_append(cache, batch, k, v, layer)
    return ctx.qp_kv_attention(cache, batch, q, plan, layer, out=out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_run_of_them_together(ctx, dtype):
    """Prompts, decoding steps, a fork into samples that go apart, a sequence that ends, a compacted pool: every result against
    attention over the rows that the cache should hold, kept aside."""
    rng = np.random.default_rng(1)
    heads, group, dim, page, layers = 2, 4, 128, 16, 2
    cache = qp.KVCache.empty(64, heads, dim, 8, 12, page, layers, device=0)
    plan = ctx.qp_kv_attention_plan(cache, heads * group)
    held = {s: ([], []) for s in range(8)}                           # fp64 rows that the cache stands for (layer 1)

    def tokens(n):
        return [torch.from_numpy(rng.standard_normal((n, h, dim)).astype(np.float32)).cuda().to(dtype) for h in (heads, heads, heads * group)]

    def go(slots, new):
        start = np.concatenate(([0], np.cumsum(new)))
        batch = qp.KVBatch(ints([0] * len(slots)), slots=ints(slots), start=ints(start), tokens=int(start[-1]), max_new=max(new))
        k, v, q = tokens(int(start[-1]))
        out = step_of(ctx, cache, batch, plan, k, v, q, torch.empty_like(q), layer=1)
        for b, s in enumerate(slots):
            for i in range(new[b]):
                r = int(start[b]) + i
                for x, to in ((k, 0), (v, 1)):
                    rows = []
                    for h in range(heads):
                        c, lo, sc = ref.quantize_row(x[r, h].float().cpu().numpy())
                        rows.append(float(lo) + float(sc) * c)
                    held[s][to].append(np.stack(rows))
                ks, vs = (torch.from_numpy(np.stack(held[s][to], 1)) for to in (0, 1))
                want = dense(ks, vs, q[r].double().cpu(), dim, group)
                # weights of 11 bits and the result's own rounding (fp32: 2^-21 and sums), of values below 4.5
                tol = (2.0 ** -11 + 2.0 ** -8 if dtype == BF16 else 2.0 ** -16) * 4.5
                assert (out[r].double().cpu() - want).abs().max() <= tol

    go([0, 3, 5], [37, 16, 1])
    go([3, 0, 5], [1, 1, 1])
    ctx.qp_kv_fork(cache, ints([0, 0, 3]), ints([1, 2, 7]))
    for s, d in ((0, 1), (0, 2), (3, 7)):
        held[d] = tuple(list(x) for x in held[s])
    go([0, 1, 2, 3, 7], [1, 2, 1, 3, 1])
    ctx.qp_kv_free(cache, ints([0, 5]))
    held[0], held[5] = ([], []), ([], [])
    ctx.qp_kv_compact(cache)
    live = int((cache.refs > 0).sum())
    assert (cache.refs[:live] > 0).all()
    go([7, 1, 5, 2], [1, 1, 20, 5])
    assert ctx.qp_get_status() == 0


@pytest.mark.gpu
def test_captured_step_replays(ctx):
    """A whole decoding step in a graph, replayed: lengths grow on the device; a second plan and graph beside it on another stream
    and another cache."""
    rng = np.random.default_rng(2)
    heads, group, dim, page = 2, 8, 64, 16
    sides = []
    for side in range(2):
        c = qp.Context(0)
        lens = [50 + side, 130, 15]
        cache = make(rng, lens, heads, dim, page, spare=30, max_pages=20)
        fill(c, rng, cache, lens)
        plan = c.qp_kv_attention_plan(cache, heads * group)
        batch = qp.KVBatch(ints([0, 0, 0]))
        k, v, q = (torch.zeros(3, h, dim, device="cuda") for h in (heads, heads, heads * group))
        out = torch.empty_like(q)
        stream = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        # warmed up on a copy of the tables, which are put back
        saved = [t.clone() for t in (cache.table, cache.lens, cache.refs)]
        with torch.cuda.stream(stream):
            stream.wait_stream(torch.cuda.default_stream())
            step_of(c, cache, batch, plan, k, v, q, out)
            for t, o in zip((cache.table, cache.lens, cache.refs), saved):
                t.copy_(o)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step_of(c, cache, batch, plan, k, v, q, out)
        sides.append((c, cache, lens, plan, batch, k, v, q, out, stream, graph))
    for step in range(20):
        for c, cache, lens, plan, batch, k, v, q, out, stream, graph in sides:
            with torch.cuda.stream(stream):
                for t in (k, v, q):
                    t.copy_(torch.from_numpy(rng.standard_normal(t.shape).astype(np.float32)))
                graph.replay()
    torch.cuda.synchronize()
    for c, cache, lens, plan, batch, k, v, q, out, stream, graph in sides:
        assert cache.lens.tolist() == [n + 20 for n in lens] and batch.pos.tolist() == [n + 19 for n in lens]
        assert c.qp_get_status() == 0
        again = c.qp_kv_attention(cache, batch, q, plan, lse=(lse := torch.empty(3, heads * group, device="cuda")))
        assert torch.equal(again, out)
        check_attention(c, cache, lens, range(3), batch.pos.tolist(), np.arange(4), q, 0, out, lse, dim ** -0.5)
        del graph
    for s in sides:
        s[0].close()


@pytest.mark.gpu
@pytest.mark.parametrize("new", [3, 60])
def test_more_tokens_than_said(ctx, new):
    """Rows beyond max_new are skipped and reported; rows at and behind `tokens` are left alone whatever start says."""
    rng = np.random.default_rng(14)
    lens, heads, group, dim = [200, 130], 1, 4, 64
    cache = make(rng, lens, heads, dim, 16)
    fill(ctx, rng, cache, lens)
    q = torch.from_numpy(rng.standard_normal((2 * new + 4, group, dim)).astype(np.float32)).cuda().to(BF16)
    pos, start = [200 - new - 2, 130 - new], [0, new + 2, 2 * new + 4]
    plan = ctx.qp_kv_attention_plan(cache, group)
    out, lse = torch.full_like(q, 5.0), torch.full((2 * new + 4, group), 5.0, device="cuda")
    batch = qp.KVBatch(ints(pos), start=ints(start), tokens=2 * new + 1, max_new=new)
    ctx.qp_kv_attention(cache, batch, q, plan, out=out, lse=lse)
    assert ctx.qp_get_status() == qp.QP_DEV_KV_RANGE
    check_attention(ctx, cache, lens, [0], pos[:1], [0, new], q, 0, out, lse, dim ** -0.5)
    assert (out[new:new + 2] == 5).all() and (out[2 * new + 1:] == 5).all() and (lse[2 * new + 1:] == 5).all()
    assert (out[new + 2:2 * new + 1] != 5).any()
    ctx.qp_kv_append(cache, batch, q[:, :1].contiguous(), q[:, :1].contiguous())
    k, _ = ctx.qp_kv_gather(cache, batch, q[:, :1].contiguous() * 0 + 5, q[:, 1:2].contiguous())
    assert (k[2 * new + 1:] == 5).all() and ctx.qp_get_status() == 0


@pytest.mark.gpu
def test_calls_follow_each_other(ctx):
    """Each call is set up while the one before it runs: chains of dependent calls without a wait between, on a stream of their own, after
    and before kernels of other kinds, give what the same calls give with a wait between."""
    rng = np.random.default_rng(15)
    heads, group, dim, page = 4, 2, 128, 16
    results = []
    for waits in (True, False):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(3)
        cache = qp.KVCache.empty(400, heads, dim, 24, 30, page, 2)
        cache.pool.zero_()
        plan = ctx.qp_kv_attention_plan(cache, heads * group)
        outs = []
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        pause = stream.synchronize if waits else (lambda: None)
        with torch.cuda.stream(stream):
            for step in range(25):
                n = 8 if step % 5 else 24
                new = 40 if step == 0 else 1
                start = torch.arange(0, (n + 1) * new, new, dtype=torch.int32, device="cuda")
                batch = qp.KVBatch(torch.zeros(n, dtype=torch.int32, device="cuda"), start=start, tokens=n * new, max_new=new)
                k, v = torch.randn(2, n * new, heads, dim, device="cuda", generator=gen).to(BF16)
                q = torch.randn(n * new, heads * group, dim, device="cuda", generator=gen).to(BF16)
                ctx.qp_kv_extend(cache, batch), pause()
                for layer in range(2):
                    ctx.qp_kv_append(cache, batch, k, v + layer, layer), pause()
                    out = ctx.qp_kv_attention(cache, batch, q, plan, layer)
                    pause()
                    outs.append(out * 2)
                    q = out + q
                if step % 7 == 3:
                    ctx.qp_kv_free(cache, ints([1, 5, 20])), pause()
                    ctx.qp_kv_fork(cache, ints([0, 2, 2]), ints([1, 5, 20])), pause()
                    ctx.qp_kv_compact(cache), pause()
        stream.synchronize()
        assert ctx.qp_get_status() == 0
        results.append((outs, cache))
    for a, b in zip(*(r[0] for r in results)):
        assert torch.equal(a, b)
    a, b = (r[1] for r in results)
    assert a.lens.tolist() == b.lens.tolist() and torch.equal(a.table, b.table) and torch.equal(a.refs, b.refs)


@pytest.mark.gpu
def test_refusals(ctx):
    b = qp.binding
    rng = np.random.default_rng(0)
    cache = make(rng, [40, 3], 2, 64, 16)
    batch = qp.KVBatch(ints([0, 0]))
    plan = ctx.qp_kv_attention_plan(cache, 4)
    q, k = torch.zeros(2, 4, 64, device="cuda"), torch.zeros(2, 2, 64, device="cuda")

    def refused(status, call, *args, **more):
        with pytest.raises(qp.QuantPipeError) as e:
            call(*args, **more)
        assert e.value.status == status

    bad = qp.QP_ERR_INVALID_ARG
    refused(bad, ctx.qp_kv_append, cache, batch, k, k, 1)                       # no such layer
    refused(bad, ctx.qp_kv_append, cache, batch, k, k, -1)
    refused(bad, ctx.qp_kv_append, cache, batch, k[:1], k)                      # too few rows
    refused(bad, ctx.qp_kv_append, cache, batch, k.bfloat16(), k)
    refused(qp.QP_ERR_UNSUPPORTED_DTYPE, ctx.qp_kv_append, cache, batch, k.half(), k.half())
    refused(bad, ctx.qp_kv_append, cache, batch, q, q)                          # heads
    refused(bad, ctx.qp_kv_append, cache, batch, k.cpu(), k.cpu())
    refused(bad, ctx.qp_kv_append, cache, batch, k.transpose(1, 2).contiguous().transpose(1, 2), k)
    refused(qp.QP_ERR_UNSUPPORTED_DTYPE, ctx.qp_kv_attention, cache, batch, q.half(), plan)
    refused(bad, ctx.qp_kv_attention, cache, batch, k, plan)
    refused(bad, ctx.qp_kv_attention, cache, batch, q, plan, 3)
    refused(bad, ctx.qp_kv_attention, cache, batch, q, plan, out=q.bfloat16())
    refused(bad, ctx.qp_kv_attention, cache, batch, q, plan, lse=torch.zeros(7, device="cuda"))
    for plan_bad in (qp.KVAttention(plan.work, 4, -1, 1.0), qp.KVAttention(plan.work, 4, 0, float("nan")),
                     qp.KVAttention(plan.work, 4, 0, float("inf"))):
        refused(bad, ctx.qp_kv_attention, cache, batch, q, plan_bad)
    refused(bad, ctx.qp_kv_attention, cache, batch, torch.zeros(2, 3, 64, device="cuda"), qp.KVAttention(plan.work, 3, 0, 1.0))
    refused(qp.QP_ERR_BUFFER_TOO_SMALL, ctx.qp_kv_attention, cache, batch, q, qp.KVAttention(plan.work[:-16], 4, 0, 1.0))
    refused(bad, ctx.qp_kv_extend, cache, qp.KVBatch(ints([0, 0, 0])))          # more sequences than slots
    refused(bad, ctx.qp_kv_fork, cache, ints([0]), ints([0, 1]))
    refused(bad, ctx.qp_kv_fork, cache, ints([0, 0, 0]), ints([1, 1, 1]))
    refused(bad, ctx.qp_kv_free, cache, torch.zeros(1, dtype=torch.int64, device="cuda"))
    refused(bad, ctx.qp_kv_copy_pages, cache, ints(range(99)), ints(range(99)))
    with pytest.raises(qp.QuantPipeError):
        qp.KVBatch(ints([0]), start=ints([0, 1]))
    with pytest.raises(qp.QuantPipeError):
        qp.KVBatch(ints([0, 1]), slots=ints([0]))
    # at the C boundary
    L, h = qp.load(), ctx._h

    def raw(**change):
        d = b.KVCacheDesc.from_buffer_copy(cache._desc)
        for f, x in change.items():
            setattr(d, f, x)
        return L.qp_kv_compact(h, C.byref(d), None, None)

    for change in (dict(d_pool=None), dict(d_table=None), dict(d_lens=None), dict(d_refs=None), dict(d_work=None), dict(head_dim=96),
                   dict(page_size=8), dict(page_size=2048), dict(layers=0), dict(heads=0), dict(num_pages=0), dict(max_seqs=0),
                   dict(max_pages=0), dict(max_pages=1 << 28), dict(layers=2, layer_stride=16)):
        assert raw(**change) == bad, change
    assert raw(d_pool=cache.pool.data_ptr() + 4) == qp.QP_ERR_ALIGNMENT
    assert raw(d_refs=cache.refs.data_ptr() + 2) == qp.QP_ERR_ALIGNMENT
    assert L.qp_kv_compact(h, None, None, None) == bad
    t = b.KVBatchDesc(None, None, None, 2, 2, 1, 0)
    assert L.qp_kv_extend(h, C.byref(cache._desc), C.byref(t), None) == bad     # null d_pos
    t = b.KVBatchDesc(None, None, batch.pos.data_ptr(), -1, 2, 1, 0)
    assert L.qp_kv_extend(h, C.byref(cache._desc), C.byref(t), None) == bad
    args = (C.byref(cache._desc), C.byref(batch._desc), 0, k.data_ptr())
    assert L.qp_kv_append(h, *args, None, 0, 1, 1, 1, 1, None) == bad
    assert L.qp_kv_append(h, *args, k.data_ptr() + 2, 0, 1, 1, 1, 1, None) == qp.QP_ERR_ALIGNMENT
    assert L.qp_kv_append(h, *args, k.data_ptr(), 2, 1, 1, 1, 1, None) == qp.QP_ERR_UNSUPPORTED_DTYPE
    # nothing to do is not an error
    none = qp.KVBatch(ints([]))
    ctx.qp_kv_extend(cache, none), ctx.qp_kv_append(cache, none, k, k), ctx.qp_kv_attention(cache, none, q, plan)
    ctx.qp_kv_free(cache, ints([])), ctx.qp_kv_fork(cache, ints([]), ints([])), ctx.qp_kv_copy_pages(cache, ints([]), ints([]))
    assert ctx.qp_get_status() == 0
