"""The 4-bit cache of keys and values where it can go wrong: rows that a query does not see or gives no weight, large scores, positions
past the table, more sequences than rows, rows that no sequence writes, queries that see nothing or whose sum passes fp32, large batches,
launches that are refused, numbers past 32 bits."""
import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2211_04515_b200 as qp
from test_kv_cache import BF16, F32, check_attention, ctx, fill, halves, ints, lib, make  # noqa: F401  (fixtures among them)


def bound_of(q, k, v, seen, scale, dtype, in_halves):
    """One query over the rows that it sees, fp64: (out, bound of |error|, bound of |difference| between the results of two calls whose
    rows of K are the same).  Nothing in the bounds comes from a row of V without weight: every term is weighted by p.  k, v as
    kv_reference.sequence gives them."""
    kv, klo, ks, _ = (x[seen] for x in k)
    vv, vlo, vs, vc = (x[seen] for x in v)
    s = kv @ q * scale
    p = np.exp(s - s.max())
    l = p.sum()
    out = p @ vv / l
    n = len(s)
    # a score's error as in kv_reference.attention_row, but each row's own; it changes its weight by at most twice that share
    ds = 2.0 ** -17 * abs(scale) * np.abs(q).sum() * (np.abs(klo) + 15 * ks)
    held = np.abs(vlo) + 15 * vs                                 # magnitudes that the sums are made of
    # weights in 11 (bf16) or 22 bits; below fp16's normal numbers to 2^-25, where the largest p * vs is 2^7 or more
    eps = 2.0 ** -11 if dtype == BF16 else 2.0 ** -21
    weights = eps * (p * vs) @ vc / l + n * 15 * 2.0 ** -32 * (p * vs).max() / l
    v_off = 0.0
    if in_halves:
        # K and V in fp16: of the value 2^-11, of the middle of the row 2^-11, of the scale 2^-11 times at most 8.  A row of K has its
        # largest value at 2^-2 or above, so a subnormal's 2^-25, twice, is 2^-22 of that.
        def rounding(x, lo, scale):
            return 2.0 ** -11 * (np.abs(x) + (np.abs(lo + 8 * scale) + 8 * scale)[:, None])
        ds = ds + abs(scale) * ((rounding(kv, klo, ks) + (2.0 ** -22 * np.abs(kv).max(1))[:, None]) @ np.abs(q))
        # Weights: 2^-11, and 2^-25 below the normal numbers.  A row's own largest value stands at 2^3 or above in its tile (below 2^11), so
        # that a subnormal value's 2^-25, twice, is at most 2^-26 of it.  The weight that O's reference was taken from is 2^5 or more, so
        # the largest p * (row's largest value) stands at 2^8 or above, and 2^-25 * 2^11 is 2^-22 of that.
        most = np.abs(vv).max(1)
        small = p @ np.repeat((2.0 ** -26 * most)[:, None], vv.shape[1], 1) / l
        weights = 2.0 ** -11 * p @ np.abs(vv) / l + n * 2.0 ** -22 * (p * most).max() / l + small
        v_off = p @ rounding(vv, vlo, vs) / l
    # exp2 2^-21 and its argument 2^-20, fp32 sums n / 8 steps; the matrix unit drops leading zeros of a subnormal code (bf16): 2^-16
    each = 2.0 ** -19 + (n / 8 + 16) * 2.0 ** -24 + (2.0 ** -16 if dtype == BF16 else 0)

    def moved(by):                                               # weights off by these shares
        return p @ (by * held) / l + (p @ by / l) * (p @ held / l)
    same = moved(np.full(n, each)) + weights
    err = same + moved(2 * ds) + v_off
    half = torch.finfo(dtype).eps / 2
    return out, err + half * (np.abs(out) + err), 2 * (same + half * (np.abs(out) + err))


def test_a_refused_launch_is_the_last(tmp_path):
    """A page call whose deciding launch is refused returns the error and starts no move: shown over a runtime of the test's own."""
    import os
    import subprocess
    from paper_2211_04515_b200 import build
    nvcc = build._nvcc()
    obj, out = str(tmp_path / "pages.o"), str(tmp_path / "refused")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    subprocess.run([nvcc, "-c", *build.NVCC_FLAGS[1:], "-I", build.INCLUDE, "-I", build.CSRC, "-o", obj,
                    os.path.join(build.CSRC, "qp_kv_pages.cu")], check=True)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-I", build.INCLUDE, "-I", build.CSRC, "-I", cuda, "-o", out,
                    os.path.join(build.ROOT, "tests", "c_abi", "kv_refused_launch.cpp"), obj], check=True)
    run = subprocess.run([out], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0 and run.stdout.strip() == "ok", run.stderr


def test_every_registered_unit_has_index_checks():
    """The header promises checked indexes in the debug build of every unit that registers for them."""
    import glob
    import os
    from paper_2211_04515_b200 import build
    units = {os.path.basename(p): open(p).read() for p in glob.glob(os.path.join(build.CSRC, "*.cu"))}
    registered = [n for n, text in units.items() if "\nQP_CK_UNIT" in text]
    assert [n for n in units if n.startswith("qp_kv_") and n not in registered] == []
    assert [n for n in registered if "QP_CK(" not in units[n]] == []


def test_numbers_past_32_bits_are_refused_on_the_host(lib):
    work = torch.zeros(16, dtype=torch.uint8)
    for more in (2**31, 2**32, 2**32 + 7, -2**31 - 1):
        for q_heads, window in ((4, more), (more, 0)):
            with pytest.raises(qp.QuantPipeError):
                qp.KVAttention(work, q_heads, window, 1.0)
    assert qp.KVAttention(work, 4, 2**31 - 1, 1.0)._desc.window == 2**31 - 1


OUTLIERS = [
    # dim, dtype, group, new, window
    (128, BF16, 4, 1, 0), (128, F32, 4, 1, 0), (64, F32, 1, 1, 0), (256, BF16, 2, 1, 0), (256, F32, 3, 4, 0),
    (128, BF16, 8, 1, 700), (64, F32, 2, 3, 700), (128, BF16, 4, 9, 0), (64, BF16, 16, 2, 300), (128, F32, 4, 9, 500),
    (128, BF16, 4, 80, 0), (64, BF16, 2, 100, 0), (128, BF16, 3, 150, 650), (64, BF16, 4, 300, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("octaves", [12, 24, 60])
@pytest.mark.parametrize("case", OUTLIERS, ids=str)
def test_values_without_weight(ctx, case, octaves):
    """Rows of V that are 2^octaves times as large as the others but are masked for a query, lie in front of its window or have no
    weight: they leave no trace in its result."""
    dim, dtype, group, new, window = case
    rng = np.random.default_rng(dim + new + octaves)
    n, page = 1999, 32
    cache = make(rng, [n], 1, dim, page)
    base = rng.standard_normal(dim)
    base *= dim ** 0.5 / np.linalg.norm(base)
    k = rng.standard_normal((n, 1, dim)) * 0.7
    v = rng.standard_normal((n, 1, dim)) * rng.uniform(0.3, 1.5, (n, 1, 1))
    big = [5, 700, n - new - 1]                                     # without weight
    k[big] = -8 * base                                              # 8 * sqrt(dim) below, in nats
    later = [n - 1] + ([n - new // 2] if new > 2 else [])           # masked for the rows in front of them
    k[later] = -8 * base
    before = [n - new - window - 1, n - new - window - 5] if window else []    # seen by nobody, in slices that are read
    v[40] = 0                                                       # a row of zeros, and one much smaller than the others
    v[41] *= 2.0 ** -30
    k = torch.from_numpy(k.astype(np.float32)).cuda()
    q = torch.from_numpy((base + 1.2 * rng.standard_normal((new, group, dim))).astype(np.float32)).cuda().to(dtype)
    batch = qp.KVBatch(ints([n - new]), start=ints([0, new]), tokens=new, max_new=new)
    plan = ctx.qp_kv_attention_plan(cache, group, window)
    got, rows = [], []
    for times in (1.0, 2.0 ** octaves):
        v[big + later + before] *= times
        ctx.qp_kv_append(cache, qp.KVBatch(ints([0]), start=ints([0, n]), tokens=n, max_new=n), k, torch.from_numpy(v.astype(np.float32)).cuda())
        got.append(ctx.qp_kv_attention(cache, batch, q, plan, out=torch.empty_like(q)).double().cpu().numpy())
        rows.append(ref.sequence(cache.pool[0].cpu().numpy(), cache.table[0].cpu().numpy(), 0, n, page, dim))
    assert ctx.qp_get_status() == 0
    qn = q.double().cpu().numpy()
    u = np.arange(n)
    for i in range(new):
        t = n - new + i
        seen = (u <= t) & ((u > t - window) if window else True)
        for g in range(group):
            wants = [bound_of(qn[i, g], *r, seen, dim ** -0.5, dtype, halves(dtype, dim, new * group)) for r in rows]
            apart = np.abs(got[1][i, g] - got[0][i, g])
            limit = np.abs(wants[1][0] - wants[0][0]) + np.maximum(wants[0][2], wants[1][2])
            assert (apart <= limit).all(), (i, g, float((apart / limit).max()), float(apart.max()), float(np.abs(wants[0][0]).max()))
            for have, (want, bound, _) in zip(got, wants):
                off = np.abs(have[i, g] - want)
                assert (off <= bound).all(), (i, g, float((off / bound).max()), float(off.max()), float(np.abs(want).max()))


@pytest.mark.gpu
@pytest.mark.parametrize("octaves", [12, 24, 60, 100])
@pytest.mark.parametrize("case", OUTLIERS, ids=str)
def test_keys_without_weight(ctx, case, octaves):
    """The same with rows of K: 2^octaves times as large as the others, masked, in front of the window or far below the other scores."""
    dim, dtype, group, new, window = case
    rng = np.random.default_rng(dim + new + octaves + 1)
    n, page = 1999, 32
    cache = make(rng, [n], 1, dim, page)
    base = rng.standard_normal(dim)
    base *= dim ** 0.5 / np.linalg.norm(base)
    k = rng.standard_normal((n, 1, dim)) * 0.7
    v = torch.from_numpy((rng.standard_normal((n, 1, dim)) * rng.uniform(0.3, 1.5, (n, 1, 1))).astype(np.float32)).cuda()
    large = [5, 700, n - new - 1, n - 1] + ([n - new // 2] if new > 2 else [])
    large += [n - new - window - 1, n - new - window - 5] if window else []
    k[large] = -8 * base                                            # 8 * sqrt(dim) below, in nats
    k[40] = 0
    k[41] *= 2.0 ** -30
    q = torch.from_numpy((base + 1.2 * rng.standard_normal((new, group, dim))).astype(np.float32)).cuda().to(dtype)
    batch = qp.KVBatch(ints([n - new]), start=ints([0, new]), tokens=new, max_new=new)
    plan = ctx.qp_kv_attention_plan(cache, group, window)
    got, rows = [], []
    for times in (1.0, 2.0 ** octaves):
        k[large] *= times
        ctx.qp_kv_append(cache, qp.KVBatch(ints([0]), start=ints([0, n]), tokens=n, max_new=n), torch.from_numpy(k.astype(np.float32)).cuda(), v)
        got.append(ctx.qp_kv_attention(cache, batch, q, plan, out=torch.empty_like(q)).double().cpu().numpy())
        rows.append(ref.sequence(cache.pool[0].cpu().numpy(), cache.table[0].cpu().numpy(), 0, n, page, dim))
    assert ctx.qp_get_status() == 0
    qn = q.double().cpu().numpy()
    u = np.arange(n)
    for i in range(new):
        t = n - new + i
        seen = (u <= t) & ((u > t - window) if window else True)
        for g in range(group):
            wants = [bound_of(qn[i, g], *r, seen, dim ** -0.5, dtype, halves(dtype, dim, new * group)) for r in rows]
            apart = np.abs(got[1][i, g] - got[0][i, g])
            limit = np.abs(wants[1][0] - wants[0][0]) + np.maximum(wants[0][2], wants[1][2])
            assert (apart <= limit).all(), (i, g, float((apart / limit).max()), float(apart.max()), float(np.abs(wants[0][0]).max()))
            for have, (want, bound, _) in zip(got, wants):
                off = np.abs(have[i, g] - want)
                assert (off <= bound).all(), (i, g, float((off / bound).max()), float(off.max()), float(np.abs(want).max()))


@pytest.mark.gpu
@pytest.mark.parametrize("case", OUTLIERS, ids=str)
def test_values_of_many_sizes(ctx, case):
    """Every row of V has a size of its own, 24 octaves between them, and the scores go up along the sequence or down."""
    dim, dtype, group, new, window = case
    rng = np.random.default_rng(dim + new)
    n, page = 1200, 16
    cache = make(rng, [n, n], 1, dim, page)
    base = rng.standard_normal(dim)
    base *= dim ** 0.5 / np.linalg.norm(base)
    slope = np.concatenate((np.linspace(-1.5, 1.5, n), np.linspace(1, -1, n)))[:, None, None]
    k = (rng.standard_normal((2 * n, 1, dim)) * 0.5 + slope * base).astype(np.float32)
    v = (rng.standard_normal((2 * n, 1, dim)) * 2.0 ** rng.uniform(-12, 12, (2 * n, 1, 1))).astype(np.float32)
    v[rng.integers(0, 2 * n, 200)] = 0
    ctx.qp_kv_append(cache, qp.KVBatch(ints([0, 0]), start=ints([0, n, 2 * n]), tokens=2 * n, max_new=n), *(torch.from_numpy(x).cuda() for x in (k, v)))
    q = torch.from_numpy((base + 0.8 * rng.standard_normal((2 * new, group, dim))).astype(np.float32)).cuda().to(dtype)
    batch = qp.KVBatch(ints([n - new] * 2), start=ints([0, new, 2 * new]), tokens=2 * new, max_new=new)
    out = ctx.qp_kv_attention(cache, batch, q, ctx.qp_kv_attention_plan(cache, group, window), out=torch.empty_like(q)).double().cpu().numpy()
    assert ctx.qp_get_status() == 0
    u = np.arange(n)
    for b in range(2):
        rows = ref.sequence(cache.pool[0].cpu().numpy(), cache.table[b].cpu().numpy(), 0, n, page, dim)
        for i in range(new):
            t = n - new + i
            seen = (u <= t) & ((u > t - window) if window else True)
            for g in range(group):
                want, bound, _ = bound_of(q[b * new + i, g].double().cpu().numpy(), *rows, seen, dim ** -0.5, dtype, halves(dtype, dim, new * group))
                off = np.abs(out[b * new + i, g] - want)
                assert (off <= bound).all(), (b, i, g, float((off / bound).max()), float(off.max()), float(np.abs(want).max()))


@pytest.mark.gpu
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dim,dtype,group,new", [(128, BF16, 4, 80), (64, BF16, 2, 100), (128, BF16, 4, 1), (128, F32, 2, 3)])
def test_large_scores(ctx, dim, dtype, group, new, sign):
    """Scores of 10^6 and more, whose own rounding moves the weights: where all rows of V are the same, so is the result."""
    rng = np.random.default_rng(27)
    n = 700
    cache = make(rng, [n], 1, dim, 16)
    base = rng.standard_normal(dim)
    base *= dim ** 0.5 / np.linalg.norm(base)
    k = (base * 600 + rng.standard_normal((n, 1, dim)) * 0.01).astype(np.float32) * sign
    v = np.full((n, 1, dim), -2.0, np.float32)
    ctx.qp_kv_append(cache, qp.KVBatch(ints([0]), start=ints([0, n]), tokens=n, max_new=n), *(torch.from_numpy(x.copy()).cuda() for x in (k, v)))
    q = torch.from_numpy((base * rng.uniform(180, 420, (new, group, 1))).astype(np.float32)).cuda().to(dtype)
    batch = qp.KVBatch(ints([n - new]), start=ints([0, new]), tokens=new, max_new=new)
    out = ctx.qp_kv_attention(cache, batch, q, ctx.qp_kv_attention_plan(cache, group)).double().cpu().numpy()
    assert ctx.qp_get_status() == 0
    # The same weights in O and in l: what is left are the weights' rounding (2^-11; fp32 2^-21, and 2^-21 of exp2 where references move), sums
    # of n / 8 steps and the result's own rounding.
    share = (2.0 ** -11 if dtype == BF16 else 2.0 ** -19) + (n / 8 + 16) * 2.0 ** -24
    assert (np.abs(out + 2) <= 2 * (share + torch.finfo(dtype).eps / 2 * (1 + share))).all(), float(np.abs(out + 2).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,group,new,window", [(BF16, 4, 1, 0), (F32, 2, 1, 20), (BF16, 4, 7, 0), (BF16, 8, 40, 0), (BF16, 4, 60, 50),
                                                    (F32, 1, 30, 10)])
@pytest.mark.parametrize("past", [1, 20, 300])
def test_positions_past_the_table(ctx, dtype, group, new, window, past):
    """Tokens behind the last page that the table has room for count as masked, and are reported."""
    rng = np.random.default_rng(past)
    dim, page, full = 128, 16, 416
    cache = make(rng, [full], 1, dim, page, max_pages=full // page)
    fill(ctx, rng, cache, [full])
    end = full + past                                               # behind the last query's position
    q = torch.from_numpy(rng.standard_normal((new, group, dim)).astype(np.float32)).cuda().to(dtype)
    plan = ctx.qp_kv_attention_plan(cache, group, window)
    lse = torch.empty(new, group, device="cuda")
    for pos, status in ((full - new, 0), (end - new, qp.QP_DEV_KV_RANGE)):
        batch = qp.KVBatch(ints([pos]), start=ints([0, new]), tokens=new, max_new=new)
        out = ctx.qp_kv_attention(cache, batch, q, plan, lse=lse)
        assert ctx.qp_get_status() == status
        k, v = ref.sequence(cache.pool[0].cpu().numpy(), cache.table[0].cpu().numpy(), 0, full, page, dim)
        u = np.arange(full)
        for i in range(new):
            t = pos + i
            seen = (u <= t) & ((u > t - window) if window else True)
            for g in range(group):
                if not seen.any():
                    assert (out[i, g] == 0).all() and lse[i, g] == -np.inf
                    continue
                want, bound, _ = bound_of(q[i, g].double().cpu().numpy(), k, v, seen, dim ** -0.5, dtype, halves(dtype, dim, new * group))
                assert (np.abs(out[i, g].double().cpu().numpy() - want) <= bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,group", [(BF16, 4), (F32, 2), (BF16, 160), (BF16, 16)])
def test_batches_of_more_sequences_than_rows(ctx, dtype, group):
    """Without start sequence b has row b: those at and behind `tokens` have none, and no row behind is read or written."""
    rng = np.random.default_rng(26)
    dim, lens, tokens = 64, [60, 100, 40, 70, 90, 33, 21], 3
    cache = make(rng, lens, 1, dim, 16)
    k, v = fill(ctx, rng, cache, lens)
    q = torch.from_numpy(rng.standard_normal((8, group, dim)).astype(np.float32)).cuda().to(dtype)
    pos = [n - 1 for n in lens]
    for slots in (None, ints(range(7))):
        batch = qp.KVBatch(ints(pos), slots=slots, tokens=tokens)
        plan = ctx.qp_kv_attention_plan(cache, group)
        out, lse = torch.full_like(q, 5.0), torch.full((8, group), 5.0, device="cuda")
        ctx.qp_kv_attention(cache, batch, q, plan, out=out, lse=lse)
        assert (out[tokens:] == 5).all() and (lse[tokens:] == 5).all() and ctx.qp_get_status() == 0
        check_attention(ctx, cache, lens, range(3), pos[:3], np.arange(4), q, 0, out, lse, dim ** -0.5)
        ko, vo = torch.full((8, 1, dim), 5.0, device="cuda"), torch.full((8, 1, dim), 5.0, device="cuda")
        ctx.qp_kv_gather(cache, batch, ko, vo)
        assert (ko[tokens:] == 5).all() and (vo[tokens:] == 5).all() and (ko[:tokens] != 5).any()
        before = cache.pool.clone()
        ctx.qp_kv_append(cache, batch, ko, vo)
        for s in range(tokens, 7):
            ids = cache.table[s, :-(-lens[s] // 16)].long()
            assert torch.equal(cache.pool[0, ids], before[0, ids])


def poisoned(like):
    """The next allocation of this size on this stream comes from memory full of NaN."""
    x = torch.full_like(like, float("nan"))
    torch.cuda.current_stream().synchronize()
    del x


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 50])
def test_new_output_is_zero_where_no_sequence_writes(ctx, dtype, new):
    rng = np.random.default_rng(21)
    heads, group, dim, page, lens = 2, 4, 128, 16, [100, 200, 300]
    cache = make(rng, lens, heads, dim, page)
    fill(ctx, rng, cache, lens)
    plan = ctx.qp_kv_attention_plan(cache, heads * group)
    rows = 4 * new + 9
    q = torch.from_numpy(rng.standard_normal((rows, heads * group, dim)).astype(np.float32)).cuda().to(dtype)

    def run(pos, start, tokens, max_new=new, slots=None):
        batch = qp.KVBatch(ints(pos), start=None if start is None else ints(start), tokens=tokens, max_new=max_new,
                           slots=None if slots is None else ints(slots))
        kept = ctx.qp_kv_attention(cache, batch, q, plan, out=torch.full_like(q, 5.0))
        poisoned(q)
        got = ctx.qp_kv_attention(cache, batch, q, plan)
        want = torch.where(kept == 5, torch.zeros_like(kept), kept)
        bits = torch.int16 if dtype == BF16 else torch.int32        # (NaN of rows that were never written are the same too)
        assert torch.equal(got.view(bits), want.view(bits))
        assert (kept[tokens:] == 5).all()                           # what a caller gives keeps its rows
        return kept

    n = new
    assert (run([50, 120, 200], [0, n, 2 * n, 3 * n], 3 * n)[:3 * n] != 5).all()           # nothing left out but q's last rows
    kept = run([50, -1, 200], [0, n, 2 * n, 3 * n], 3 * n)                                 # one takes no part
    assert (kept[n:2 * n] == 5).all() and (kept[2 * n:3 * n] != 5).all()
    run([-1, -1, -1], [0, n, 2 * n, 3 * n], 3 * n)                                         # nobody does
    run([50, 120, 200], [3, 3 + n, 3 + n, 3 + 2 * n], 4 * n + 9)                           # rows in front, behind, and an empty sequence
    run([50, 120], [0, n + 2, 2 * n + 4], 2 * n + 4)                                       # more tokens than max_new
    run([50, 2 ** 31 - 2], [0, n, 2 * n], 2 * n + 1)                                       # a position past 2^31 - 1 (n > 1), or past the table
    run([50, 120, 200], None, 3), run([50, -1, 200], None, 3), run([50, 120], None, 4 * n + 9)
    run([50, 120], [n, n, 0], 2 * n)                                                       # start goes down
    run([], None, 0), run([], None, 5), run([50], [0, 0], 0), run([50], [0, n], n, 0)      # nothing to do
    many = 290                                                      # more sequences than a block looks at at a time
    pos = [50 if b % 3 else -1 for b in range(many)]
    run(pos, [0] * 200 + [1] * 40 + [2 + n] * (many - 239), 2 + n, slots=[b % 3 for b in range(many)])
    ctx.qp_get_status()


@pytest.mark.gpu
def test_rows_of_an_exhausted_step_are_zero(ctx):
    heads, dim = 2, 64
    cache = qp.KVCache.empty(2, heads, dim, 3, 4, 16)
    batch = qp.KVBatch(ints([0, 0, 0]))
    plan = ctx.qp_kv_attention_plan(cache, heads)
    q = torch.randn(3, heads, dim, device="cuda").to(BF16)
    ctx.qp_kv_extend(cache, batch)
    ctx.qp_kv_append(cache, batch, q, q)
    poisoned(q)
    assert (ctx.qp_kv_attention(cache, batch, q, plan) == 0).all()
    assert ctx.qp_get_status() == qp.QP_DEV_KV_EXHAUSTED


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 80])
def test_queries_that_see_nothing(ctx, dtype, new):
    """A row that sees no key is 0 with lse -inf, whatever its query holds; one that sees a key and has a non-finite element is NaN."""
    rng = np.random.default_rng(22)
    group, dim, lens = 4, 128, [300, 90 + new]
    cache = make(rng, lens, 1, dim, 16)
    fill(ctx, rng, cache, lens)
    q = torch.from_numpy(rng.standard_normal((2 * new, group, dim)).astype(np.float32)).cuda().to(dtype)
    q[0, 1, 3] = float("nan")
    q[0, 2, 5] = float("inf")
    q[new, 0, 7] = float("nan")
    q[2 * new - 1, 3, 9] = -float("inf")
    batch = qp.KVBatch(ints([200, 90]), slots=ints([7, 1]), start=ints([0, new, 2 * new]), tokens=2 * new, max_new=new)   # there is no slot 7
    plan = ctx.qp_kv_attention_plan(cache, group)
    lse = torch.empty(2 * new, group, device="cuda")
    out = ctx.qp_kv_attention(cache, batch, q, plan, out=torch.full_like(q, 5.0), lse=lse)
    assert ctx.qp_get_status() == qp.QP_DEV_KV_RANGE
    assert (out[:new] == 0).all() and (lse[:new] == -np.inf).all()
    bad = ~q[new:].isfinite().all(-1)
    assert bad.sum() == 2 and out[new:][bad].isnan().all() and lse[new:][bad].isnan().all()
    assert out[new:][~bad].isfinite().all() and lse[new:][~bad].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,new", [(F32, 1), (BF16, 1), (BF16, 50)])
def test_queries_whose_sum_passes_fp32(ctx, dtype, new):
    """The elements are finite and so are the scores: the rows are too."""
    rng = np.random.default_rng(23)
    group, dim, n = 4, 128, 200
    cache = make(rng, [n], 1, dim, 16)
    fill(ctx, rng, cache, [n])
    q = torch.from_numpy((np.abs(rng.standard_normal((new, group, dim))) * 5e37).astype(np.float32)).cuda().to(dtype)
    scale = 1e-38
    batch = qp.KVBatch(ints([n - new]), start=ints([0, new]), tokens=new, max_new=new)
    plan = ctx.qp_kv_attention_plan(cache, group, scale=scale)
    scale = float(np.float32(scale))
    out = ctx.qp_kv_attention(cache, batch, q, plan).double().cpu().numpy()
    assert ctx.qp_get_status() == 0
    k, v = ref.sequence(cache.pool[0].cpu().numpy(), cache.table[0].cpu().numpy(), 0, n, 16, dim)
    for i in range(new):
        for g in range(group):
            want, bound, _ = bound_of(q[i, g].double().cpu().numpy(), k, v, np.arange(n) <= n - new + i, scale, dtype, halves(dtype, dim, new * group))
            assert (np.abs(out[i, g] - want) <= bound).all()


@pytest.mark.gpu
def test_refusals_of_numbers(ctx):
    """Sizes, layers and windows past 32 bits, unknown flags: an error, not the number's low bits."""
    import ctypes as C
    cache = make(np.random.default_rng(0), [40, 3], 2, 64, 16)
    pos = ints([0, 0])
    for more in (2**31, 2**32 + 2):
        for sizes in (dict(tokens=more), dict(max_new=more), dict(start=ints([0, 1, 2]), tokens=2, max_new=more)):
            with pytest.raises(qp.QuantPipeError):
                qp.KVBatch(pos, **sizes)
    batch, plan = qp.KVBatch(pos), ctx.qp_kv_attention_plan(cache, 4)
    q, k = torch.zeros(2, 4, 64, device="cuda"), torch.zeros(2, 2, 64, device="cuda")
    for call, args in ((ctx.qp_kv_append, (k, k)), (ctx.qp_kv_gather, (k, k)), (ctx.qp_kv_attention, (q, plan))):
        for layer in (1, -1, 2**32, 2**64):
            with pytest.raises(qp.QuantPipeError) as e:
                call(cache, batch, *args, layer)
            assert e.value.status == qp.QP_ERR_INVALID_ARG
    for flags in (2, -1, 1 << 30):
        d = qp.binding.KVAttentionDesc.from_buffer_copy(plan._desc)
        d.flags = flags
        assert qp.load().qp_kv_attention(ctx._h, C.byref(cache._desc), C.byref(batch._desc), C.byref(d), 0, q.data_ptr(), 0, 256, 64, q.data_ptr(),
                                         256, 64, None, None) == qp.QP_ERR_INVALID_ARG
    assert ctx.qp_get_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_of_a_large_batch(ctx, dtype):
    """More sequences than a block holds at a time (128), runs of work that cross these borders, a long sequence behind the first of them;
    sequences without tokens and ones that take no part in between."""
    rng = np.random.default_rng(24)
    heads, group, dim, page, batch_size = 12, 2, 64, 16, 300
    lens = [int(x) for x in rng.integers(1, 70, batch_size)]
    lens[205], lens[290] = 5000, 900
    cache = make(rng, lens, heads, dim, page)
    fill(ctx, rng, cache, lens)
    slots = rng.permutation(batch_size)
    counts = [int(min(lens[s], rng.choice([0, 1, 1, 1, 2, 5]))) for s in slots]
    pos = [lens[s] - c if b % 11 else -1 for b, (s, c) in enumerate(zip(slots, counts))]
    start = np.concatenate(([0], np.cumsum(counts)))
    total = int(start[-1])
    q = torch.from_numpy(rng.standard_normal((total, heads * group, dim)).astype(np.float32)).cuda().to(dtype)
    for window in (0, 100):
        batch = qp.KVBatch(ints(pos), slots=ints(slots), start=ints(start), tokens=total, max_new=5)
        plan = ctx.qp_kv_attention_plan(cache, heads * group, window)
        out, lse = torch.full_like(q, 5.0), torch.full((total, heads * group), 5.0, device="cuda")
        ctx.qp_kv_attention(cache, batch, q, plan, out=out, lse=lse)
        assert ctx.qp_get_status() == 0
        for b in range(batch_size):
            if pos[b] < 0:
                assert (out[start[b]:start[b + 1]] == 5).all()
        check_attention(ctx, cache, lens, slots, pos, start, q, window, out, lse, dim ** -0.5)
        assert int(plan.work[:4096 * 4].count_nonzero()) == 0
    # a token each, no start: rows of 300 sequences
    at = [lens[s] - 1 for s in slots]
    q1 = torch.from_numpy(rng.standard_normal((batch_size, heads * group, dim)).astype(np.float32)).cuda().to(dtype)
    plan = ctx.qp_kv_attention_plan(cache, heads * group)
    lse = torch.empty(batch_size, heads * group, device="cuda")
    out = ctx.qp_kv_attention(cache, qp.KVBatch(ints(at), slots=ints(slots)), q1, plan, lse=lse)
    check_attention(ctx, cache, lens, slots, at, np.arange(batch_size + 1), q1, 0, out, lse, dim ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128])
def test_chunks_of_a_large_batch(ctx, dim):
    """More than 32 sequences with 160 or more query rows, more parts of items to a block than its list holds (32), sequences of the other
    kernel among them."""
    rng = np.random.default_rng(25)
    heads, group, page = 120, 4, 16
    lens = [int(x) for x in rng.integers(45, 130, 46)]
    counts = [int(x) for x in rng.integers(40, 45, 46)]
    counts[3], counts[20], counts[44] = 1, 0, 7
    cache = make(rng, lens, heads, dim, page)
    fill(ctx, rng, cache, lens, dtype=BF16)
    pos = [n - c for n, c in zip(lens, counts)]
    pos[10] = -1
    start = np.concatenate(([0], np.cumsum(counts)))
    total = int(start[-1])
    q = torch.from_numpy(rng.standard_normal((total, heads * group, dim), dtype=np.float32)).cuda().to(BF16)
    batch = qp.KVBatch(ints(pos), start=ints(start), tokens=total, max_new=max(counts))
    plan = ctx.qp_kv_attention_plan(cache, heads * group)
    out, lse = torch.full_like(q, 5.0), torch.full((total, heads * group), 5.0, device="cuda")
    ctx.qp_kv_attention(cache, batch, q, plan, out=out, lse=lse)
    assert ctx.qp_get_status() == 0 and int(plan.work[:4096 * 4].count_nonzero()) == 0
    assert (out[start[10]:start[11]] == 5).all()
    pool, table = cache.pool[0].cpu().numpy(), cache.table.cpu().numpy()
    on, ln, qn = out.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
    written = np.ones(total, bool)
    written[start[10]:start[11]] = False
    assert np.isfinite(on).all() and (np.abs(on[written]).max(-1) < 5).mean() > 0.9
    for b in range(46):
        if pos[b] < 0 or counts[b] == 0:
            continue
        for _ in range(12):
            i, hq = int(rng.integers(counts[b])), int(rng.integers(heads * group))
            k, v = ref.sequence(pool, table[b], hq // group, lens[b], page, dim)
            row = int(start[b]) + i
            want, e, bound, lb = ref.attention_row(qn[row, hq], k, v, np.arange(lens[b]) <= pos[b] + i, dim ** -0.5, 2.0 ** -11, torch.finfo(BF16).eps / 2,
                                                   halves(BF16, dim, counts[b] * group))
            assert (np.abs(on[row, hq] - want) <= bound).all() and abs(ln[row, hq] - e) <= lb
