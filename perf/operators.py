"""Performance cases of the cache that keeps attention's keys and values in 4 bits.

The library sends activations between pipeline stages with one quantizer per token (a row of `head_dim` contiguous elements);
a stage that decodes keeps its keys and values the same way: every (token, head) row is 4-bit codes and one min/max
quantizer.  Measured are the operators that such a stage calls:

  append   new keys and values into the cache's pages, and the rows read back as the values that they stand for
  attend   attention of queries over the cache: single tokens, drafted tokens, chunks of a prompt
  pages    the cache's pages themselves: growing and freeing sequences, forking them, copying pages, compacting the pool

The cache's memory.  pool [layers, pages, heads, page_size / 16, 16 * (head_dim + 16)] bytes: 16 tokens of one head lie together
as K codes (16 rows of head_dim / 2 bytes, the even element in the low four bits), K quantizers (16 pairs lo, scale in fp32), V
codes, V quantizers.  table [slots, pages per sequence] int32 names a sequence's pages (-1: none), lens [slots] its tokens, refs
[pages] how many sequences hold a page (0: free).  Element d of a row is lo + scale * code.

A row's quantizer is the min/max clip at 4 bits: lo = min, scale = fp32((max - min) / 15), inv = fp32(15 / (max - min)), code =
rint(fp32(fp32(x - lo) * inv)).  These roundings are part of the format, so every form below makes the same codes.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_DEV = "cuda"
_LEVELS = 15


# ------------------------------------------------------------------------------------------------ cases

def _attend(name, dtype, batch, q_heads, heads, dim, page, shortest, longest, new, window=0):
    return {"name": name, "op": "attend", "dtype": dtype, "batch": batch, "q_heads": q_heads, "heads": heads, "dim": dim,
            "page": page, "shortest": shortest, "longest": longest, "new": new, "window": window}


def _append(name, dtype, batch, heads, dim, page, held, new):
    return {"name": name, "op": "append", "dtype": dtype, "batch": batch, "heads": heads, "dim": dim, "page": page,
            "held": held, "new": new}


def _pages(name, kind, layers, pages, heads, dim, page, slots, longest, count):
    return {"name": name, "op": "pages", "kind": kind, "layers": layers, "pages": pages, "heads": heads, "dim": dim,
            "page": page, "slots": slots, "longest": longest, "count": count}


def listed():
    return [
        # one user's next token over about a thousand: the smallest call, where latency counts
        _attend("attend_one_token", "bf16", 1, 32, 8, 128, 64, 1021, 1021, 1),
        # a serving batch's next tokens, lengths of every kind
        _attend("attend_batch_ragged", "bf16", 64, 32, 8, 128, 64, 200, 8191, 1),
        # two long documents, 16 queries to a head: few rows, a long axis
        _attend("attend_long", "bf16", 2, 64, 4, 128, 64, 120001, 131071, 1),
        # full precision at ViT-Base's head layout (12 heads of 64), a query head to each cached head
        _attend("attend_f32_vit_base", "f32", 24, 12, 12, 64, 32, 197, 1500, 1),
        # drafted tokens checked in one call, over a sliding window
        _attend("attend_drafts_window", "bf16", 16, 32, 4, 128, 16, 700, 6000, 5, 2048),
        # a chunk of a long prompt over what the cache holds of it already
        _attend("attend_prompt_chunk", "bf16", 2, 32, 8, 128, 64, 9001, 16384, 2048),
        # a serving batch's next keys and values
        _append("append_step", "bf16", 64, 8, 128, 64, 4000, 1),
        # ragged prompts of a batch
        _append("append_prompts", "bf16", 6, 8, 128, 64, 300, 4097),
        # the bookkeeping of a decoding step: every sequence grows by a token, some end
        _pages("pages_step", "step", 1, 8192, 8, 128, 64, 256, 2000, 8),
        # parallel samples of a few prompts: their full pages shared, the part-filled one copied
        _pages("pages_fork", "fork", 4, 2048, 8, 128, 64, 128, 1000, 96),
        # pages moved aside, to another place of the pool
        _pages("pages_copy", "copy", 2, 4096, 8, 128, 64, 64, 2000, 1001),
        # a pool with holes made dense, so that its end can be given back
        _pages("pages_compact", "compact", 2, 4096, 8, 128, 64, 96, 2600, 48),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attend", "attend", "attend", "append", "append", "pages", "pages"))
    dim = rng.choice((64, 128, 128, 256))
    page = rng.choice((16, 32, 64, 128))
    if op == "attend":
        heads, group = rng.choice((1, 2, 3, 4, 8, 12)), rng.choice((1, 2, 4, 5, 8, 16))
        new = rng.choice((1, 1, 1, 2, 5, _log(rng, 7, 1500)))
        batch = _log(rng, 1, 100) if new < 7 else rng.randint(1, 4)
        longest = _log(rng, max(40, new), 30000)
        while batch * heads * longest * dim > 4 * 131072 * 128 * 2 or batch * heads * group * new * longest > 2e9:
            longest = max(new, longest // 2)
            batch = max(1, batch - batch // 3)
            if longest == new and batch == 1:
                break
        return _attend("", rng.choice(("bf16", "bf16", "f32")), batch, heads * group, heads, dim, page,
                       rng.randint(min(new, longest), longest), longest, new, rng.choice((0, 0, _log(rng, 20, 5000)))) | {"name": "drawn"}
    if op == "append":
        new = rng.choice((1, 1, 3, _log(rng, 2, 4000)))
        heads = rng.choice((1, 2, 4, 8, 12))
        batch = _log(rng, 1, 200) if new < 4 else rng.randint(1, 6)
        return _append("drawn", rng.choice(("bf16", "bf16", "f32")), batch, heads, dim, page, _log(rng, 1, 5000), new)
    kind = rng.choice(("step", "fork", "copy", "compact"))
    pages = _log(rng, 300, 4000)
    slots = _log(rng, 8, min(200, pages // 8))
    longest = max(2, pages * page // (2 * slots))
    count = max(1, _log(rng, 1, slots // 2 if kind != "copy" else pages // 3))
    return _pages("drawn", kind, rng.choice((1, 2, 3)), pages, rng.choice((1, 4, 8)), min(dim, 128), page, slots, longest, count)


# ------------------------------------------------------------------------------------------------ the format, in torch

def _parts(pool, dim):
    """K codes [..., 16, dim / 2], K quantizers [..., 16, 8], V codes, V quantizers: views of the pool's bytes."""
    k = 8 * dim
    return (pool[..., :k].unflatten(-1, (16, dim // 2)), pool[..., k:k + 128].unflatten(-1, (16, 8)),
            pool[..., k + 128:2 * k + 128].unflatten(-1, (16, dim // 2)), pool[..., 2 * k + 128:].unflatten(-1, (16, 8)))


def _quantize(x):
    """Codes [..., dim / 2] and quantizers [..., 8], as bytes, of rows x [..., dim]."""
    x = x.float()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    width = hi.double() - lo.double()
    scale, inv = (width / _LEVELS).float(), (_LEVELS / width).float()
    code = torch.round((x - lo) * inv).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.cat((lo, scale), -1).contiguous().view(torch.uint8)


def _values(codes, quantizers):
    """fp32 rows [..., dim] of codes [..., dim / 2] and quantizers [..., 8]."""
    q = quantizers.contiguous().view(torch.float32)
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float()
    return code * q[..., 1:] + q[..., :1]


# ------------------------------------------------------------------------------------------------ inputs

def _fill(pool, dim, gen):
    """The pool's rows: keys with an offset per channel and some channels of larger spread, values around zero."""
    heads = pool.shape[2]
    offset = torch.randn(heads, 1, 1, dim, device=_DEV, generator=gen) * 0.7
    spread = 0.5 + torch.rand(heads, 1, 1, dim, device=_DEV, generator=gen) + 3.0 * (torch.rand(heads, 1, 1, dim, device=_DEV, generator=gen) < 0.02)
    for layer in pool:
        for some in layer.split(max(1, (1 << 26) // (layer[0].numel())), 0):
            kc, kq, vc, vq = _parts(some, dim)
            shape = (some.shape[0], heads, some.shape[2], 16, dim)
            c, q = _quantize(torch.randn(shape, device=_DEV, generator=gen) * spread + offset)
            kc.copy_(c), kq.copy_(q)
            c, q = _quantize(torch.randn(shape, device=_DEV, generator=gen) * 0.8)
            vc.copy_(c), vq.copy_(q)


def _pool(layers, pages, heads, page, dim):
    return torch.empty(layers, pages, heads, page // 16, 16 * (dim + 16), dtype=torch.uint8, device=_DEV)


def _sequences(lens, pages, page, width, gen):
    """table [slots, width] with pages of a random order, and refs: every page of a sequence is its own."""
    need = (lens + page - 1) // page
    at = torch.arange(width, device=_DEV).unsqueeze(0)
    mine = at < need.unsqueeze(1)
    order = torch.randperm(pages, device=_DEV, generator=gen)
    table = torch.full((lens.numel(), width), -1, dtype=torch.int32, device=_DEV)
    table[mine] = order[: int(need.sum())].to(torch.int32)
    refs = torch.zeros(pages, dtype=torch.int32, device=_DEV)
    refs[table[mine].long()] = 1
    return table, refs


def _spread_lens(n, shortest, longest, gen):
    """n lengths over [shortest, longest], more short ones than long, the longest among them, in a random order; their sum is
    the same for every seed."""
    u = (torch.arange(n, device=_DEV, dtype=torch.float64) + 0.5) / n
    lens = (shortest + u * u * (longest - shortest + 1)).int().clamp(max=longest)
    lens[n - 1] = longest
    return lens[torch.randperm(n, device=_DEV, generator=gen)]


_context = None


def _ctx(qp):
    """One context for the whole program."""
    global _context
    if _context is None:
        _context = qp.Context(0)
    return _context


def prepare(case, seed):
    gen = torch.Generator(device=_DEV)
    gen.manual_seed(seed)
    s = {"case": case}
    {"attend": _prepare_attend, "append": _prepare_append, "pages": _prepare_pages}[case["op"]](case, s, gen)
    if own:
        import paper_2211_04515_b200 as qp

        s["ctx"] = _ctx(qp)
        s["cache"] = qp.KVCache(s["pool"], s["table"], s["lens"], s["refs"], case["dim"])
        if "pos" in s:
            s["batch"] = qp.KVBatch(s["pos"], slots=s.get("slots"), start=s.get("start"), tokens=s["tokens"], max_new=case.get("new", 1))
        if case["op"] == "attend":
            s["plan"] = s["ctx"].qp_kv_attention_plan(s["cache"], case["q_heads"], window=case["window"])
    return s


def _starts(new):
    start = torch.zeros(new.numel() + 1, dtype=torch.int32, device=_DEV)
    start[1:] = new.cumsum(0)
    return start


def _prepare_attend(c, s, gen):
    b, page, dim = c["batch"], c["page"], c["dim"]
    lens = _spread_lens(b, c["shortest"], c["longest"], gen)
    width = -(-c["longest"] // page)
    pages = int(((lens + page - 1) // page).sum()) + 3
    s["table"], s["refs"] = _sequences(lens, pages, page, width, gen)
    s["lens"] = lens
    s["pool"] = _pool(1, pages, c["heads"], page, dim)
    _fill(s["pool"], dim, gen)
    new = torch.full((b,), c["new"], dtype=torch.int32, device=_DEV)
    s["tokens"], s["start"] = b * c["new"], None if c["new"] == 1 else _starts(new)
    s["pos"] = lens - new
    s["slots"] = torch.randperm(b, device=_DEV, generator=gen).to(torch.int32)      # the batch is in another order than the slots
    s["pos"] = s["pos"][s["slots"].long()].contiguous()
    s["q"] = (torch.randn(s["tokens"], c["q_heads"], dim, device=_DEV, generator=gen) * 1.2).to(_DTYPES[c["dtype"]])


def _prepare_append(c, s, gen):
    b, page, dim = c["batch"], c["page"], c["dim"]
    held = _spread_lens(b, 0, c["held"], gen)
    new = torch.ones(b, dtype=torch.int32, device=_DEV) if c["new"] == 1 else _spread_lens(b, 1, c["new"], gen)
    s["lens"] = held + new
    width = -(-(c["held"] + c["new"]) // page)
    pages = int(((s["lens"] + page - 1) // page).sum()) + 3
    s["table"], s["refs"] = _sequences(s["lens"], pages, page, width, gen)
    s["pool"] = _pool(1, pages, c["heads"], page, dim)
    _fill(s["pool"], dim, gen)
    s["tokens"], s["pos"], s["slots"] = int(new.sum()), held, None
    s["start"] = None if c["new"] == 1 else _starts(new)
    shape = (s["tokens"], c["heads"], dim)
    s["k"] = (torch.randn(shape, device=_DEV, generator=gen) * 1.3 + 0.2).to(_DTYPES[c["dtype"]])
    s["v"] = (torch.randn(shape, device=_DEV, generator=gen) * 0.8).to(_DTYPES[c["dtype"]])
    s["k_out"], s["v_out"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])


def _prepare_pages(c, s, gen):
    page, slots, pages = c["page"], c["slots"], c["pages"]
    width = -(-c["longest"] // page) + 1
    half = slots // 2
    lens = _spread_lens(slots, 1, c["longest"], gen)
    if c["kind"] == "fork":
        lens[half:] = 0                                       # room for the copies
    need = ((lens + page - 1) // page).cumsum(0)
    lens[need > pages - 2 * slots] = 0
    table, refs = _sequences(lens, pages, page, width, gen)
    if c["kind"] == "compact":                                # sequences that ended have left holes
        gone = torch.randperm(slots, device=_DEV, generator=gen)[: c["count"]]
        held = table[gone]
        refs[held[held >= 0].long()] = 0
        table[gone] = -1
        lens[gone] = 0
    n = c["count"]
    if c["kind"] == "fork":
        s["src"] = torch.randint(0, half, (n,), device=_DEV, generator=gen).sort().values.to(torch.int32)
        s["src"], s["dst"] = s["src"][: slots - half], torch.arange(half, slots, device=_DEV, dtype=torch.int32)[:n]
    if c["kind"] == "copy":
        at = torch.randperm(pages, device=_DEV, generator=gen).to(torch.int32)
        s["src"], s["dst"] = at[:n].contiguous(), at[n:2 * n].contiguous()
    if c["kind"] == "step":
        s["tokens"], s["pos"], s["start"], s["slots"] = slots, torch.empty(slots, dtype=torch.int32, device=_DEV), None, None
        s["gone"] = torch.randperm(slots, device=_DEV, generator=gen)[:n].to(torch.int32)
    # lens, refs and table in one buffer, and what they hold at the start: a pass begins by putting that back
    parts = [lens, refs, table.flatten()]
    s["start_meta"] = torch.cat(parts)
    s["meta"] = s["start_meta"].clone()
    s["lens"], s["refs"], t = s["meta"].split([p.numel() for p in parts])
    s["table"] = t.view(slots, width)
    s["pool"] = _pool(c["layers"], pages, c["heads"], page, c["dim"])
    if c["kind"] != "step":
        _fill(s["pool"], c["dim"], gen)


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    op = s["case"]["op"]
    if op == "attend":
        return _own_attend(s) if own else _plain_attend(s)
    if op == "append":
        return _own_append(s) if own else _plain_append(s)
    if s["case"]["kind"] != "copy":
        s["meta"].copy_(s["start_meta"])
    return _own_pages(s) if own else _plain_pages(s)


def _own_attend(s):
    return s["ctx"].qp_kv_attention(s["cache"], s["batch"], s["q"], s["plan"])


def _own_append(s):
    s["ctx"].qp_kv_append(s["cache"], s["batch"], s["k"], s["v"])
    return s["ctx"].qp_kv_gather(s["cache"], s["batch"], s["k_out"], s["v_out"])


def _own_pages(s):
    ctx, cache, kind = s["ctx"], s["cache"], s["case"]["kind"]
    if kind == "step":
        ctx.qp_kv_extend(cache, s["batch"])
        ctx.qp_kv_free(cache, s["gone"])
        return s["table"], s["lens"], s["refs"], s["pos"]
    if kind == "fork":
        ctx.qp_kv_fork(cache, s["src"], s["dst"])
    elif kind == "copy":
        ctx.qp_kv_copy_pages(cache, s["src"], s["dst"])
    else:
        ctx.qp_kv_compact(cache)
    return s["table"], s["lens"], s["refs"], s["pool"]


# ---- plain forms

def _batch_rows(s, most):
    """Row of the batch's buffers [batch, most], and whether it is one."""
    pos = s["pos"]
    start = s["start"] if s["start"] is not None else torch.arange(pos.numel() + 1, device=_DEV, dtype=torch.int32)
    i = torch.arange(most, device=_DEV)
    row = start[:-1].unsqueeze(1) + i
    return row.clamp(max=s["tokens"] - 1), row < start[1:].unsqueeze(1)


def _plain_attend(s):
    c = s["case"]
    dim, heads, new = c["dim"], c["heads"], c["new"]
    group = c["q_heads"] // heads
    pages = s["table"][s["slots"].long()].long().clamp(min=0)                    # [b, width]
    kc, kq, vc, vq = _parts(s["pool"][0], dim)

    def rows(codes, quantizers):                                               # [b, heads, tokens, dim]
        return _values(codes[pages].transpose(1, 2).flatten(2, 4), quantizers[pages].transpose(1, 2).flatten(2, 4))

    at, valid = _batch_rows(s, new)
    b = at.shape[0]
    q = s["q"][at].float().view(b, new, heads, group, dim).permute(0, 2, 3, 1, 4).reshape(b, heads, group * new, dim)
    score = (q @ rows(kc, kq).transpose(2, 3)).view(b, heads, group, new, -1) * (1.0 / math.sqrt(dim))
    key = torch.arange(score.shape[-1], device=_DEV)
    last = (s["pos"].unsqueeze(1) + torch.arange(new, device=_DEV)).unsqueeze(-1)   # [b, new, 1]
    seen = (key <= last) & valid.unsqueeze(-1)
    if c["window"]:
        seen = seen & (key > last - c["window"])
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(score - top)
    del score
    total = p.sum(-1, keepdim=True)
    o = (p.view(b, heads, group * new, -1) @ rows(vc, vq)).view(b, heads, group, new, dim) / total.clamp(min=1e-38)
    o = o.permute(0, 3, 1, 2, 4).reshape(b, new, c["q_heads"], dim).to(s["q"].dtype)
    return o.flatten(0, 1)                                                     # all of a batch's sequences have `new` rows


def _plain_places(s, most):
    """Page, slice and row of the batch's new tokens [tokens]."""
    page = s["case"]["page"]
    at, valid = _batch_rows(s, most)
    pos = (s["pos"].unsqueeze(1) + torch.arange(most, device=_DEV))[valid].long()
    slot = torch.arange(s["pos"].numel(), device=_DEV).unsqueeze(1).expand_as(valid)[valid]
    return s["table"][slot, pos // page].long(), pos % page // 16, pos % 16


def _plain_append(s):
    c = s["case"]
    p, sl, r = (t.unsqueeze(1) for t in _plain_places(s, c["new"]))
    h = torch.arange(c["heads"], device=_DEV).unsqueeze(0)
    kc, kq, vc, vq = _parts(s["pool"][0], c["dim"])
    kc[p, h, sl, r], kq[p, h, sl, r] = _quantize(s["k"])
    vc[p, h, sl, r], vq[p, h, sl, r] = _quantize(s["v"])
    s["k_out"].copy_(_values(kc[p, h, sl, r], kq[p, h, sl, r]))
    s["v_out"].copy_(_values(vc[p, h, sl, r], vq[p, h, sl, r]))
    return s["k_out"], s["v_out"]


def _free_pages(refs):
    """The pool's pages, the free ones first, each kind in its order."""
    return torch.argsort((refs != 0).int(), stable=True).to(torch.int32)


def _plain_pages(s):
    c, table, lens, refs = s["case"], s["table"], s["lens"], s["refs"]
    page, kind = c["page"], s["case"]["kind"]
    if kind == "step":
        s["pos"].copy_(lens)
        new = lens % page == 0                                                # the token opens a page
        which = (new.cumsum(0) - 1).clamp(min=0)
        take = _free_pages(refs)[which]
        slot = torch.arange(lens.numel(), device=_DEV)
        at = (lens // page).long()
        table[slot, at] = torch.where(new, take, table[slot, at])
        refs.index_add_(0, take.long(), new.int())
        lens += 1
        gone = s["gone"].long()
        held = table[gone]
        refs.index_add_(0, held.clamp(min=0).long().flatten(), -(held >= 0).int().flatten())
        table[gone] = -1
        lens[gone] = 0
        return table, lens, refs, s["pos"]
    pool = s["pool"]
    if kind == "fork":
        src, dst = s["src"].long(), s["dst"].long()
        n, rows = lens[src], table[src]
        tail = n % page != 0
        which = (tail.cumsum(0) - 1).clamp(min=0)
        take = _free_pages(refs)[which]
        at = torch.arange(table.shape[1], device=_DEV).unsqueeze(0)
        part = tail.unsqueeze(1) & (at == (n // page).unsqueeze(1))
        old = rows.gather(1, (n // page).long().unsqueeze(1).clamp(max=table.shape[1] - 1)).squeeze(1)[tail].long()
        pool[:, take[tail].long()] = pool[:, old]
        rows = torch.where(part, take.unsqueeze(1), rows)
        refs.index_add_(0, rows.clamp(min=0).long().flatten(), (rows >= 0).int().flatten())
        table[dst], lens[dst] = rows, n
    elif kind == "copy":
        pool[:, s["dst"].long()] = pool[:, s["src"].long()]
    else:
        live = refs > 0
        count = live.sum()
        at = torch.arange(refs.numel(), device=_DEV)
        hole, mover = (~live & (at < count)).nonzero().squeeze(1), (live & (at >= count)).nonzero().squeeze(1)
        pool[:, hole] = pool[:, mover]
        to = at.to(torch.int32)
        to[mover] = hole.to(torch.int32)
        refs[hole] = refs[mover]
        refs[mover] = 0
        table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], table))
    return table, lens, refs, pool


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def _row_bytes(dim):
    return dim // 2 + 8


def work(c):
    if c["op"] == "attend":
        b, mean = c["batch"], c["shortest"] + (c["longest"] - c["shortest"]) / 3
        new = c["new"]
        span = min(mean, c["window"] + new - 1) if c["window"] else mean          # tokens of the cache that are read
        seen = min(mean - (new - 1) / 2, c["window"]) if c["window"] else mean - (new - 1) / 2
        e = 4 if c["dtype"] == "f32" else 2
        return {"bytes": b * (span * c["heads"] * 2 * _row_bytes(c["dim"]) + 2 * new * c["q_heads"] * c["dim"] * e),
                "flops": 4.0 * b * c["q_heads"] * new * seen * c["dim"]}
    if c["op"] == "append":
        tokens = c["batch"] * (c["new"] if c["new"] == 1 else 1 + c["new"] / 3)
        e = 4 if c["dtype"] == "f32" else 2
        # the rows in, their codes out; the codes in again, the values out
        return {"bytes": 4.0 * tokens * c["heads"] * (c["dim"] * e + _row_bytes(c["dim"])), "flops": 12.0 * tokens * c["heads"] * c["dim"]}
    one = c["layers"] * c["heads"] * c["page"] * 2 * _row_bytes(c["dim"])          # bytes of a page
    width = -(-c["longest"] // c["page"]) + 1
    held = max(1.0, c["longest"] / 3 / c["page"])                                  # pages of a sequence
    if c["kind"] == "step":
        return {"bytes": 4.0 * (3 * c["slots"] + c["slots"] / c["page"] * 3 + c["count"] * (width + 3 * held)), "flops": 0}
    if c["kind"] == "fork":
        n = min(c["count"], c["slots"] - c["slots"] // 2)
        return {"bytes": 2.0 * n * one + 4 * n * (2 * width + 2 * held), "flops": 0}
    if c["kind"] == "copy":
        return {"bytes": 2.0 * c["count"] * one, "flops": 0}
    live = min(held * (c["slots"] - c["count"]), 0.9 * c["pages"])
    return {"bytes": 2.0 * one * live * (1 - live / c["pages"]) + 8 * c["pages"] + 8 * c["slots"] * width, "flops": 0}


# ------------------------------------------------------------------------------------------------ in 64 bits, from the definition

def _exact_row_values(raw, dim):
    """raw: int64 bytes [..., dim / 2 + 8] of a row (codes, then lo and scale as little-endian fp32): fp64 [..., dim]."""
    codes, q = raw[..., : dim // 2], raw[..., dim // 2:]
    word = q.to(torch.uint8).contiguous().view(torch.float32).double()
    out = torch.empty(*raw.shape[:-1], dim, dtype=torch.float64, device=raw.device)
    out[..., 0::2] = (codes % 16).double()
    out[..., 1::2] = (codes // 16).double()
    return out * word[..., 1, None] + word[..., 0, None]


def exact(case, seed):
    if case["op"] == "pages":
        return None                                      # bytes and page numbers: nothing there is computed in floating point
    s = prepare(case, seed)
    return _exact_attend(case, s) if case["op"] == "attend" else _exact_append(case, s)


def _exact_attend(c, s):
    dim, heads, page, new = c["dim"], c["heads"], c["page"], c["new"]
    group = c["q_heads"] // heads
    out = torch.empty(s["tokens"], c["q_heads"], dim, dtype=torch.float64, device=_DEV)
    for b, (slot, pos) in enumerate(zip(s["slots"].tolist(), s["pos"].tolist())):
        n = pos + new
        first = max(0, pos - c["window"] + 1) if c["window"] else 0
        ids = s["table"][slot, : -(-n // page)].long()
        for h in range(heads):
            sl = s["pool"][0, ids, h].reshape(-1, 16 * (dim + 16))               # [slices, bytes]
            half = 8 * dim
            def rows(at):
                both = torch.cat((sl[:, at:at + half].reshape(-1, dim // 2), sl[:, at + half:at + half + 128].reshape(-1, 8)), 1)
                return _exact_row_values(both[first:n].long(), dim)
            k, v = rows(0), rows(half + 128)
            q = s["q"][b * new:(b + 1) * new, h * group:(h + 1) * group].double()
            t = torch.einsum("ngd,td->gnt", q, k) / math.sqrt(dim)
            key = torch.arange(first, n, device=_DEV)
            mine = torch.arange(pos, n, device=_DEV).unsqueeze(1)
            off = (key > mine) | ((key <= mine - c["window"]) if c["window"] else False)
            p = torch.softmax(t.masked_fill(off, -math.inf), -1)
            out[b * new:(b + 1) * new, h * group:(h + 1) * group] = torch.einsum("gnt,td->ngd", p, v)
    return out


def _exact_append(c, s):
    def stands_for(x):
        x = x.double()
        lo = x.min(-1, keepdim=True).values
        width = x.max(-1, keepdim=True).values - lo
        scale, inv = (width / _LEVELS).float().double(), (_LEVELS / width).float().double()
        at = ((x - lo).float().double() * inv).float().double()                  # the position on the grid is an fp32 number
        return lo + torch.round(at) * scale
    return stands_for(s["k"]), stands_for(s["v"])
