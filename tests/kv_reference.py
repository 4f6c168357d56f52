"""The 4-bit cache of keys and values in plain numpy and Python, fp64 where the format does not fix fp32: what the GPU
tests compare with.  Shares no code with the library."""
import numpy as np


def quantize_row(x):
    """(codes [D] ints, lo, scale) of one row of fp32 values, each step of the format in its own rounding."""
    f = np.float32
    x = np.asarray(x, f)
    fin = x[np.isfinite(x)]
    lo, hi = (f(fin.min()), f(fin.max())) if fin.size else (f(0), f(0))
    width = float(hi) - float(lo)
    with np.errstate(all="ignore"):
        scale = f(width / 15)
        inv = f(15 / width) if width > 0 else f(np.inf)
        if not np.isfinite(inv):
            return np.zeros(x.size, int), lo, f(0)
        t = np.where(np.isnan(x), lo, np.minimum(np.maximum(x, lo), hi)).astype(f)
        if np.isinf(f(hi - lo)):
            at = (t * f(0.5) - lo * f(0.5)).astype(f) * f(inv * f(2))
        else:
            at = (t - lo).astype(f) * inv
        return np.rint(at.astype(f)).astype(int), lo, scale


def pack_row(codes):
    return (codes[0::2] | (codes[1::2] << 4)).astype(np.uint8)


def parts(pool, dim):
    """Views of the K codes, K quantizers, V codes and V quantizers of a pool [..., 16 * (dim + 16)] of bytes."""
    k = 8 * dim
    lead = pool.shape[:-1]
    return (pool[..., :k].reshape(*lead, 16, dim // 2), pool[..., k:k + 128].reshape(*lead, 16, 8),
            pool[..., k + 128:2 * k + 128].reshape(*lead, 16, dim // 2), pool[..., 2 * k + 128:].reshape(*lead, 16, 8))


def values(codes, quant):
    """fp64 rows of codes [..., dim / 2] and quantizers [..., 8], and their (lo, scale)."""
    with np.errstate(invalid="ignore"):                             # quantizers of rows that were never written may be NaN
        q = np.ascontiguousarray(quant).view(np.float32).astype(np.float64)
    c = np.empty(codes.shape[:-1] + (2 * codes.shape[-1],))
    c[..., 0::2] = codes & 15
    c[..., 1::2] = codes >> 4
    return q[..., :1] + q[..., 1:] * c, q[..., 0], q[..., 1], c


def sequence(pool, pages, head, n, page_size, dim):
    """K and V of tokens 0 .. n - 1 of one head: ((values, lo, scale, codes), the same); pool [pages, heads, slices, bytes]."""
    need = -(-n // page_size)
    s = pool[np.asarray(pages[:need], int), head].reshape(need * (page_size // 16), pool.shape[-1])
    kc, kq, vc, vq = parts(s, dim)
    return [tuple(a.reshape(-1, *a.shape[2:])[:n] for a in values(c, q)) for c, q in ((kc, kq), (vc, vq))]


def attention_row(q, k, v, visible, scale, weight_eps, out_eps, halves=False):
    """(out, lse, bound of |error|, of lse's) of one query over the rows of `sequence`, fp64; visible [n] truth values.  halves: for
    the kernel that rounds the rows of K and V to fp16 first."""
    kv, klo, ks, _ = k
    vv, vlo, vs, vc = v
    if not visible.any():
        return np.zeros(len(q)), -np.inf, np.zeros(len(q)), 0.0
    kv, klo, ks, vv, vlo, vs, vc = (x[visible] for x in (kv, klo, ks, vv, vlo, vs, vc))
    s = kv @ q * scale
    top = s.max()
    p = np.exp(s - top)
    l = p.sum()
    out = p @ vv / l
    # Errors.  A score: products of fp16 halves of q (2^-22 off together, 0 for bf16) with whole numbers, summed in fp32 in up
    # to 2 * 16 matrix steps and scaled in 3 roundings: under 64 steps of 2^-23 of the sum of magnitudes.  A change ds of every
    # score moves the result by at most 2 ds times the spread of the values.
    ds = 2.0 ** -17 * abs(scale) * (np.abs(q).sum() * (np.abs(klo) + 15 * ks).max())
    # exp2 of it: 2^-21 of itself.  A weight p * vs is rounded to 11 (bf16) or 22 bits, and below the smallest normal to
    # 2^-25 / 16 of the largest scale; sums of up to n terms in fp32 add n / 8 steps at most (a lane sums an eighth of a warp's share).
    spread = np.abs(vv).max() + np.abs(out).max()
    n = len(s)
    weights = weight_eps * (p * vs) @ vc / l + n * 15 * 2.0 ** -29 * vs.max() / l
    if halves:
        # A row's value v = mid + scale (c - 8), mid = lo + 8 scale, is rounded to fp16 (2^-11 of itself), and so are mid (2^-11) and
        # scale (2^-11, times at most 8); values are scaled to a tile's largest at 2^10 or above, so a subnormal's
        # 2^-25 is 2^-35 of that largest, twice (mid and the result).  A weight p is rounded to fp16 too, or to 2^-25 / 2^5 of its
        # value at the power of two of the largest values.
        def rounding(x, lo, scale):
            return 2.0 ** -11 * (np.abs(x) + (np.abs(lo + 8 * scale) + 8 * scale)[:, None]) + 2.0 ** -34 * np.abs(x).max()
        ds += abs(scale) * (rounding(kv, klo, ks) @ np.abs(q)).max()
        weights = p @ (rounding(vv, vlo, vs) + 2.0 ** -11 * np.abs(vv)) / l + n * 2.0 ** -28 * np.abs(vv).max() / l
    err = (2 * ds + 2.0 ** -20 + (n / 8 + 16) * 2.0 ** -24) * spread + weights
    return out, top + np.log(l), err + out_eps * (np.abs(out) + err), 2 * ds + (n / 8 + 16) * 2.0 ** -23 + 2.0 ** -20 * (1 + abs(top))


class Book:
    """Pages, table, lengths of a cache, and what the calls do to them."""

    def __init__(self, pages, slots, max_pages, page_size):
        self.refs, self.table = [0] * pages, [[-1] * max_pages for _ in range(slots)]
        self.lens, self.page_size, self.max_pages = [0] * slots, page_size, max_pages

    def need(self, n):
        return -(-n // self.page_size)

    def free_pages(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def extend(self, slots, new):
        """The positions; (range flag, exhausted flag)."""
        seen, take, flag = set(), [], False
        for s, n in zip(slots, new):
            ok = 0 <= s < len(self.lens) and s not in seen and n >= 0 and self.lens[s] + n <= self.max_pages * self.page_size
            if 0 <= s < len(self.lens):
                seen.add(s)
            flag |= not ok
            take.append((s, n) if ok else None)
        want = sum(self.need(self.lens[s] + n) - self.need(self.lens[s]) for s, n in filter(None, take))
        free = self.free_pages()
        if want > len(free):
            return [-1] * len(slots), flag, True
        pos = []
        for t in take:
            if t is None:
                pos.append(-1)
                continue
            s, n = t
            pos.append(self.lens[s])
            for j in range(self.need(self.lens[s]), self.need(self.lens[s] + n)):
                p = free.pop(0)
                self.table[s][j], self.refs[p] = p, 1
            self.lens[s] += n
        return pos, flag, False

    def free(self, slots):
        flag = False
        for s in slots:
            if not 0 <= s < len(self.lens):
                flag = True
                continue
            for j in range(self.need(self.lens[s])):
                self.refs[self.table[s][j]] -= 1
                self.table[s][j] = -1
            self.lens[s] = 0
        return flag

    def fork(self, src, dst):
        """[(page, page that takes its bytes)]; (range flag, exhausted flag)."""
        lens, table = list(self.lens), [list(r) for r in self.table]
        n, seen, pairs, flag = len(lens), set(), [], False
        for s, d in zip(src, dst):
            ok = 0 <= s < n and 0 <= d < n and d not in seen and lens[d] == 0
            if 0 <= d < n:
                seen.add(d)
            flag |= not ok
            if ok:
                pairs.append((s, d))
        tails = [s for s, _ in pairs if lens[s] % self.page_size]
        free = self.free_pages()
        if len(tails) > len(free):
            return [], flag, True
        moves = []
        for s, d in pairs:
            full = lens[s] // self.page_size
            for j in range(full):
                self.table[d][j] = table[s][j]
                self.refs[table[s][j]] += 1
            if lens[s] % self.page_size:
                p = free.pop(0)
                self.table[d][full], self.refs[p] = p, 1
                moves.append((table[s][full], p))
            self.lens[d] = lens[s]
        return moves, flag, False

    def copies(self, src, dst):
        """The pairs that are copied, and the range flag."""
        n, first, moves, flag = len(self.refs), {}, [], False
        inside = [0 <= s < n and 0 <= d < n for s, d in zip(src, dst)]
        for i, d in enumerate(dst):
            if inside[i]:
                first.setdefault(d, i)
        for i, (s, d) in enumerate(zip(src, dst)):
            if inside[i] and first[d] == i and (s == d or s not in first):
                moves.append((s, d))
            else:
                flag = True
        return moves, flag

    def compact(self):
        live = sum(r != 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] == 0]
        movers = [p for p in range(live, len(self.refs)) if self.refs[p] != 0]
        to = dict(zip(movers, holes))
        for f, t in to.items():
            self.refs[t], self.refs[f] = self.refs[f], 0
        self.table = [[to.get(p, p) for p in r] for r in self.table]
        return list(to.items()), live
