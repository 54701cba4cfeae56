"""Plain references of the calls on drafted tokens, in 64 bits on the CPU,
straight from the definitions in include/art.h."""
from __future__ import annotations

import math

import torch

D = 128


def spans(B, rows, offsets, context, cap):
    """(sequence, first row, nodes, context) of the sequences that are worked on."""
    for b in range(B):
        if offsets is None:
            first, end = b * (rows // B), (b + 1) * (rows // B)
        else:
            first, end = int(offsets[b]), int(offsets[b + 1])
        n, c = end - first, int(context[b])
        if n > 0 and c >= 0 and c + n <= cap:
            yield b, first, n, c


def ancestors(parents, i):
    """Node i and its ancestors; a parent that is no earlier node ends the walk."""
    path = [i]
    while 0 <= parents[path[-1]] < path[-1]:
        path.append(parents[path[-1]])
    return path


def bits(nodes, words):
    """int64 words with the bits of `nodes`."""
    out = [0] * words
    for j in nodes:
        if j < 64 * words:
            out[j // 64] |= 1 << (j % 64)
    return [w - (1 << 64) if w >> 63 else w for w in out]


def rotate(x, positions, freqs, layout, scale):
    """Rows [n][heads][128] in fp64 turned to positions [n], and per value a bound
    of what enters it: |x| + |y| of its pair times the scale."""
    x = x.double()
    half = len(freqs)
    angle = positions.double()[:, None] * freqs.double()
    c, s = (angle.cos() * scale)[:, None], (angle.sin() * scale)[:, None]
    y, size = x.clone(), x.abs()
    first = slice(0, 2 * half, 2) if layout == "interleaved" else slice(0, half)
    second = slice(1, 2 * half, 2) if layout == "interleaved" else slice(half, 2 * half)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    both = (a.abs() + b.abs()) * abs(scale)
    size[..., first], size[..., second] = both, both
    return y, size


def attend(q, k_cache, v_cache, table, context, offsets, mask, scale):
    """(out, lse, mean of |v| under the weights, largest sum of |q k| in base 2,
    tokens seen) of every row, fp64; rows of no sequence are NaN."""
    rows, Hq, _ = q.shape
    P, H, page, _ = k_cache.shape
    g = Hq // H
    out = torch.full((rows, Hq, D), math.nan, dtype=torch.float64)
    lse = torch.full((rows, Hq), math.nan, dtype=torch.float64)
    size = torch.zeros((rows, Hq, D), dtype=torch.float64)
    work = torch.zeros((rows, Hq), dtype=torch.float64)
    count = torch.zeros((rows, 1), dtype=torch.float64)
    c = abs(scale) / math.log(2)
    for b, first, n, ctx in spans(table.shape[0], rows, offsets, context, table.shape[1] * page):
        t = torch.arange(ctx + n)
        pages = table[b][t // page].long().clamp(0, P - 1)
        keys, values = k_cache[pages, :, t % page].double(), v_cache[pages, :, t % page].double()
        for i in range(n):
            if mask is None:
                nodes = list(range(i + 1))
            else:
                nodes = [j for j in range(min(n, 64 * mask.shape[1])) if int(mask[first + i][j // 64]) >> (j % 64) & 1]
            see = torch.tensor(list(range(ctx)) + [ctx + j for j in nodes], dtype=torch.long)
            count[first + i] = len(see)
            for h in range(Hq):
                kk, vv, x = keys[see, h // g], values[see, h // g], q[first + i, h].double()
                s = (kk * x).sum(-1) * scale
                if len(see) == 0:
                    out[first + i, h], lse[first + i, h] = 0.0, -math.inf
                    continue
                lse[first + i, h] = torch.logsumexp(s, 0)
                w = torch.exp(s - lse[first + i, h])
                out[first + i, h] = (w[:, None] * vv).sum(0)
                size[first + i, h] = (w[:, None] * vv.abs()).sum(0)
                work[first + i, h] = (kk.abs() * x.abs()).sum(-1).max() * c
    return out, lse, size, work, count


def attend_bounds(out, lse, size, work, count, bf16):
    """How far a kernel may be off in out and lse.  Scores: fp32 sums of exact
    products, at most 130 roundings of 2^-24 of the sum of magnitudes, one of the
    fused multiply-add, whose reference is of that size too (base 2, hence ln 2);
    2^x and the reciprocal: 2^-22; sums of p and of p v in fp32: `count` roundings
    of 2^-24 and a few for the joins.  A bf16 output: probabilities rounded to bf16
    (2^-8), and the output (2^-8)."""
    score = math.log(2) * 133 * work * 2.0 ** -24 + 2.0 ** -22
    sums = (count + 16) * 2.0 ** -24
    each = 2 * (score + sums) + (2.0 ** -8 if bf16 else 2.0 ** -22)
    far = size * each[..., None]
    if bf16:
        far = far + 2.0 ** -8 * (out.abs() + far)
    return far, score + sums + 2.0 ** -21 * (lse.abs() + 1)


def verify(target, draft, tokens, parents, uniforms, last, max_path):
    """One sequence: (accepted nodes, next token)."""
    V, n = target.shape[1], len(parents)
    now, path = 0, [0]
    while True:
        p = target[now].double()
        q = None if draft is None else draft[now].double()
        a, f, w, chosen = 0.0, 1.0, p.clone(), None
        for c in range(now + 1, n if len(path) < max_path else 0):
            if parents[c] != now or not 0 <= tokens[c] < V:
                continue
            x, u = tokens[c], float(uniforms[c])
            if q is not None:
                if u * float(q[x]) * f < float(w[x]):
                    chosen = c
                    break
                a += f
                w = (p - a * q).clamp_min(0)
                f = float(w.sum())
            else:
                if u * f < float(w[x]):
                    chosen = c
                    break
                f = max(f - float(w[x]), 0.0)
                w[x] = 0.0
        if chosen is None:
            break
        now = chosen
        path.append(now)
    if not float(w.sum()) > 0:
        w = p
    run = w.cumsum(0)
    over = torch.nonzero(run > float(last) * run[-1])
    if len(over) == 0:
        over = torch.nonzero(w > 0)[-1:]
    return path, int(over[0]) if len(over) else 0


def verify_all(target, draft, tokens, parents, uniforms, last, offsets, max_path):
    B = len(last)
    accepted, counts, following = torch.full((B, max_path), -1, dtype=torch.int32), [], []
    for b in range(B):
        rows = len(tokens)
        first, end = (b * (rows // B), (b + 1) * (rows // B)) if offsets is None else (int(offsets[b]), int(offsets[b + 1]))
        if not 0 < end - first <= 1024:
            counts.append(0)
            following.append(-1)
            continue
        s = slice(first, end)
        path, token = verify(target[s], None if draft is None else draft[s], tokens[s].tolist(), parents[s].tolist(),
                             uniforms[s].tolist(), last[b], max_path)
        accepted[b, : len(path)] = torch.tensor(path, dtype=torch.int32)
        counts.append(len(path))
        following.append(token)
    return accepted, torch.tensor(counts, dtype=torch.int32), torch.tensor(following, dtype=torch.int32)


def random_parents(gen, n, chain=False):
    return [i - 1 if chain or i == 0 else int(torch.randint((i - 1) // 3, i, (1,), generator=gen)) for i in range(n)]


class Cache:
    """Pools with pages in random order and a table over them; slots of no token
    hold NaN.  `pad`: extra elements between tokens, heads and pages."""

    def __init__(self, gen, lens, heads, page, spare=2, pad=0, extra_width=0):
        need = [-(-n // page) for n in lens]
        width, pages = max(1, max(need)) + extra_width, sum(need) + spare
        shape = (pages, heads + (1 if pad else 0), page + (1 if pad else 0), D + 8 * pad)
        self.k, self.v = (torch.full(shape, math.nan, dtype=torch.bfloat16)[:, :heads, :page, :D] for _ in range(2))
        self.table = torch.full((len(lens), width), -5, dtype=torch.int32)
        order = torch.randperm(pages, generator=gen).int()
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at: at + n]
            at += n
        for b, n in enumerate(lens):
            t = torch.arange(n)
            where = self.table[b][t // page].long(), t % page
            for pool in (self.k, self.v):
                pool[where[0], :, where[1]] = torch.randn(n, heads, D, generator=gen).bfloat16()

    def to(self, device):
        """The same strides on a device."""
        c = object.__new__(Cache)
        for name in ("k", "v"):
            x = getattr(self, name)
            base = torch.full((x.stride(0) * x.shape[0],), math.nan, dtype=torch.bfloat16, device=device)
            y = base.as_strided(x.shape, x.stride())
            y.copy_(x)
            setattr(c, name, y)
        c.table = self.table.to(device)
        return c
