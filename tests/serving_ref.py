"""64-bit forms of the serving operators (paged append, attention over pages, token
log probabilities) and the error bounds the GPU tests hold them to. A rounding to a
type is off by at most finfo(type).eps / 2 relative to the value."""
import math
import random

import torch

U32 = 2.0 ** -24  # half a step of fp32


class Batch:
    """A ragged batch over shuffled pages. lens: (new rows, tokens with them) a sequence."""

    def __init__(self, lens, page, kv_heads, d, dtype, seed, fill=None, extra=2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        need = [-(-m // page) for _, m in lens]
        n_pages = sum(need) + extra
        order = list(range(n_pages))
        random.Random(seed).shuffle(order)
        table, at = [[-7] * (max(need) + 1) for _ in lens], 0
        for s, n in enumerate(need):
            table[s][:n] = order[at:at + n]
            at += n
        start = [0]
        for n, _ in lens:
            start.append(start[-1] + n)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.lens, self.page, self.rows, self.dtype = lens, page, start[-1], dtype
        self.start = start
        self.table, self.q_start = torch.tensor(table, **i32), torch.tensor(start, **i32)
        self.kv_len = torch.tensor([m for _, m in lens], **i32)
        self.max_rows, self.max_len = max(n for n, _ in lens), max(m for _, m in lens)
        shape = (n_pages, kv_heads, page, d)
        self.k = torch.randn(shape, generator=g, device="cuda").to(dtype)
        self.v = torch.randn(shape, generator=g, device="cuda").to(dtype)
        if fill is not None:  # everything no sequence holds
            keep = torch.zeros((n_pages, page), dtype=torch.bool, device="cuda")
            for s, (_, m) in enumerate(lens):
                for p in range(0, m, page):
                    keep[table[s][p // page], :min(page, m - p)] = True
            for t in (self.k, self.v):
                t.masked_fill_(~keep[:, None, :, None], fill)

    def keys(self, pool, s):
        """K or V of sequence s: [kv_heads][tokens][d], and which tokens have a page"""
        m = self.lens[s][1]
        ids = self.table[s, :-(-m // self.page)].long()
        there = ((ids >= 0) & (ids < pool.shape[0])).repeat_interleave(self.page)[:m]
        rows = pool[ids.clamp(0, pool.shape[0] - 1)].transpose(0, 1).reshape(pool.shape[1], -1, pool.shape[3])
        return rows[:, :m], there


def attention(b, q, block, scale, softcap):
    """out [rows][heads][d], lse [rows][heads] and their error bounds, in 64 bits.

    Bounds. A score is a sum of d products in fp32, off by at most (d + 4) U32 scale
    sum |q k| (and 8 U32 softcap after a cap, whose slope is at most 1), a numerator
    2^x off by that and 2^-21 relative, its rounding for V's product by eps / 2, a sum
    of n terms by n U32: together w relative to the weighted |V|; then one rounding."""
    rows, heads, d = q.shape
    eps = torch.finfo(q.dtype).eps
    out = torch.zeros((rows, heads, d), dtype=torch.float64, device="cuda")
    lse = torch.full((rows, heads), -math.inf, dtype=torch.float64, device="cuda")
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for s, (n, m) in enumerate(b.lens):
        if n == 0 or m == 0:
            continue
        k, there = b.keys(b.k, s)
        v, _ = b.keys(b.v, s)
        pos = torch.arange(m - n, m, device="cuda")[:, None]
        key = torch.arange(m, device="cuda")[None]
        seen = there[None].expand(n, m)
        if block:
            seen = seen & (key < (pos.div(block, rounding_mode="floor") + 1) * block) & (pos >= 0)
        # what no row sees has no part, whatever it holds
        at = slice(b.start[s], b.start[s] + n)
        for h in range(heads):
            kk, vv = k[h // (heads // k.shape[0])].double(), v[h // (heads // k.shape[0])].double()
            qq = q[at, h].double()
            clean = torch.where(torch.isfinite(kk), kk, 0.0)
            x = qq @ clean.T * scale
            mag = qq.abs() @ clean.abs().T * abs(scale)
            if softcap:
                x = softcap * torch.tanh(x / softcap)
            x = torch.where(seen, x, -math.inf)
            top = x.amax(1, keepdim=True)
            some = torch.isfinite(top)
            p = torch.where(some, torch.exp(x - torch.where(some, top, 0.0)), 0.0)
            total = p.sum(1, keepdim=True)
            w = p / torch.where(total > 0, total, 1.0)
            fin = torch.where(torch.isfinite(vv), vv, 0.0)
            o = w @ fin
            ds = ((d + 4) * U32 * torch.where(seen, mag, 0.0).amax(1, keepdim=True) + 8 * U32 * softcap
                  + 2 * U32 * torch.where(seen, x.abs(), 0.0).amax(1, keepdim=True))
            rel = 2 * ds + 2 ** -20 + 2 * (m + 64) * U32
            out[at, h] = o
            tol[at, h] = eps / 2 * (1 + eps) * o.abs() + (eps / 2 + rel) * (w @ fin.abs()) + 2.0 ** -24
            lse[at, h] = torch.where(some, top + torch.log(total), -math.inf)[:, 0]
            ltol[at, h] = (rel + 4 * U32 * torch.where(some, top, 0.0).abs())[:, 0]
    return out, lse, tol, ltol


def append(b, q, k, v, q_norm, k_norm, eps, theta):
    """q_out and the new K rows [rows][heads][d] in 64 bits, and their bounds.

    A normed value is off by (d + 8) U32 relative, an fp32 sine or cosine of a reduced
    angle by 8 U32, a product and the sum by U32 each; then one rounding."""
    d, half = q.shape[2], q.shape[2] // 2
    place = torch.tensor([p for n, m in b.lens for p in range(m - n, m)], dtype=torch.float64, device="cuda")
    res = []
    for x, w in ((q, q_norm), (k, k_norm)):
        y = x[:len(place)].double()
        if w is not None:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
        if theta:
            ang = place[:, None, None] * theta ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
            a, e = y[..., :half], y[..., half:]
            z = torch.cat([a * ang.cos() - e * ang.sin(), e * ang.cos() + a * ang.sin()], -1)
            mag = (a.abs() + e.abs()).repeat(1, 1, 2)
        else:
            z, mag = y, y.abs()
        u = torch.finfo(x.dtype).eps / 2
        tiny = torch.finfo(x.dtype).smallest_normal * u
        # fp32 work only where there is any: without norm and rotation the copy is exact
        slack = (d + 24) * U32 if (w is not None or theta) else 0.0
        res += [z, (u * z.abs() * (1 + 2 * u) + tiny if slack else 0.0) + slack * mag]
    return res


def logprobs(x, tokens, exclude, n):
    """logprob, entropy, ids, top log probabilities in 64 bits, and the bound on them.

    Terms 2^y with y = (x - m) log2 e rounded: off by 4 U32 |x - m| + 2^-21 relative; sums
    of at most 2^12 terms in a row and a tree: 2^12 U32 is above any order's error; the
    logarithm and the differences 4 U32 of their size."""
    x = x.double().clone()
    if exclude >= 0:
        x[:, exclude] = -math.inf
    R, V = x.shape
    bad = (torch.isnan(x) | (x == math.inf)).any(1)
    m = x.amax(1, keepdim=True)
    none = (m == -math.inf)[:, 0]
    dm = x - torch.where(torch.isfinite(m), m, 0.0)
    e = torch.exp(dm)
    S = e.sum(1)
    mom = torch.where(e > 0, dm * e, 0.0).sum(1)
    # x - m first: m + ln S loses ln S where m is a type's lowest value
    minus_lse = lambda y: y - torch.where(torch.isfinite(m), m, 0.0) - torch.log(S)[:, None]
    ent = torch.where(none, 0.0, torch.log(S) - mom / S)
    t = tokens.long()
    pick = minus_lse(x.gather(1, t.clamp(0, V - 1)[:, None]))[:, 0]
    nan = torch.tensor(math.nan, dtype=torch.float64, device=x.device)
    lp = torch.where(none | (pick == -math.inf), -math.inf, pick)
    lp = torch.where(bad | (t >= V), nan, lp)
    lp = torch.where(t < 0, 0.0, lp)
    ent = torch.where(bad, nan, ent)
    ids = torch.sort(torch.where(torch.isnan(x), -math.inf, x) + 0.0, dim=1, descending=True, stable=True).indices
    ids = torch.cat([ids, ids.new_zeros((R, max(0, n - V)))], 1)[:, :n]
    val = x.gather(1, ids)
    gone = (val == -math.inf) | (torch.arange(n, device=x.device)[None] >= V)
    top = torch.where(gone, -math.inf, minus_lse(val))
    ids = torch.where(gone | bad[:, None], -1, ids)
    top = torch.where(bad[:, None], nan, top)
    mean = torch.where(none | bad, 0.0, -mom / S)
    rel = 2 ** -21 + 2 ** 12 * U32 + 8 * U32 * mean
    return lp, ent, ids.to(torch.int32), top, rel


def close(got, want, tol):
    """finite values within tol, the others equal (NaN with NaN)"""
    got, want = got.double(), want.double()
    tol = torch.as_tensor(tol, dtype=torch.float64, device=want.device).expand(want.shape)
    fin = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN in other places"
    rest = ~fin & ~torch.isnan(want)
    assert torch.equal(got[rest], want[rest]), "infinities in other places"
    err = (got - want).abs()[fin] - tol[fin]
    if err.numel():
        worst = err.max().item()
        assert worst <= 0, f"off by {worst:.3g} more than the bound; {(err > 0).sum().item()} of {err.numel()} values"
