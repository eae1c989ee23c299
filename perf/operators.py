"""The serving operators whose time is tracked: a paged K / V cache with the
attention that reads it, and the log probabilities of what a model answers.

  append    new tokens enter a paged cache: RMSNorm of every query and key head,
            rotate-half position rotation, K and V written to their pages, the
            rotated queries to the attention's input
  attend    attention of each sequence's newest rows over its pages: grouped
            query heads, causal, block-causal or full, scores capped by a tanh
            if asked for
  logprobs  log probability of a given token per row of logits, the entropy of
            the row and its most probable tokens

`run` makes the package's calls where `own` is true, and computes the plain form
(elementary torch operations in 32 bits, rounded once) where it is false. Head
layouts are those of synth.shapes; lengths of a ragged batch follow from the
case alone.
"""
from __future__ import annotations

import math
import random

import torch

own = False

# (query heads, K / V heads, head dimension) of the layouts in synth.shapes
LAYOUTS = {"tiny": (4, 2, 64), "small": (8, 2, 64), "small128": (4, 2, 128),
           "wide1536": (12, 4, 128), "wide6144": (48, 8, 128), "dream7b": (28, 4, 128),
           "llada8b": (32, 32, 128)}
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------- the cases
def _paged(name, op, layout, seqs, rows, ctx, shape="even", page=64, dtype="bf16", block=1,
           softcap=0.0, shared=False, norm=True, mix=1):
    """seqs sequences. shape "even": each adds `rows` tokens to `ctx` cached ones;
    "ragged": 1 to `rows` tokens and 0 to `ctx` cached ones, drawn by `mix`; "mixed":
    the first adds `rows` tokens, the others one each, ragged contexts. block: 0 full
    attention, 1 causal, c block-causal in blocks of c. shared: the sequences share
    the pages of their cached tokens, whole pages of them (branches of one prefix)."""
    return dict(name=name, op=op, layout=layout, seqs=seqs, rows=rows, ctx=ctx, shape=shape,
                page=page, dtype=dtype, block=block, softcap=softcap, shared=shared, norm=norm,
                mix=mix)


def _logits(name, rows, vocab, dtype, top, exclude=True):
    return dict(name=name, op="logprobs", rows=rows, vocab=vocab, dtype=dtype, top=top,
                exclude=exclude)


def listed():
    return [
        # one sequence's next token enters the cache: the smallest call, all latency
        _paged("append one token", "append", "dream7b", 1, 1, 512),
        # blocks of many sequences, ragged, small pages, no norms (a layout without them)
        _paged("append ragged blocks", "append", "wide6144", 37, 61, 900, "ragged", page=16,
               dtype="f16", norm=False, mix=3),
        # prompts of a serving batch enter together
        _paged("append prompts", "append", "dream7b", 8, 1024, 1000),
        # one sequence, one token: the inner loop of an interactive session
        _paged("attend one token", "attend", "dream7b", 1, 1, 1500),
        # one token over a long document
        _paged("attend one token, long", "attend", "wide6144", 1, 1, 131071, dtype="f16", page=128),
        # a decode batch of unequal lengths, one K / V head per query head
        _paged("attend decode batch", "attend", "llada8b", 48, 1, 4000, "ragged", page=32, mix=5),
        # eight lookahead branches of a 32-row block over one prefix, full inside the block
        _paged("attend branches", "attend", "dream7b", 8, 32, 512, block=0, shared=True),
        # a prompt's last chunk over what is cached already
        _paged("attend prompt chunk", "attend", "dream7b", 1, 8191, 6000),
        # a prompt chunk beside running sequences, capped scores, small heads
        _paged("attend mixed batch", "attend", "small", 25, 777, 1900, "mixed", page=16, softcap=30.0,
               mix=7),
        # the next token's log probabilities of one sequence
        _logits("logprobs one row", 1, 152064, "bf16", 5),
        # a verify forward's rows: 8 branches of 32 with alternatives
        _logits("logprobs branches", 256, 152064, "f32", 20),
        # scoring a document: the given tokens and the entropy, no alternatives
        _logits("logprobs document", 2047, 126464, "bf16", 0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = {}
    for c in listed():
        w = work(c)
        t = top.setdefault(c["op"], dict(bytes=0, flops=0))
        for k in t:
            t[k] = max(t[k], w[k])
    while True:
        c = _draw(rng)
        w = work(c)
        if all(w[k] <= top[c["op"]][k] for k in w):
            del c["name"]
            return c


def _draw(rng):
    op = rng.choice(["append", "attend", "attend", "logprobs"])
    if op == "logprobs":
        vocab = rng.choice([1024, 2048, 3000, 126464, 152064, _log_uniform(rng, 500, 160000)])
        return _logits("", _log_uniform(rng, 1, 2048), vocab, rng.choice(["bf16", "f16", "f32"]),
                       rng.choice([0, 1, rng.randint(2, 20), rng.randint(2, 32)]),
                       rng.random() < 0.7)
    layout = rng.choice(["dream7b", "dream7b", "llada8b", "wide6144", "wide1536", "small128",
                         "small", "tiny"])
    shape = rng.choice(["even", "ragged", "ragged", "mixed"])
    seqs = _log_uniform(rng, 1, 64)
    dtype, page = rng.choice(["bf16", "f16"]), rng.choice([16, 32, 64, 128, 256])
    mix = rng.randrange(1 << 30)
    if op == "append":
        return _paged("", op, layout, seqs, _log_uniform(rng, 1, 2048), _log_uniform(rng, 1, 4000),
                      shape, page, dtype, norm=rng.random() < 0.7, mix=mix)
    rows = rng.choice([1, 1, _log_uniform(rng, 2, 64), _log_uniform(rng, 2, 4096)])
    ctx = _log_uniform(rng, 1, 131072) if seqs <= 2 else _log_uniform(rng, 1, 8000)
    return _paged("", op, layout, seqs, rows, ctx, shape, page, dtype,
                  block=rng.choice([0, 1, 1, 1, 16, 32, rng.randint(2, 100)]),
                  softcap=rng.choice([0.0, 0.0, 0.0, 20.0, 50.0]),
                  shared=shape == "even" and rng.random() < 0.3, mix=mix)


# --------------------------------------------------------------------- lengths
def _lens(case):
    """(new rows, tokens in the cache with them) of every sequence"""
    rng = random.Random(case["mix"])
    out = []
    for s in range(case["seqs"]):
        n, c = case["rows"], case["ctx"]
        if case["shape"] == "ragged":
            n, c = _log_uniform(rng, 1, n), rng.randint(0, c)
        elif case["shape"] == "mixed":
            n, c = (n if s == 0 else 1), rng.randint(0, c)
        out.append((n, n + c))
    return out


def _shared_pages(case):
    return case["ctx"] // case["page"] if case["shared"] else 0


def work(case):
    if case["op"] == "logprobs":
        R, V = case["rows"], case["vocab"]
        # per logit: a maximum, a difference, an exponential, two sums and a product
        return dict(bytes=R * V * SIZE[case["dtype"]] + R * (4 + 8 + 8 * case["top"]), flops=6 * R * V)
    Hq, Hkv, d = LAYOUTS[case["layout"]]
    lens, size = _lens(case), SIZE[case["dtype"]]
    rows = sum(n for n, _ in lens)
    table = sum(-(-m // case["page"]) for _, m in lens) * 4 + 8 * len(lens)
    if case["op"] == "append":
        values = rows * (Hq + 2 * Hkv) * d
        return dict(bytes=2 * values * size + table, flops=10 * values)
    keys = sum(m for _, m in lens) - (len(lens) - 1) * _shared_pages(case) * case["page"]
    pairs = 0
    for n, m in lens:
        if case["block"] == 0:
            pairs += n * m
        else:
            c = case["block"]
            pairs += sum(min(m, (p // c + 1) * c) for p in range(m - n, m))
    return dict(bytes=(2 * rows * Hq + 2 * keys * Hkv) * d * size + rows * Hq * 4 + table,
                flops=4 * pairs * Hq * d)


# ---------------------------------------------------------------------- inputs
def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed(1000003 * (seed + 1) + stream)


def _normal(gen, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _batch(case, seed):
    """Pages in shuffled order over the pool, so that a sequence's are scattered."""
    lens, page = _lens(case), case["page"]
    share = _shared_pages(case)
    need = [-(-m // page) for _, m in lens]
    n_pages = sum(need) - (len(lens) - 1) * share + 3
    order = list(range(n_pages))
    random.Random(seed + 17).shuffle(order)
    table = [[-1] * (max(need) + 1) for _ in lens]
    common, at = order[:share], share
    for s, n in enumerate(need):
        own_pages = order[at:at + n - share]
        at += n - share
        table[s][:n] = common + own_pages
    start = [0]
    for n, _ in lens:
        start.append(start[-1] + n)
    i32 = dict(dtype=torch.int32, device="cuda")
    return dict(lens=lens, n_pages=n_pages, rows=start[-1], table=torch.tensor(table, **i32),
                q_start=torch.tensor(start, **i32), kv_len=torch.tensor([m for _, m in lens], **i32),
                max_rows=max(n for n, _ in lens), max_len=max(m for _, m in lens))


def _inputs(case, seed):
    if case["op"] == "logprobs":
        g, R, V = _gen(seed, 1), case["rows"], case["vocab"]
        # logits of standard deviation 2 to 4 with a few likely tokens in every row,
        # rounded to their type (16-bit rows hold many equal values)
        x = torch.empty((R, V), dtype=TYPES[case["dtype"]], device="cuda")
        for r in range(0, R, 256):
            n = min(256, R - r)
            y = torch.randn((n, V), generator=g, device="cuda")
            y *= 2 + 2 * torch.rand((n, 1), generator=g, device="cuda")
            at = torch.randint(0, V, (n, 4), generator=g, device="cuda")
            y.scatter_add_(1, at, 12 * torch.rand((n, 4), generator=g, device="cuda"))
            x[r:r + n] = y
        tokens = torch.randint(0, V, (R,), generator=g, device="cuda")
        best = x.float().argmax(1) if R * V < 1 << 27 else x.argmax(1)
        tokens = torch.where(torch.rand(R, generator=g, device="cuda") < 0.5, best, tokens)
        return dict(logits=x, tokens=tokens.to(torch.int32))
    Hq, Hkv, d = LAYOUTS[case["layout"]]
    t, g, b = TYPES[case["dtype"]], _gen(seed, 2), _batch(case, seed)
    pool = (b["n_pages"], Hkv, case["page"], d)
    b["k_pages"], b["v_pages"] = _normal(g, pool, t), _normal(g, pool, t)
    if case["op"] == "attend":
        b["q"] = _normal(g, (b["rows"], Hq, d), t, 1.5)
        return b
    # the packed rows of a QKV projection; its channels differ in scale
    qkv = torch.randn((b["rows"], (Hq + 2 * Hkv) * d), generator=g, device="cuda")
    qkv *= torch.exp(0.5 * torch.randn((Hq + 2 * Hkv) * d, generator=g, device="cuda"))
    b["qkv"] = qkv.to(t)
    b["q_norm"] = (1 + _normal(g, (d,), torch.float32, 0.1)).to(t) if case["norm"] else None
    b["k_norm"] = (1 + _normal(g, (d,), torch.float32, 0.1)).to(t) if case["norm"] else None
    return b


EPS, THETA = 1e-6, 1e6


def prepare(case, seed):
    st = dict(_inputs(case, seed), case=case)
    if case["op"] == "append":
        Hq, _, d = LAYOUTS[case["layout"]]
        st["q_out"] = torch.empty((st["rows"], Hq, d), dtype=TYPES[case["dtype"]], device="cuda")
    if own:
        import paper_2512_16229_amd as lp
        st["lp"] = lp
        f32 = dict(dtype=torch.float32, device="cuda")
        need = 0
        if case["op"] == "attend":
            Hq, Hkv, d = LAYOUTS[case["layout"]]
            st["out"], st["lse"] = torch.empty_like(st["q"]), torch.empty((st["rows"], Hq), **f32)
            need = lp.lopa_paged_attention_workspace(Hq, Hkv, d, case["seqs"], st["rows"],
                                                     st["max_rows"], st["max_len"])
        elif case["op"] == "logprobs":
            R, n = case["rows"], case["top"]
            st["logprob"], st["entropy"] = torch.empty(R, **f32), torch.empty(R, **f32)
            st["top_ids"] = torch.empty((R, n), dtype=torch.int32, device="cuda") if n else None
            st["top_logprobs"] = torch.empty((R, n), **f32) if n else None
            need = lp.lopa_token_logprobs_workspace(R, case["vocab"], n)
        st["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return st


# ------------------------------------------------------------------------ pass
def run(st):
    if own:
        return _run_own(st)
    return {"append": _plain_append, "attend": _plain_attend, "logprobs": _plain_logprobs}[
        st["case"]["op"]](st)


def _run_own(st):
    lp, case = st["lp"], st["case"]
    if case["op"] == "append":
        Hq, Hkv, d = LAYOUTS[case["layout"]]
        q, k, v = st["qkv"].view(st["rows"], Hq + 2 * Hkv, d).split([Hq, Hkv, Hkv], 1)
        lp.lopa_paged_append(st["k_pages"], st["v_pages"], st["table"], st["q_start"], st["kv_len"],
                             q, k, v, st["q_norm"], st["k_norm"], EPS, THETA, st["q_out"])
        return st["q_out"], st["k_pages"], st["v_pages"]
    if case["op"] == "attend":
        d = st["q"].shape[2]
        lp.lopa_paged_attention(st["q"], st["k_pages"], st["v_pages"], st["table"], st["q_start"],
                                st["kv_len"], st["max_rows"], st["max_len"], case["block"],
                                d ** -0.5, case["softcap"], st["out"], st["lse"], st["workspace"])
        return st["out"], st["lse"]
    exclude = case["vocab"] - 1 if case["exclude"] else -1
    lp.lopa_token_logprobs(st["logits"], st["tokens"], exclude, st["logprob"], st["entropy"],
                           st["top_ids"], st["top_logprobs"], st["workspace"])
    if case["top"]:
        return st["logprob"], st["entropy"], st["top_ids"], st["top_logprobs"]
    return st["logprob"], st["entropy"]


# ----------------------------------------------------------------- plain forms
def _row_places(st):
    """sequence and position of every new row"""
    start, kv_len = st["q_start"].long(), st["kv_len"].long()
    n = start[1:] - start[:-1]
    seq = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n, output_size=st["rows"])
    pos = torch.arange(st["rows"], device="cuda") - start[seq] + kv_len[seq] - n[seq]
    return seq, pos


def _plain_append(st):
    case = st["case"]
    Hq, Hkv, d = LAYOUTS[case["layout"]]
    seq, pos = _row_places(st)
    x = st["qkv"].view(st["rows"], Hq + 2 * Hkv, d).float()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if case["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + EPS) * st["q_norm"].float()
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + EPS) * st["k_norm"].float()
    half = d // 2
    inv = THETA ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    angle = pos.double()[:, None] * inv
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def rotate(y):
        a, b = y[..., :half], y[..., half:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    st["q_out"].copy_(rotate(q))
    page, slot = st["table"].long()[seq, pos // case["page"]], pos % case["page"]
    st["k_pages"][page, :, slot] = rotate(k).to(st["k_pages"].dtype)
    st["v_pages"][page, :, slot] = v.to(st["v_pages"].dtype)
    return st["q_out"], st["k_pages"], st["v_pages"]


def _plain_attend(st):
    case = st["case"]
    Hq, Hkv, d = LAYOUTS[case["layout"]]
    G, c = Hq // Hkv, case["block"]
    out = torch.empty_like(st["q"])
    lse = torch.empty((st["rows"], Hq), dtype=torch.float32, device="cuda")
    row = 0
    for s, (n, m) in enumerate(st["lens"]):
        pages = st["table"][s, :-(-m // case["page"])].long()
        # [kv heads][keys][d], first m keys
        k, v = (p[pages].transpose(0, 1).reshape(Hkv, -1, d)[:, :m].float()
                for p in (st["k_pages"], st["v_pages"]))
        q = st["q"][row:row + n].float().view(n, Hkv, G, d).permute(1, 2, 0, 3).reshape(Hkv, G * n, d)
        hidden = None
        if c:
            at = torch.arange(m - n, m, device="cuda")
            last = ((at // c + 1) * c).repeat(G)
            hidden = torch.arange(m, device="cuda")[None, :] >= last[:, None]
        step = max(1, min(Hkv, (1 << 30) // (G * n * m)))  # heads at a time
        for h in range(0, Hkv, step):
            score = torch.matmul(q[h:h + step], k[h:h + step].transpose(1, 2).contiguous()) * d ** -0.5
            if case["softcap"]:
                score = case["softcap"] * torch.tanh(score / case["softcap"])
            if hidden is not None:
                score.masked_fill_(hidden, -math.inf)
            top = score.amax(-1, keepdim=True)
            p = torch.exp(score - top)
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p, v[h:h + step]) / total
            hs = o.shape[0]
            out[row:row + n, h * G:(h + hs) * G] = o.view(hs * G, n, d).transpose(0, 1).to(out.dtype)
            lse[row:row + n, h * G:(h + hs) * G] = (top + torch.log(total)).view(hs * G, n).T
        row += n
    return out, lse


def _plain_logprobs(st):
    case, n = st["case"], st["case"]["top"]
    R, V = case["rows"], case["vocab"]
    outs = []
    for r in range(0, R, 512):  # rows at a time
        x = st["logits"][r:r + 512].float()
        if case["exclude"]:
            x[:, V - 1] = -math.inf
        top = x.amax(1, keepdim=True)
        e = torch.exp(x - top)
        total = e.sum(1, keepdim=True)
        # a token of probability zero adds nothing to the entropy
        moment = torch.where(e > 0, (x - top) * e, 0.0).sum(1, keepdim=True)
        log_total = torch.log(total)
        tokens = st["tokens"][r:r + 512].long()[:, None]
        logprob = torch.gather(x, 1, tokens) - top - log_total
        o = [logprob[:, 0], (log_total - moment / total)[:, 0]]
        if n:
            # distinct keys that order by value and then by lowest token
            bits = (x + 0.0).view(torch.int32)
            order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
            key = (order << 32) | (0xFFFFFFFF - torch.arange(V, device="cuda"))
            ids = 0xFFFFFFFF - (torch.topk(key, n, 1).values & 0xFFFFFFFF)
            o += [ids.to(torch.int32), torch.gather(x, 1, ids) - top - log_total]
        outs.append(o)
    return tuple(torch.cat(c) for c in zip(*outs))


# -------------------------------------------------------------- 64-bit results
def exact(case, seed):
    b = _inputs(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "logprobs": _exact_logprobs}[
        case["op"]](case, b)


def _exact_append(case, b):
    Hq, Hkv, d = LAYOUTS[case["layout"]]
    x = b["qkv"].double().view(b["rows"], -1, d)
    place = torch.tensor([(s, p) for s, (n, m) in enumerate(b["lens"]) for p in range(m - n, m)],
                         device="cuda")
    # rotation of the pair (j, j + d / 2) as a product of complex numbers
    freq = torch.exp(-math.log(THETA) * torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    angle = place[:, 1:].double() * freq
    turn = torch.complex(torch.cos(angle), torch.sin(angle))[:, None]

    def turned(y, w):
        if w is not None:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / d + EPS) * w.double()
        z = torch.complex(y[..., :d // 2].contiguous(), y[..., d // 2:].contiguous()) * turn
        return torch.cat([z.real, z.imag], -1)

    q = turned(x[:, :Hq], b["q_norm"])
    k, v = turned(x[:, Hq:Hq + Hkv], b["k_norm"]), x[:, Hq + Hkv:]
    kp, vp = b["k_pages"].double(), b["v_pages"].double()
    flat = b["table"].long()[place[:, 0], place[:, 1] // case["page"]] * case["page"] + place[:, 1] % case["page"]
    for pool, new in ((kp, k), (vp, v)):
        rows = pool.transpose(1, 2).reshape(-1, Hkv, d)
        rows[flat] = new
        pool.copy_(rows.view(pool.shape[0], case["page"], Hkv, d).transpose(1, 2))
    return q, kp, vp


def _exact_attend(case, b):
    Hq, Hkv, d = LAYOUTS[case["layout"]]
    out = torch.empty((b["rows"], Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((b["rows"], Hq), dtype=torch.float64, device="cuda")
    if work(case)["flops"] > 4e12:
        return None
    first = 0
    for s, (n, m) in enumerate(b["lens"]):
        ids = b["table"][s].tolist()[:-(-m // case["page"])]
        for h in range(Hkv):
            k, v = (torch.cat([p[i, h] for i in ids])[:m].double() for p in (b["k_pages"], b["v_pages"]))
            for r in range(0, n, 2048):
                rows = min(2048, n - r)
                pos = torch.arange(m - n + r, m - n + r + rows, device="cuda")[:, None]
                key = torch.arange(m, device="cuda")[None, :]
                c = case["block"]
                seen = key // c <= pos // c if c else None
                for g in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                    sc = b["q"][first + r:first + r + rows, g].double() @ k.T / math.sqrt(d)
                    if case["softcap"]:
                        sc = torch.tanh(sc / case["softcap"]) * case["softcap"]
                    if seen is not None:
                        sc = torch.where(seen, sc, -math.inf)
                    z = torch.logsumexp(sc, 1)
                    out[first + r:first + r + rows, g] = torch.exp(sc - z[:, None]) @ v
                    lse[first + r:first + r + rows, g] = z
        first += n
    return out, lse


def _exact_logprobs(case, b):
    outs, n = [], case["top"]
    for r in range(0, case["rows"], 128):
        x = b["logits"][r:r + 128].double()
        if case["exclude"]:
            x[:, case["vocab"] - 1] = -math.inf
        lp = x - torch.logsumexp(x, 1, keepdim=True)
        p = torch.exp(lp)
        o = [lp[torch.arange(lp.shape[0], device="cuda"), b["tokens"][r:r + 128].long()],
             -torch.where(p > 0, p * lp, 0.0).sum(1)]
        if n:
            ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :n]
            o += [ids.to(torch.int32), torch.gather(lp, 1, ids)]
        outs.append(o)
    return tuple(torch.cat(c) for c in zip(*outs))
