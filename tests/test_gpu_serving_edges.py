"""The serving operators at the edges of what their header promises."""
import math
import random

import pytest
import torch

import serving_ref as ref
from test_paged_plan import FORMS
from test_gpu_serving import BF, HF, VARIANTS, attend, check_attend, randn, score, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lp():
    import paper_2512_16229_amd as lp
    return lp


# ------------------------------------------------------------------- attention
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("lens,heads,kv_heads,d", [([(1, 5000)], 4, 1, 128), ([(1, 70000)], 2, 2, 64),
                                                   ([(700, 9000)], 2, 1, 128)])
def test_values_seen_far_below_the_maximum(lp, what, lens, heads, kv_heads, d):
    """A key that a row sees has its part however far its score lies below the largest: key 0 scores
    about 220, the others 0. A NaN in a later key makes the row NaN, an infinite value of V is not
    lost (its weight e^-220 is no zero; as an fp32 factor it is, and the product NaN)."""
    (n, m), = lens
    b = ref.Batch(lens, 64, kv_heads, d, BF, 5)
    b.k.zero_()
    q = randn(3, (1, 1, d), BF).expand(n, heads, d).contiguous()
    page = b.table[0, 0].long()
    b.k[page, :, 0] = q[0, 0] * (220 * d ** 0.5 / q[0, 0].float().square().sum()).to(BF)
    out, lse = attend(lp, b, q, 1)
    v0 = b.v[page, :, 0].repeat_interleave(heads // kv_heads, 0)  # the other weights are below 9000 e^-200
    ref.close(out, v0.double().expand_as(out), 2.0 ** -7 * v0.abs().double())
    assert torch.isfinite(lse).all() and (lse > 200).all()
    p = m - n - 1 if n > 1 else m - 1  # seen by every row
    at = b.table[0, p // 64].long()
    pool = b.k if what == "k" else b.v
    pool[at, :, p % 64, 3] = math.nan if what == "k" else math.inf
    out, lse = attend(lp, b, q, 1)
    if what == "k":
        assert torch.isnan(out).all() and torch.isnan(lse).all()
    else:
        assert not torch.isfinite(out[..., 3]).any()
        rest = [i for i in range(d) if i != 3]
        assert torch.isfinite(out[..., rest]).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype,page,block,softcap", [(BF, 64, 1, 0.0), (HF, 32, 7, 0.0), (BF, 16, 0, 20.0),
                                                      (HF, 128, 1, 20.0)])
def test_attention_forms(lp, form, dtype, page, block, softcap):
    """Every kernel form that a batch's sizes can choose (the launches are checked on the host by the
    same table), in both types, with and without a cap."""
    lens, heads, kv_heads, d, _ = FORMS[form]
    b = ref.Batch(lens, page, kv_heads, d, dtype, 41, fill=math.nan)
    q = randn(8, (b.rows, heads, d), dtype, 1.5)
    check_attend(lp, b, q, block, softcap)


@pytest.mark.parametrize("shape", VARIANTS)
@pytest.mark.parametrize("dtype,page,block,softcap", [(HF, 16, 1, 20.0), (BF, 128, 32, 0.0)])
def test_attention_variants_without_tail(lp, shape, dtype, page, block, softcap):
    """The shapes of test_attention_variants without rows behind the last sequence, which make other
    launches of some of them."""
    lens, heads, kv_heads, d = VARIANTS[shape]
    b = ref.Batch(lens, page, kv_heads, d, dtype, 33, fill=math.nan)
    q = randn(9, (b.rows, heads, d), dtype, 1.5)
    check_attend(lp, b, q, block, softcap)


@pytest.mark.parametrize("scale,softcap", [(0.0, 0.0), (0.0, 30.0), (-0.2, 0.0), (-0.2, 5.0), (1.0, 2.0), (2.0 ** -100, 0.0),
                                           (0.125, 2.0 ** -90), (0.125, 2.0 ** 90), (0.125, 1e6)])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (HF, 64)])
def test_scales_and_caps(lp, scale, softcap, dtype, d):
    """Scales that are zero, negative or tiny, caps far from the scores."""
    b = ref.Batch([(1, 1500), (40, 90), (0, 3), (3, 33)], 32, 2, d, dtype, 7, fill=math.nan)
    q = randn(3, (b.rows, 6, d), dtype, 0.5)
    q[:, 0] = 0  # scores of 0
    out, lse = attend(lp, b, q, 1, softcap, scale=scale)
    want, wlse, tol, ltol = ref.attention(b, q, 1, scale, softcap)
    # ref's bound counts 8 U32 of the cap for the quotient, whose error is bounded by the cap's own
    # slope too: |capped| <= |s|, 8 U32 of which the products' bound (d + 4) U32 covers
    if softcap > 1000:
        _, _, tol, ltol = ref.attention(b, q, 1, scale, 0.0)
    ref.close(out, want, tol)
    ref.close(lse, wlse, ltol)


def test_empty_batches(lp):
    """No rows, with and without sequences: the calls return, and nothing changes."""
    i32 = dict(dtype=torch.int32, device="cuda")
    for n_seq in (0, 2):
        b = ref.Batch([(1, 20), (1, 30)], 16, 2, 64, BF, 3)
        k0, v0 = b.k.clone(), b.v.clone()
        args = (b.table[:n_seq], torch.zeros(n_seq + 1, **i32), b.kv_len[:n_seq])
        q, kv = (torch.empty((0, h, 64), dtype=BF, device="cuda") for h in (4, 2))
        lp.lopa_paged_append(b.k, b.v, *args, q, kv, kv, None, None, 0.0, 1e4, torch.empty_like(q))
        lp.lopa_paged_attention(q, b.k, b.v, *args, 0, 30, 1, 0.125, 0.0, torch.empty_like(q),
                                torch.empty((0, 4), device="cuda"))
        assert torch.equal(b.k, k0) and torch.equal(b.v, v0)
    for n in (0, 3):
        f = lambda *s: torch.empty(s, device="cuda")
        lp.lopa_token_logprobs(f(0, 100), torch.empty(0, **i32), -1, f(0), f(0),
                               torch.empty((0, n), **i32), f(0, n))


def test_views_of_one_buffer(lp):
    """q and out as views of one buffer that interleave without sharing an element: the result of
    separate arrays, and nothing else of the buffer changes."""
    b = ref.Batch([(3, 40), (1, 700), (4, 4)], 16, 2, 64, BF, 3)
    q = randn(5, (b.rows, 4, 64), BF)
    want, _ = attend(lp, b, q)
    ws = workspace(lp, 4, 2, 64, 3, b.rows, 4, 700)
    rng, found, width = random.Random(4), 0, 256
    for _ in range(400):
        ld_q, ld_o = (8 * rng.randint(32, 150) for _ in range(2))
        if rng.random() < 0.6:
            ld_o = ld_q
        at_q, at_o = (8 * rng.randint(0, 200) for _ in range(2))
        if any(abs(at_q + i * ld_q - at_o - j * ld_o) < width for i in range(b.rows) for j in range(b.rows)):
            continue
        found += 1
        store = torch.full((12000,), 7.0, dtype=BF, device="cuda")
        view = lambda at, ld: store.as_strided((b.rows, 4, 64), (ld, 64, 1), at)
        view(at_q, ld_q).copy_(q)
        left = store.clone()
        lp.lopa_paged_attention(view(at_q, ld_q), b.k, b.v, b.table, b.q_start, b.kv_len, 4, 700, 1, 0.125, 0.0,
                                view(at_o, ld_o), None, ws)
        left.as_strided((b.rows, 4, 64), (ld_o, 64, 1), at_o).copy_(want)
        assert torch.equal(store, left), (ld_q, ld_o, at_q, at_o)
    assert found > 50


# -------------------------------------------------------------------- logprobs
def logprob_bounds(x, exclude):
    """What the kernel's arithmetic allows (logprob, entropy and the 64-bit mean and variance behind
    them), with U = 2^-24:
    * a term 2^d, d = x log2 e - r, is off by |d| ln 2 U from the rounding of d, by a step (2 U) from
      the exponential and |d| U from that of log2 e; each change of reference multiplies by a power
      rounded like a term and rounds the product: 4 U, and once more |d| ln 2 U, all changes together
      (they add up to at most |d|). There are at most the segments' changes and 4 of the joins.
    * sums: 32 terms of a segment, the segments, 6 + 4 + 6 + 4 steps of the joins.
    So S is off by (K + 3 E|d|) U relative, d in nats. The sum of d 2^d has these errors times |d|,
      and 2 |d| U and 3 |d| U more for the products and for d; over S, whose error comes once more:
      K (1 + 2 E|d|) + 8 E|d| + 6 E d^2.
    * ln S and the value's own difference add 8 U of their size each."""
    x = x.double().clone()
    if exclude >= 0:
        x[:, exclude] = -math.inf
    V = x.shape[1]
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    p = e / e.sum(1, keepdim=True)
    dist = torch.where(p > 0, m - x, 0.0)
    mean, square = (p * dist).sum(1), (p * dist * dist).sum(1)
    segments = V // 4096 + 5  # 1024 vectors a segment, of 4 elements at least
    K = 32 + segments + 20 + 4 * (segments + 4) + 4
    U = ref.U32
    return (K + 3 * mean) * U, (K * (1 + 2 * mean) + 8 * mean + 6 * square) * U


@pytest.mark.parametrize("dtype", [BF, HF, torch.float32])
@pytest.mark.parametrize("rows,vocab,std,shift", [(3, 1000, 1.0, 0.0), (2, 152064, 3.0, 0.0), (300, 8191, 3.0, 50.0),
                                                  (40, 30000, 0.01, -500.0), (1100, 20001, 8.0, 3.0)])
def test_logprobs_accuracy(lp, dtype, rows, vocab, std, shift):
    """Within what the sums' depths allow: some 1e-5, not the order of any sum of the row's terms."""
    x = (randn(vocab, (rows, vocab), torch.float32, std) + shift).to(dtype)
    tokens = torch.randint(0, vocab, (rows,), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    tokens = tokens.to(torch.int32)
    tokens[::2] = x[::2].float().argmax(1).to(torch.int32)
    n, exclude = 8, vocab // 3
    tokens[tokens == exclude] = 0
    lo, en, ids, tl = score(lp, x, tokens, exclude, n)
    wl, we, wi, wt, _ = ref.logprobs(x, tokens, exclude, n)
    bound, ebound = logprob_bounds(x, exclude)
    assert bound.max() < 5e-5
    assert torch.equal(ids, wi)
    ref.close(lo, wl, bound + 8 * ref.U32 * wl.abs())
    ref.close(tl, wt, bound[:, None] + 8 * ref.U32 * wt.abs())
    ref.close(en, we, ebound + 8 * ref.U32 * we.abs())


# ------------------------------------------------------------------- batch tables
@pytest.mark.parametrize("starts", [[40, 0, 8, 20], [0, 40, 8, 20], [0, 8, 4, 20, 12, 30], [-3, 5, 60, 10], [0, 1, 30, 60, 2, 3],
                                    [0, 2, 40, 70, 3, 4, 5]])
@pytest.mark.parametrize("m", [100, 9000])
def test_starts_out_of_order(lp, starts, m):
    """q_start has to be in order. Where it is not the rows it names are undefined, but nothing lies
    outside the arrays: rows past every start stay as they are, and so do pages of no table."""
    n_seq, rows, hkv, d = len(starts) - 1, 70, 2, 64
    b = ref.Batch([(1, m)] * n_seq, 16, hkv, d, BF, 5)
    b.q_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    k0, v0 = b.k.clone(), b.v.clone()
    q, kv = randn(3, (rows, 8, d), BF), randn(4, (rows, hkv, d), BF)
    out = torch.full_like(q, 7.0)
    ws = workspace(lp, 8, hkv, d, n_seq, rows, rows, m)
    lp.lopa_paged_attention(q, b.k, b.v, b.table, b.q_start, b.kv_len, rows, m, 1, 0.125, 0.0, out, None, ws)
    assert (out[max(starts):] == 7).all()
    out.fill_(7.0)
    lp.lopa_paged_append(b.k, b.v, b.table, b.q_start, b.kv_len, q, kv, kv, None, None, 0.0, 1e4, out)
    assert (out[max(starts):] == 7).all()
    free = torch.ones(b.k.shape[0], dtype=torch.bool, device="cuda")
    free[b.table[b.table >= 0].long()] = False
    assert free.any() and torch.equal(b.k[free], k0[free]) and torch.equal(b.v[free], v0[free])


@pytest.mark.parametrize("form", ["64 rows", "tiles of 64, split", "tiles of 128", "tiles of 128, split, d 64",
                                  "two launches"])
def test_other_lengths_within_the_bounds(lp, form):
    """The launches are laid out for rows, max_rows and max_len: a captured call serves every batch
    within them. Here sequences shrink, empty and move, rows behind the last one stay."""
    lens, heads, kv_heads, d, _ = FORMS[form]
    rows, max_rows, max_len = sum(n for n, _ in lens), max(n for n, _ in lens), max(m for _, m in lens)
    rng = random.Random(7)
    for shrink in (1, 3, 40):
        less = [(rng.randint(0, -(-n // shrink)), m) for n, m in lens]
        less = [(n, rng.randint(n, m)) for n, m in less]
        b = ref.Batch(less, 32, kv_heads, d, BF, 43, fill=math.nan)
        pad = torch.full((len(lens), -(-max_len // 32)), -1, dtype=torch.int32, device="cuda")
        pad[:, :b.table.shape[1]] = b.table[:, :pad.shape[1]]
        b.table = pad
        q = randn(10, (rows, heads, d), BF)
        check_attend(lp, b, q, 1, max_rows=max_rows, max_len=max_len)


# ---------------------------------------------------------------------- append
@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 2, 64), (5, 1, 128), (17, 17, 64)])
def test_append_one_norm(lp, which, heads, kv_heads, d):
    """A norm for the queries or the keys alone (heads of both kinds share a wavefront), the queries
    written in place in the packed rows that the keys and values lie in too."""
    b = ref.Batch([(5, 90), (0, 3), (1, 17)], 16, kv_heads, d, HF, 4)
    qkv = randn(9, (b.rows + 2, heads + 2 * kv_heads, d), HF, 2.0)
    before = qkv.clone()
    q, k, v = qkv.split([heads, kv_heads, kv_heads], 1)
    w = (1 + randn(1, (d,), torch.float32, 0.2)).to(HF)
    norms = (w, None) if which == "q" else (None, w)
    wq, tq, wk, tk = ref.append(b, q.clone(), k, v, *norms, 1e-6, 1e4)
    lp.lopa_paged_append(b.k, b.v, b.table, b.q_start, b.kv_len, q, k, v, *norms, 1e-6, 1e4, q)
    ref.close(q[:b.rows], wq, tq)
    assert torch.equal(qkv[:, heads:], before[:, heads:]) and torch.equal(qkv[b.rows:], before[b.rows:])
    for row, (s, p) in enumerate([(0, i) for i in range(85, 90)] + [(2, 16)]):
        page = b.table[s, p // 16].long()
        ref.close(b.k[page, :, p % 16], wk[row], tk[row])
        assert torch.equal(b.v[page, :, p % 16], v[row])


@pytest.mark.parametrize("heads,kv_heads", [(1024, 1), (1024, 1024), (1024, 8), (1, 1)])
def test_many_heads(lp, heads, kv_heads):
    b = ref.Batch([(1, 40), (3, 5), (2, 600)], 32, kv_heads, 64, BF, 4, fill=math.nan)
    q, kv = randn(3, (b.rows, heads, 64), BF, 1.5), randn(4, (b.rows, kv_heads, 64), BF)
    out = torch.empty_like(q)
    lp.lopa_paged_append(b.k, b.v, b.table, b.q_start, b.kv_len, q, kv, kv, None, None, 0.0, 1e4, out)
    wq, tq, _, _ = ref.append(b, q, kv, kv, None, None, 0.0, 1e4)
    ref.close(out, wq, tq)
    check_attend(lp, b, q, 1)


def test_shared_pages(lp):
    """Branches of one prefix: the same pages in several tables, full and causal."""
    n, m, ps = 3, 150, 32
    b = ref.Batch([(9, m)] * n, ps, 2, 128, BF, 4, fill=math.nan)
    share = (m - 9) // ps
    b.table[1:, :share] = b.table[0, :share]
    q = randn(3, (b.rows, 8, 128), BF)
    for block in (0, 1):
        out, _ = check_attend(lp, b, q, block)
    q[9:] = q[:9].repeat(2, 1, 1)
    for s in range(1, n):  # the same new tokens: the same answers
        for p in range(share, -(-m // ps)):
            b.k[b.table[s, p].long()], b.v[b.table[s, p].long()] = b.k[b.table[0, p].long()], b.v[b.table[0, p].long()]
    out, lse = attend(lp, b, q, 1)
    assert torch.equal(out[9:], out[:9].repeat(2, 1, 1)) and torch.equal(lse[9:], lse[:9].repeat(2, 1))


def test_two_streams_at_once(lp):
    """The same pages read by two streams, each with its own outputs and workspace."""
    b = ref.Batch([(1, 5000), (40, 900)], 64, 2, 128, BF, 4)
    q = randn(3, (b.rows, 8, 128), BF)
    want = attend(lp, b, q)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [(torch.empty_like(q), torch.empty((b.rows, 8), device="cuda"),
            workspace(lp, 8, 2, 128, 2, b.rows, 40, 5000)) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(10):
        for st, (out, lse, ws) in zip(streams, got):
            lp.lopa_paged_attention(q, b.k, b.v, b.table, b.q_start, b.kv_len, 40, 5000, 1, 128 ** -0.5, 0.0, out,
                                    lse, ws, stream=st)
    torch.cuda.synchronize()
    for out, lse, _ in got:
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
