"""The serving operators (paged append, attention over pages, token log probabilities)
against 64-bit forms, over layouts, types, lengths, masks and strides."""
import math

import pytest
import torch

import serving_ref as ref
import synth

pytestmark = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
I32 = torch.int32


@pytest.fixture(scope="module")
def lp():
    import paper_2512_16229_amd as lp
    return lp


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(seed, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * std).to(dtype)


def workspace(lp, heads, kv_heads, d, n_seq, rows, max_rows, max_len, fill=0xFF):
    n = lp.lopa_paged_attention_workspace(heads, kv_heads, d, n_seq, rows, max_rows, max_len)
    return torch.full((n,), fill, dtype=torch.uint8, device="cuda") if n else None


def attend(lp, b, q, block=1, softcap=0.0, scale=None, max_rows=None, max_len=None):
    rows, heads, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    max_rows, max_len = max_rows or b.max_rows, max_len or b.max_len
    out = torch.full_like(q, 7.0)
    lse = torch.full((rows, heads), 7.0, device="cuda")
    ws = workspace(lp, heads, b.k.shape[1], d, len(b.lens), rows, max_rows, max_len)
    lp.lopa_paged_attention(q, b.k, b.v, b.table, b.q_start, b.kv_len, max_rows, max_len, block, scale,
                            softcap, out, lse, ws)
    return out, lse


def check_attend(lp, b, q, block=1, softcap=0.0, **kw):
    out, lse = attend(lp, b, q, block, softcap, **kw)
    want, wlse, tol, ltol = ref.attention(b, q, block, q.shape[2] ** -0.5, softcap)
    n = b.rows
    ref.close(out[:n], want[:n], tol[:n])
    ref.close(lse[:n], wlse[:n], ltol[:n])
    # rows behind the last sequence stay as they were
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()
    return out, lse


LENS = {
    "one": [(1, 1)],
    "token": [(1, 700)],
    "tokens": [(1, 33), (1, 1), (1, 512), (1, 64), (1, 1000)],
    "block": [(32, 300), (32, 32), (32, 95)],
    "prompt": [(333, 333)],
    "chunk": [(130, 1200), (257, 300)],
    "mixed": [(70, 500), (1, 900), (0, 40), (3, 3), (1, 2), (0, 0), (17, 65)],
}


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 2, 64), (28, 4, 128), (6, 6, 128), (16, 1, 64)])
@pytest.mark.parametrize("dtype,page,block", [(BF, 16, 1), (HF, 64, 0), (BF, 256, 32), (HF, 32, 7)])
def test_attention(lp, lens, heads, kv_heads, d, dtype, page, block):
    # unwritten slots hold NaN: no row may see them
    b = ref.Batch(LENS[lens], page, kv_heads, d, dtype, 11, fill=math.nan)
    q = randn(3, (b.rows, heads, d), dtype, 1.5)
    check_attend(lp, b, q, block)


@pytest.mark.parametrize("lens", ["tokens", "chunk", "mixed"])
@pytest.mark.parametrize("dtype,softcap", [(BF, 5.0), (HF, 50.0)])
def test_attention_softcap(lp, lens, dtype, softcap):
    b = ref.Batch(LENS[lens], 64, 4, 128, dtype, 5, fill=math.nan)
    q = randn(4, (b.rows, 8, 128), dtype, 6.0)
    check_attend(lp, b, q, 1, softcap)


@pytest.mark.parametrize("std", [0.01, 0.3, 3.0, 30.0])
def test_attention_softcap_relative(lp, std):
    """Scores far below the cap keep their relative accuracy: one key, whose lse is the capped score
    (a sum of d products, a factor, the series or the quotient: within (d + 24) U32 of sum |q k|)."""
    b = ref.Batch([(1, 1)] * 40, 16, 1, 64, HF, 5)
    q = randn(4, (40, 2, 64), HF, std)
    _, lse = attend(lp, b, q, 1, 50.0)
    k = b.k[b.table[:, 0].long(), 0, 0].double()
    s = (q.double() * k[:, None]).sum(-1) / 8
    mag = (q.double() * k[:, None]).abs().sum(-1) / 8
    want = 50 * torch.tanh(s / 50)
    # past TINY of the cap the quotient's error counts against the cap. An fp16 numerator is
    # 2^(8 + d), d the rounding of the reference (score - 8: at most half a step of 8 to 16, 2^-21):
    # an exponential and a logarithm of 2^-23 relative each, on values within 2^-21 of 2^8 and 1,
    # bring 2^-22 / ln 2 into log2 l, and so 2^-22 into lse
    ref.close(lse, want, (64 + 24) * ref.U32 * mag + torch.where(s.abs() > 15, 8 * ref.U32 * 50, 0.0) + 2 ** -22)


@pytest.mark.parametrize("m", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1023, 4097])
@pytest.mark.parametrize("n", [1, 5, 40])
def test_attention_lengths(lp, m, n):
    b = ref.Batch([(min(n, m), m)], 16, 2, 128, BF, m, fill=math.inf)
    q = randn(m, (b.rows, 8, 128), BF, 1.5)
    check_attend(lp, b, q, 1)


@pytest.mark.parametrize("rows_seq", [1, 2, 8, 9, 16, 33])
@pytest.mark.parametrize("heads,kv_heads", [(4, 1), (7, 1), (48, 8), (40, 1)])
def test_attention_row_tiles(lp, rows_seq, heads, kv_heads):
    b = ref.Batch([(rows_seq, 200 + 3 * s) for s in range(3)], 32, kv_heads, 128, BF, rows_seq, fill=math.nan)
    q = randn(6, (b.rows, heads, 128), BF)
    check_attend(lp, b, q, 1)


@pytest.mark.parametrize("n,m", [(1, 40000), (64, 20001), (700, 9000)])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_long(lp, n, m, d):
    b = ref.Batch([(n, m)], 128, 1, d, BF, 9, fill=math.nan)
    q = randn(8, (n, 2, d), BF, 1.5)
    check_attend(lp, b, q, 1)


# What the launch plan makes of a batch goes by its sizes: these reach the tiles of 64 and of 128
# rows, whole and with split keys, one and several of a sequence, and two launches in one call.
VARIANTS = {
    "64 rows": ([(64, 1000)] * 32, 8, 8, 128),
    "64 rows, d 64": ([(64, 1000)] * 32, 8, 8, 64),
    "tiles of 64, split": ([(700, 9000)], 2, 1, 128),
    "tiles of 64, split, d 64": ([(900, 12000)], 4, 1, 64),
    "tiles of 128": ([(300, 300)] * 16, 28, 4, 128),
    "tiles of 128, d 64": ([(300, 300)] * 16, 28, 4, 64),
    "tiles of 128, split": ([(700, 8300)], 8, 2, 128),
    "tiles of 128, split, d 64": ([(1500, 9000)], 8, 2, 64),
    "two launches": ([(1600, 2500)] + [(1, 60 * s + 1) for s in range(38)] + [(2, 2)], 16, 4, 128),
    "two launches, d 64": ([(1, 55 * s + 1) for s in range(69)] + [(4000, 4000)], 12, 4, 64),
}


@pytest.mark.parametrize("shape", VARIANTS)
@pytest.mark.parametrize("dtype,page,block,softcap", [(BF, 16, 1, 0.0), (HF, 128, 32, 0.0), (BF, 64, 0, 20.0)])
def test_attention_variants(lp, shape, dtype, page, block, softcap):
    lens, heads, kv_heads, d = VARIANTS[shape]
    b = ref.Batch(lens, page, kv_heads, d, dtype, 31, fill=math.nan)
    q = randn(7, (b.rows + 2, heads, d), dtype, 1.5)
    check_attend(lp, b, q, block, softcap)


@pytest.mark.parametrize("shape", ["64 rows", "tiles of 64, split", "tiles of 128", "tiles of 128, split, d 64"])
def test_attention_variants_missing_and_hidden(lp, shape):
    """Missing pages, and values that are not finite in keys some rows see and some do not."""
    lens, heads, kv_heads, d = VARIANTS[shape]
    b = ref.Batch(lens, 32, kv_heads, d, BF, 32)
    q = randn(7, (b.rows, heads, d), BF)
    n, m = lens[0]
    b.table[0, 1] = -1
    b.table[0, 5] = 10 ** 8
    clean, clse = check_attend(lp, b, q, 1)
    at = m - n // 2  # rows of the sequence before n - n // 2 do not see it
    page, slot = b.table[0, at // 32].long(), at % 32
    b.v[page, :, slot, 3] = math.inf
    b.v[page, :, slot, 60] = math.nan
    out, lse = attend(lp, b, q, 1)
    k = n - n // 2
    assert torch.equal(out[:k], clean[:k]) and torch.equal(lse, clse)
    assert (out[k:n, :, 3] == math.inf).all() and torch.isnan(out[k:n, :, 60]).all()
    rest = [i for i in range(d) if i not in (3, 60)]
    # the other values travel with the key's as before
    ref.close(out[k:n][..., rest], clean[k:n][..., rest], 0.0)
    assert torch.equal(out[n:], clean[n:])


@pytest.mark.parametrize("m", [500, 700, 1000, 1500, 3000, 70000])
@pytest.mark.parametrize("heads,kv_heads,d", [(8, 2, 64), (28, 4, 128), (1, 1, 64)])
def test_attention_parts(lp, m, heads, kv_heads, d):
    """One token whose keys are split over few and many workgroups, with scores far below zero
    (a joined part's reference is not near 0)."""
    b = ref.Batch([(1, m), (1, m // 2)], 64, kv_heads, d, BF, m, fill=math.nan)
    q = randn(6, (2, heads, d), BF, 2.0)
    b.k = torch.where(torch.isnan(b.k), b.k, b.k * 0.2 - 1.0 * q[0, 0].sign() * (heads == 1))
    check_attend(lp, b, q, 1)


def test_attention_peaked(lp):
    """The largest score comes first, last or in the middle, far above the rest."""
    b = ref.Batch([(1, 900), (40, 900)], 64, 2, 128, BF, 2)
    q = randn(8, (b.rows, 4, 128), BF, 4.0)
    for s, at in ((0, 0), (1, 3), (1, 500), (0, 899)):
        page, slot = b.table[s, at // 64].long(), at % 64
        b.k[page, :, slot] = b.k[page, :, slot] * 6
    check_attend(lp, b, q, 0)


@pytest.mark.parametrize("where", [-1, 10 ** 6])
def test_attention_missing_pages(lp, where):
    """Pages that are not there are not seen: some, the first, and all of a sequence."""
    b = ref.Batch([(1, 500), (40, 300), (20, 100), (1, 70)], 16, 2, 64, BF, 4, fill=math.nan)
    b.table[0, 3:9] = where
    b.table[0, 20] = where
    b.table[1, 0] = where
    b.table[2, :] = where
    b.table[3, :] = where
    q = randn(5, (b.rows, 4, 64), BF)
    out, lse = check_attend(lp, b, q, 1)
    assert (out[41:61] == 0).all() and (lse[41:61] == -math.inf).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("n,m", [(1, 500), (3, 70), (200, 500)])
def test_attention_hidden_values(lp, bad, n, m):
    """K and V rows that a row does not see have no part in it: a causal row whose later
    rows of the same sequence are not finite, in the same key tile and behind it."""
    b = ref.Batch([(n, m)], 32, 2, 128, BF, 21)
    q = randn(5, (n, 4, 128), BF)
    clean, clse = attend(lp, b, q, 1)
    hit = m - n // 2  # rows before this position do not see it
    for p in range(hit, m):
        page, slot = b.table[0, p // 32].long(), p % 32
        b.v[page, :, slot] = bad
        b.k[page, :, slot, ::3] = bad
    out, lse = attend(lp, b, q, 1)
    k = n - n // 2
    assert torch.equal(out[:k], clean[:k]) and torch.equal(lse[:k], clse[:k])


@pytest.mark.parametrize("n,m", [(1, 300), (150, 300)])
def test_attention_seen_values(lp, n, m):
    """A value that is not finite is seen by the rows that may see it, in its dimension."""
    b = ref.Batch([(n, m)], 32, 1, 128, BF, 22)
    q = randn(5, (n, 2, 128), BF)
    at = m - n + n // 3 if n > 1 else m - 1
    page, slot = b.table[0, at // 32].long(), at % 32
    b.v[page, 0, slot, 5] = math.inf
    b.v[page, 0, slot, 77] = -math.inf
    b.v[page, 0, slot, 100] = math.nan
    out, _ = attend(lp, b, q, 1)
    first = at - (m - n)
    assert torch.isfinite(out[:first]).all()
    assert (out[first:, :, 5] == math.inf).all() and (out[first:, :, 77] == -math.inf).all()
    assert torch.isnan(out[first:, :, 100]).all()
    rest = [i for i in range(128) if i not in (5, 77, 100)]
    assert torch.isfinite(out[:, :, rest]).all()


@pytest.mark.parametrize("n,m", [(1, 300), (150, 300), (1, 5000)])
@pytest.mark.parametrize("what", ["k", "q"])
def test_attention_nan_scores(lp, n, m, what):
    """A NaN score reaches the rows that see it, and no other."""
    b = ref.Batch([(n, m), (2, 40)], 32, 1, 128, BF, 23)
    q = randn(5, (n + 2, 2, 128), BF)
    at = n // 3 if n > 1 else 0  # row of sequence 0
    if what == "k":
        p = m - n + at
        b.k[b.table[0, p // 32].long(), 0, p % 32, 7] = math.nan
        bad = torch.arange(n, device="cuda") >= at
    else:
        q[at, :, 9] = math.nan
        bad = torch.arange(n, device="cuda") == at
    out, lse = attend(lp, b, q, 1)
    assert torch.isnan(out[:n][bad]).all() and torch.isnan(lse[:n][bad]).all()
    assert torch.isfinite(out[:n][~bad]).all() and torch.isfinite(lse[:n][~bad]).all()
    assert torch.isfinite(out[n:]).all()


@pytest.mark.parametrize("heads,kv_heads,d", [(4, 2, 64), (28, 4, 128)])
@pytest.mark.parametrize("block", [0, 1, 4])
def test_attention_more_rows_than_keys(lp, heads, kv_heads, d, block):
    """Rows at positions before 0 see nothing unless the attention is full; no keys at all."""
    b = ref.Batch([(5, 3), (40, 7), (3, 0), (2, 20)], 16, kv_heads, d, BF, 3, fill=math.nan)
    q = randn(5, (b.rows, heads, d), BF)
    out, lse = check_attend(lp, b, q, block)
    assert (out[45:48] == 0).all() and (lse[45:48] == -math.inf).all()


@pytest.mark.parametrize("n_seq", [63, 64, 65, 130, 2000])
def test_many_sequences(lp, n_seq):
    """Batches of many short sequences, some without rows, one long: attention and append find
    each row's own."""
    lens = [((i * 7) % 4, 3 + i % 50) for i in range(n_seq)]
    lens[n_seq // 3] = (150, 160)
    b = ref.Batch(lens, 16, 1, 64, BF, 3)
    q = randn(5, (b.rows, 2, 64), BF)
    check_attend(lp, b, q, 1)
    kv = randn(6, (b.rows, 1, 64), BF)
    out = torch.empty_like(q)
    lp.lopa_paged_append(b.k, b.v, b.table, b.q_start, b.kv_len, q, kv, kv, None, None, 0.0, 0.0, out)
    assert torch.equal(out, q)
    seq = torch.tensor([s for s, (n, m) in enumerate(lens) for _ in range(n)], device="cuda")
    pos = torch.tensor([p for n, m in lens for p in range(m - n, m)], device="cuda")
    page = b.table[seq, pos // 16].long()
    assert torch.equal(b.k[page, :, pos % 16], kv) and torch.equal(b.v[page, :, pos % 16], kv)


def test_rows_before_the_first_sequence(lp):
    """q_start need not begin at 0: rows before it stay as they are."""
    b = ref.Batch([(2, 30), (33, 50)], 16, 2, 64, BF, 3)
    q = randn(5, (b.rows, 4, 64), BF)
    want, wlse = attend(lp, b, q)
    q5 = torch.cat([q[:5], q])
    b.q_start += 5
    out, lse = attend(lp, b, q5)
    assert torch.equal(out[5:], want) and torch.equal(lse[5:], wlse) and (out[:5] == 7).all()
    got = torch.full_like(q5, 7.0)
    kv = randn(6, (b.rows + 5, 2, 64), BF)
    lp.lopa_paged_append(b.k, b.v, b.table, b.q_start, b.kv_len, q5, kv, kv, None, None, 0.0, 0.0, got)
    assert torch.equal(got[5:], q) and (got[:5] == 7).all()
    assert torch.equal(b.v[b.table[0, 1].long(), :, 13], kv[6])  # row 6: position 29 of sequence 0


def test_append_more_rows_than_tokens(lp):
    """Rows at positions before 0 have no slot: their queries are rotated, nothing is written."""
    b = ref.Batch([(4, 20)], 16, 2, 64, HF, 3)
    b.kv_len[0] = 2
    q, kv = randn(1, (4, 4, 64), HF), randn(2, (4, 2, 64), HF)
    k0 = b.k.clone()
    out = torch.empty_like(q)
    lp.lopa_paged_append(b.k, b.v, b.table, b.q_start, b.kv_len, q, kv, kv, None, None, 0.0, 1e4, out)
    b.lens = [(4, 2)]
    wq, tq, wk, tk = ref.append(b, q, kv, kv, None, None, 0.0, 1e4)
    ref.close(out, wq, tq)
    page = b.table[0, 0].long()
    ref.close(b.k[page, :, :2].transpose(0, 1), wk[2:], tk[2:])
    b.k[page, :, :2] = k0[page, :, :2]
    assert torch.equal(b.k, k0)


def test_attention_strides_and_tail(lp):
    """q and out as views of wider rows; rows behind the last sequence stay as they were."""
    b = ref.Batch(LENS["mixed"], 32, 2, 64, BF, 3, fill=math.nan)
    wide = randn(5, (b.rows + 6, 4 + 4, 64), BF)
    q = wide[:, :4]
    check_attend(lp, b, q.contiguous(), 1)
    store = torch.full((b.rows + 6, 3, 4, 64), 7.0, dtype=BF, device="cuda")
    out = store[:, 1]
    ws = workspace(lp, 4, 2, 64, len(b.lens), b.rows + 6, b.max_rows, b.max_len)
    lp.lopa_paged_attention(q, b.k, b.v, b.table, b.q_start, b.kv_len, b.max_rows, b.max_len, 1, 0.125, 0.0,
                            out, None, ws)
    want, _, tol, _ = ref.attention(b, q, 1, 0.125, 0.0)
    ref.close(out[:b.rows], want[:b.rows], tol[:b.rows])
    assert (out[b.rows:] == 7).all() and (store[:, 0] == 7).all() and (store[:, 2] == 7).all()


def test_attention_bounds_skip(lp):
    """A sequence past max_rows or max_len is left out, the others are not touched by it."""
    b = ref.Batch([(5, 40), (9, 30), (2, 90)], 16, 2, 64, BF, 3)
    q = randn(5, (b.rows, 4, 64), BF)
    out, lse = attend(lp, b, q, max_rows=5, max_len=64)
    want, wlse, tol, ltol = ref.attention(b, q, 1, 0.125, 0.0)
    ref.close(out[:5], want[:5], tol[:5])
    assert (out[5:] == 7).all() and (lse[5:] == 7).all()
    wide, _ = attend(lp, b, q, max_rows=16, max_len=96)  # looser bounds, all of them
    ref.close(wide, want, tol)


def test_attention_far_pages(lp):
    """Pages more than 2^32 elements into the pool."""
    n_pages, hkv, ps, d = 150000, 2, 128, 128
    k = torch.empty((n_pages, hkv, ps, d), dtype=BF, device="cuda")
    v = torch.empty_like(k)
    assert k.numel() > 2 ** 32
    b = ref.Batch([(3, 200), (1, 700)], ps, hkv, d, BF, 3)
    far = torch.tensor([n_pages - 1 - i for i in range(b.k.shape[0])], dtype=I32, device="cuda")
    k[far.long()], v[far.long()] = b.k, b.v
    small = attend(lp, b, q := randn(5, (b.rows, 4, d), BF))
    b.k, b.v = k, v
    b.table = torch.where(b.table >= 0, far[b.table.clamp(0).long()], b.table)
    big = attend(lp, b, q)
    assert torch.equal(small[0], big[0]) and torch.equal(small[1], big[1])
    qkv = randn(6, (b.rows, 4 + 2 * hkv, d), BF)
    lp.lopa_paged_append(k, v, b.table, b.q_start, b.kv_len, *qkv.split([4, hkv, hkv], 1), None, None, 0.0,
                         0.0, torch.empty_like(q))
    for s, (n, m) in enumerate(b.lens):
        for i in range(n):
            p = m - n + i
            page = b.table[s, p // ps].long()
            assert torch.equal(k[page, :, p % ps], qkv[b.start[s] + i, 4:4 + hkv])
            assert torch.equal(v[page, :, p % ps], qkv[b.start[s] + i, 4 + hkv:])


def test_attention_repeats_bitwise(lp):
    b = ref.Batch(LENS["mixed"] + [(1, 5000)], 16, 4, 128, BF, 3)
    q = randn(5, (b.rows, 28, 128), BF)
    first = attend(lp, b, q)
    for _ in range(3):
        again = attend(lp, b, q)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# ---------------------------------------------------------------------- append
@pytest.mark.parametrize("lens", ["one", "tokens", "mixed", "chunk"])
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 2, 64), (28, 4, 128), (3, 3, 128), (17, 1, 64)])
@pytest.mark.parametrize("dtype,page,norm,theta", [(BF, 16, True, 1e6), (HF, 128, False, 1e4),
                                                   (HF, 64, True, 0.0), (BF, 32, False, 0.0)])
def test_append(lp, lens, heads, kv_heads, d, dtype, page, norm, theta):
    b = ref.Batch(LENS[lens], page, kv_heads, d, dtype, 4)
    k0, v0 = b.k.clone(), b.v.clone()
    rows = b.rows + 3
    qkv = randn(9, (rows, heads + 2 * kv_heads, d), dtype, 2.0)
    q, k, v = qkv.split([heads, kv_heads, kv_heads], 1)
    qn = (1 + randn(1, (d,), F32, 0.2)).to(dtype) if norm else None
    kn = (1 + randn(2, (d,), F32, 0.2)).to(dtype) if norm else None
    out = torch.full((rows, heads, d), 7.0, dtype=dtype, device="cuda")
    lp.lopa_paged_append(b.k, b.v, b.table, b.q_start, b.kv_len, q, k, v, qn, kn, 1e-6, theta, out)
    wq, tq, wk, tk = ref.append(b, q, k, v, qn, kn, 1e-6, theta)
    ref.close(out[:b.rows], wq, tq)
    assert (out[b.rows:] == 7).all()
    row = 0
    for s, (n, m) in enumerate(b.lens):
        for p in range(m - n, m):
            page_id = b.table[s, p // page].long()
            ref.close(b.k[page_id, :, p % page], wk[row], tk[row] if torch.is_tensor(tk) else tk)
            assert torch.equal(b.v[page_id, :, p % page], v[row])
            k0[page_id, :, p % page] = b.k[page_id, :, p % page]
            v0[page_id, :, p % page] = v[row]
            row += 1
    assert torch.equal(b.k, k0) and torch.equal(b.v, v0)  # nothing else was written


@pytest.mark.parametrize("start", [0, 131071, 900000, 50_000_000])
def test_append_far_positions(lp, start):
    """The angle of a far position keeps its accuracy (the table's first pages are not there:
    only the queries come back)."""
    d, n = 128, 5
    i32 = dict(dtype=I32, device="cuda")
    table = torch.full((1, -(-(start + n) // 256)), -1, **i32)
    b = ref.Batch([(n, n)], 256, 1, d, HF, 3)
    b.lens = [(n, start + n)]
    q = randn(1, (n, 2, d), HF)
    kv = randn(2, (n, 1, d), HF)
    k0 = b.k.clone()
    out = torch.empty_like(q)
    lp.lopa_paged_append(b.k, b.v, table, torch.tensor([0, n], **i32), torch.tensor([start + n], **i32), q, kv,
                         kv, None, None, 0.0, 1e6, out)
    wq, tq, _, _ = ref.append(b, q, kv, kv, None, None, 0.0, 1e6)
    ref.close(out, wq, tq)
    assert torch.equal(b.k, k0)


def test_append_in_place_and_zero_rows(lp):
    b = ref.Batch([(3, 10)], 16, 2, 64, BF, 3)
    q, kv = randn(1, (3, 4, 64), BF), randn(2, (3, 2, 64), BF)
    q[1] = 0  # the norm of a zero head is zero
    want = torch.empty_like(q)
    w = torch.ones(64, dtype=BF, device="cuda")
    args = (b.k, b.v, b.table, b.q_start, b.kv_len)
    lp.lopa_paged_append(*args, q, kv, kv, w, w, 1e-6, 1e4, want)
    lp.lopa_paged_append(*args, q, kv, kv, w, w, 1e-6, 1e4, q)
    assert torch.equal(q, want) and (q[1] == 0).all()


# -------------------------------------------------------------------- logprobs
def score(lp, x, tokens=None, exclude=-1, n=0, entropy=True):
    R, V = x.shape
    f = lambda *s: torch.full(s, 7.0, device="cuda")
    lo = f(R) if tokens is not None else None
    en = f(R) if entropy else None
    ids = torch.full((R, n), 77, dtype=I32, device="cuda") if n else None
    tl = f(R, n) if n else None
    need = lp.lopa_token_logprobs_workspace(R, V, n)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") if need else None
    lp.lopa_token_logprobs(x, tokens, exclude, lo, en, ids, tl, ws)
    return lo, en, ids, tl


def check_score(lp, x, tokens, exclude, n):
    lo, en, ids, tl = score(lp, x, tokens, exclude, n)
    wl, we, wi, wt, rel = ref.logprobs(x, tokens, exclude, n)
    mag = lambda w: torch.where(torch.isfinite(w), w.abs(), 0.0)
    ref.close(lo, wl, rel + 8 * ref.U32 * mag(wl))
    ref.close(en, we, 2 * rel * (1 + mag(we)))
    if n:
        assert torch.equal(ids, wi)
        ref.close(tl, wt, rel[:, None] + 8 * ref.U32 * mag(wt))


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (2, 63), (5, 1000), (1, 8191), (2, 8193), (3, 16384),
                                        (7, 20001), (1, 152064), (300, 1025)])
@pytest.mark.parametrize("n,excl", [(0, False), (1, True), (5, False), (32, True)])
def test_logprobs(lp, dtype, rows, vocab, n, excl):
    x = randn(vocab, (rows, vocab), dtype, 3.0)
    tokens = torch.randint(0, vocab, (rows,), generator=gen(1), device="cuda").to(I32)
    tokens[0] = vocab - 1
    check_score(lp, x, tokens, vocab // 2 if excl else -1, n)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_logprobs_ties(lp, dtype):
    """Equal logits: the lowest tokens come first, over runs, whole rows and segment ends."""
    V = 30000
    x = torch.zeros((6, V), dtype=dtype, device="cuda")
    x[1, ::7] = 2.0
    x[2, 8180:8200] = 3.0
    x[2, 29999] = 3.0
    x[3] = torch.arange(V, device="cuda").remainder(5).to(dtype)
    x[4, ::2] = -0.0
    x[5] = torch.arange(V, device="cuda").to(F32).div(3000).to(dtype)  # ascending, equal runs in 16 bits
    tokens = torch.tensor([0, 1, 8180, -1, V, V - 1], dtype=I32, device="cuda")
    check_score(lp, x, tokens, -1, 32)
    check_score(lp, x, tokens, 0, 7)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [2, 1100])
def test_logprobs_ties_long(lp, dtype, rows):
    """More equal values than any buffer holds, in a long row and in rows that one workgroup has."""
    V = 150000 if rows == 2 else 70000
    x = torch.zeros((rows, V), dtype=dtype, device="cuda")
    x[1] = -3.0
    x[1, 5::1000] = 1.0
    tokens = torch.zeros(rows, dtype=I32, device="cuda")
    for n in (3, 32):
        lo, en, ids, tl = score(lp, x, tokens, -1, n)
        want = torch.arange(n, dtype=I32, device="cuda")
        assert torch.equal(ids[0], want) and torch.equal(ids[1], 5 + 1000 * want)
        assert (ids == want)[torch.arange(rows) != 1].all()
        assert ((tl[0] + math.log(V)).abs() < 1e-4).all() and ((en[0] - math.log(V)).abs() < 1e-4).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,vocab,n", [(1, 31, 32), (6, 300, 13), (2, 696, 13), (9, 1024, 20), (1100, 1024, 32)])
def test_logprobs_small_vocabularies(lp, dtype, rows, vocab, n):
    """More top tokens than the vocabulary has groups of logits: random rows, equal ones, one
    whose best lie side by side, one with fewer tokens left than asked for."""
    x = randn(rows + vocab, (max(rows, 5), vocab), dtype, 3.0)
    x[1] = 1.0
    x[2] = torch.arange(vocab, device="cuda").to(dtype)
    x[3] = -float("inf")
    x[3, 2:: max(vocab // 5, 1)] = 2.0
    x[4, vocab // 2 : vocab // 2 + 14] += 50.0
    tokens = torch.arange(x.shape[0], device="cuda").remainder(vocab).to(I32)
    check_score(lp, x, tokens, -1, n)
    check_score(lp, x, tokens, vocab // 2, n)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
def test_logprobs_masked_rows(lp, dtype):
    """Masks of -inf and of the type's lowest value, rows with nothing left, with one token,
    with a NaN or an infinity (which have no distribution)."""
    V = 9000
    x = randn(3, (11, V), dtype, 2.0)
    low = torch.finfo(dtype).min
    x[0] = -math.inf
    x[1] = -math.inf
    x[1, 8999] = -4.0
    x[2] = low
    x[3, :8990] = low
    x[4, 10:] = -math.inf
    x[5, 77] = math.nan
    x[6, 78] = math.inf
    x[7] = torch.finfo(dtype).max
    x[8] = -math.inf
    x[8, 100] = 1.0  # the excluded one
    x[9, 100] = math.nan  # excluded: no part
    x[10, ::2] = -math.inf
    tokens = torch.tensor([5, 8999, 3, 4, 20, 6, 78, 0, 100, 1, 2], dtype=I32, device="cuda")
    check_score(lp, x, tokens, 100, 12)
    check_score(lp, x, tokens, -1, 3)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
def test_logprobs_late_extremes(lp, dtype):
    """The largest logits, the type's largest, NaN runs and -inf runs late in a long row, after
    thousands of ordinary ones; one row of NaN only."""
    V = 70000
    x = randn(3, (6, V), dtype, 2.0)
    x[0, 69990:] = torch.arange(10, device="cuda").to(dtype) * 3 + 20
    x[1, 50000] = torch.finfo(dtype).max
    x[2, 40000:60000] = math.nan
    x[3, 20000:] = -math.inf
    x[4] = math.nan
    x[5, :69000] = -math.inf
    tokens = torch.tensor([69999, 50000, 1, 30000, 3, 69999], dtype=I32, device="cuda")
    check_score(lp, x, tokens, -1, 20)
    check_score(lp, x[:, 1:], tokens - 1, 69998, 3)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 5), (7, 1)])
def test_logprobs_strides(lp, dtype, offset, pad):
    """Rows that start at any element (odd vocabularies, views), and rows far apart."""
    V, R = 5003, 4
    store = randn(5, (R, V + offset + pad), dtype, 3.0)
    x = store[:, offset:offset + V]
    tokens = torch.tensor([0, V - 1, 17, 4000], dtype=I32, device="cuda")
    check_score(lp, x, tokens, 9, 20)


def test_logprobs_many_long_rows(lp):
    """Rows that one workgroup has each, with more groups of tokens than its LDS keeps maxima of."""
    R, V = 1100, 600001
    x = torch.empty((R, V), dtype=BF, device="cuda")
    for r in range(0, R, 100):
        x[r:r + 100] = randn(r, (100, V), BF, 3.0)
    tokens = torch.randint(0, V, (R,), generator=gen(1), device="cuda").to(I32)
    lo, en, ids, tl = score(lp, x, tokens, 7, 12)
    some = torch.tensor([0, 1, 513, 1098, 1099], device="cuda")
    wl, we, wi, wt, rel = ref.logprobs(x[some], tokens[some], 7, 12)
    ref.close(lo[some], wl, rel + 8 * ref.U32 * wl.abs())
    ref.close(en[some], we, 2 * rel * (1 + we.abs()))
    assert torch.equal(ids[some], wi)
    ref.close(tl[some], wt, rel[:, None] + 8 * ref.U32 * wt.abs())


def test_logprobs_far_rows(lp):
    """A row more than 2^32 elements behind the first."""
    V, ld = 4000, 2 ** 31 + 16
    store = torch.empty(2 * ld + V, dtype=BF, device="cuda")
    x = store.as_strided((3, V), (ld, 1))
    x.copy_(randn(5, (3, V), BF, 3.0))
    check_score(lp, x, torch.tensor([1, 2, 3], dtype=I32, device="cuda"), -1, 4)


def test_logprobs_each_output_alone(lp):
    x = randn(5, (9, 12345), BF, 3.0)
    tokens = torch.arange(9, dtype=I32, device="cuda")
    lo, en, ids, tl = score(lp, x, tokens, 3, 6)
    assert torch.equal(score(lp, x, tokens, 3, 0, entropy=False)[0], lo)
    assert torch.equal(score(lp, x, None, 3, 0)[1], en)
    _, none, i2, t2 = score(lp, x, None, 3, 6, entropy=False)
    assert none is None and torch.equal(i2, ids) and torch.equal(t2, tl)


# -------------------------------------------------------------------- together
def test_streams(lp):
    """The three calls on another stream than the current one, in its order."""
    b = ref.Batch([(3, 100), (1, 50)], 16, 2, 64, BF, 3)
    qkv = randn(1, (b.rows, 8, 64), BF)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    q = torch.empty((b.rows, 4, 64), dtype=BF, device="cuda")
    out = torch.empty_like(q)
    ws = workspace(lp, 4, 2, 64, 2, b.rows, 3, 100)
    lp.lopa_paged_append(b.k, b.v, b.table, b.q_start, b.kv_len, *qkv.split([4, 2, 2], 1), None, None, 0.0, 1e4,
                         q, stream=st)
    lp.lopa_paged_attention(q, b.k, b.v, b.table, b.q_start, b.kv_len, 3, 100, 1, 0.125, 0.0, out, None, ws,
                            stream=st)
    st.synchronize()
    want, _, tol, _ = ref.attention(b, q, 1, 0.125, 0.0)
    ref.close(out, want, tol)


def test_graph_replays(lp):
    """A captured step (append, attention, log probabilities) replayed while the lengths, pages
    and inputs change, against the eager calls on the same state."""
    n_seq, hkv, heads, d, ps, cap, V = 3, 2, 8, 128, 16, 640, 5000
    i32 = dict(dtype=I32, device="cuda")
    pages = n_seq * cap // ps
    order = torch.randperm(pages, generator=gen(2), device="cuda").to(I32).view(n_seq, -1)
    table = order.contiguous()
    k = randn(1, (pages, hkv, ps, d), BF)
    v = randn(2, (pages, hkv, ps, d), BF)
    q_start = torch.arange(n_seq + 1, **i32)
    kv_len = torch.tensor([5, 300, 77], **i32)
    qkv = randn(3, (n_seq, heads + 2 * hkv, d), BF)
    head = randn(4, (heads * d, V), F32, 0.02)
    wn = torch.ones(d, dtype=BF, device="cuda")

    def buffers():
        return dict(q=torch.empty((n_seq, heads, d), dtype=BF, device="cuda"),
                    out=torch.empty((n_seq, heads, d), dtype=BF, device="cuda"),
                    x=torch.empty((n_seq, V), device="cuda"), lo=torch.empty(n_seq, device="cuda"),
                    en=torch.empty(n_seq, device="cuda"), ids=torch.empty((n_seq, 4), **i32),
                    tl=torch.empty((n_seq, 4), device="cuda"),
                    ws=workspace(lp, heads, hkv, d, n_seq, n_seq, 1, cap, 0),
                    ws2=torch.empty(max(16, lp.lopa_token_logprobs_workspace(n_seq, V, 4)), dtype=torch.uint8,
                                    device="cuda"))

    tokens = torch.tensor([1, 2, 3], **i32)

    def step(o, kp, vp):
        lp.lopa_paged_append(kp, vp, table, q_start, kv_len, *qkv.split([heads, hkv, hkv], 1), wn, wn, 1e-6, 1e6,
                             o["q"])
        lp.lopa_paged_attention(o["q"], kp, vp, table, q_start, kv_len, 1, cap, 1, d ** -0.5, 0.0, o["out"], None,
                                o["ws"])
        torch.matmul(o["out"].view(n_seq, -1).float(), head, out=o["x"])
        lp.lopa_token_logprobs(o["x"], tokens, V - 1, o["lo"], o["en"], o["ids"], o["tl"], o["ws2"])

    g, e = buffers(), buffers()
    k2, v2 = k.clone(), v.clone()
    step(e, k2, v2)  # warm
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(st):
        step(g, k, v)
        st.synchronize()
        with torch.cuda.graph(graph, stream=st):
            step(g, k, v)
    torch.cuda.synchronize()
    for i in range(5):
        kv_len += torch.tensor([1, 50, 90], **i32)
        qkv.copy_(randn(40 + i, tuple(qkv.shape), BF))
        graph.replay()
        torch.cuda.synchronize()
        step(e, k2, v2)
        torch.cuda.synchronize()
        for name in ("q", "out", "lo", "en", "ids", "tl"):
            assert torch.equal(g[name], e[name]), (i, name)


def test_decode_as_used(lp):
    """Two sequences: their prompts enter in chunks, then tokens one at a time, causal; every
    step's attention equals the 64-bit attention of the rotated keys and values so far."""
    heads, hkv, d, ps = 4, 2, 64, 16
    i32 = dict(dtype=I32, device="cuda")
    steps = [(40, 7), (25, 0), (1, 60), (1, 1), (1, 1)]
    b = ref.Batch([(1, 128), (1, 128)], ps, hkv, d, BF, 5, fill=math.nan)
    w = (1 + randn(1, (d,), F32, 0.2)).to(BF)
    have = [0, 0]
    for i, new in enumerate(steps):
        rows = sum(new)
        qkv = randn(70 + i, (rows, heads + 2 * hkv, d), BF)
        have = [h + n for h, n in zip(have, new)]
        b.lens = list(zip(new, have))
        b.start = [0, new[0], rows]
        b.rows = rows
        b.q_start, b.kv_len = torch.tensor(b.start, **i32), torch.tensor(have, **i32)
        b.max_rows, b.max_len = max(new), max(have)
        q = torch.empty((rows, heads, d), dtype=BF, device="cuda")
        parts = qkv.split([heads, hkv, hkv], 1)
        lp.lopa_paged_append(b.k, b.v, b.table, b.q_start, b.kv_len, *parts, w, w, 1e-6, 1e4, q)
        wq, tq, _, _ = ref.append(b, *parts, w, w, 1e-6, 1e4)
        ref.close(q, wq, tq)
        check_attend(lp, b, q, 1)


def test_confidence_of_a_model(lp):
    """The verify forward's Conf and candidate are the top log probability and token of the
    logits: its residual rows through the final norm and the LM head, in 64 bits."""
    cfg = synth.config("tiny")
    w = synth.model_weights(cfg)
    from __graft_entry__ import _to_device_bf16
    wd = _to_device_bf16(w)
    model = lp.Model(cfg, wd)
    L, P = 16, 32
    kv = lp.KV(model, P + L, 1, L)
    dec = lp.Decoder(model, kv, L, 1, 0.9)
    dec.prefill(synth.prompt(cfg, P))
    tok = torch.full((L,), cfg["mask_id"], dtype=I32, device="cuda")
    conf, pred = torch.empty(L, device="cuda"), torch.empty(L, dtype=I32, device="cuda")
    lp.lopa_verify_forward(model, kv, P, tok, 1, L, conf, pred)
    x = torch.empty((L, cfg["hidden"]), device="cuda")
    lp.lopa_debug_hidden(model, kv, P, tok, 1, L, cfg["layers"], x)
    x = x.double()
    x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + cfg["rms_eps"]) * wd["final_norm"].double()
    logits = (x.to(BF).double() @ wd["lm_head"].double().T).float().contiguous()
    _, ent, ids, tl = score(lp, logits, None, cfg["mask_id"], 2)
    assert ((tl[:, 0].exp() - conf).abs() <= 1e-4).all()
    clear = tl[:, 0] - tl[:, 1] > 1e-3
    assert clear.any() and torch.equal(ids[clear, 0], pred[clear])
    assert (ent >= 0).all()
