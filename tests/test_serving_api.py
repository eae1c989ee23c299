"""The serving operators refuse what they do not take on the host, before any HIP call
(pointers here are never dereferenced)."""
import ctypes as C

import pytest
import torch

FAKE = 0x1000


@pytest.fixture(scope="module")
def lp():
    import paper_2512_16229_amd as lp
    return lp


def pages(lp, **over):
    p = lp.lopa_pages(FAKE, FAKE, 10, 2, 16, 64, lp.LOPA_BF16)
    for k, v in over.items():
        setattr(p, k, v)
    return p


def batch(lp, **over):
    b = lp.lopa_paged_batch(FAKE, FAKE, FAKE, 2, 8, 5)
    for k, v in over.items():
        setattr(b, k, v)
    return b


def append(lp, p=None, b=None, heads=4, q=FAKE, ldq=256, k=FAKE, ldk=128, v=FAKE, ldv=128, qn=None, kn=None,
           eps=1e-6, theta=1e4, out=FAKE, ldo=256):
    p, b = p or pages(lp), b or batch(lp)
    return lp.lib.lopa_paged_append(C.byref(p), C.byref(b), heads, q, ldq, k, ldk, v, ldv, qn, kn, eps, theta,
                                    out, ldo, None)


def attend(lp, p=None, b=None, heads=4, max_rows=5, max_len=100, q=FAKE, ldq=256, block=1, scale=0.1, cap=0.0,
           out=FAKE, ldo=256, lse=None, ws=FAKE, size=1 << 40):
    p, b = p or pages(lp), b or batch(lp)
    return lp.lib.lopa_paged_attention(C.byref(p), C.byref(b), heads, max_rows, max_len, q, ldq, block, scale, cap,
                                       out, ldo, lse, ws, size, None)


BAD_PAGED = [
    (dict(dtype=2), {}, -1), (dict(dtype=-1), {}, -1), (dict(head_dim=96), {}, -2), (dict(head_dim=0), {}, -2),
    (dict(kv_heads=3), {}, -2), (dict(kv_heads=0), {}, -2), (dict(page_size=8), {}, -2),
    (dict(page_size=48), {}, -2), (dict(page_size=512), {}, -2), (dict(n_pages=0), {}, -1), (dict(k=None), {}, -1),
    (dict(v=None), {}, -1), (dict(k=FAKE + 2), {}, -1), (dict(v=FAKE + 8), {}, -1), ({}, dict(n_seq=-1), -2),
    ({}, dict(n_seq=65536), -2), ({}, dict(rows=-1), -2), ({}, dict(rows=(1 << 24) + 1), -2),
    ({}, dict(table=None), -1), ({}, dict(q_start=None), -1), ({}, dict(kv_len=None), -1),
    ({}, dict(table_ld=0), -2), ({}, dict(table_ld=1 << 26), -2)]


@pytest.mark.parametrize("po,bo,code", BAD_PAGED)
def test_paged_refusals(lp, po, bo, code):
    assert append(lp, pages(lp, **po), batch(lp, **bo)) == code, lp.lib.lopa_last_error()
    assert attend(lp, pages(lp, **po), batch(lp, **bo)) == code, lp.lib.lopa_last_error()
    assert lp.lib.lopa_last_error()


def test_paged_null_structs(lp):
    f = lp.lib.lopa_paged_append
    assert f(None, C.byref(batch(lp)), 4, FAKE, 256, FAKE, 128, FAKE, 128, None, None, 0, 0, FAKE, 256, None) == -1
    assert f(C.byref(pages(lp)), None, 4, FAKE, 256, FAKE, 128, FAKE, 128, None, None, 0, 0, FAKE, 256, None) == -1


@pytest.mark.parametrize("over,code", [
    (dict(heads=0), -2), (dict(heads=5), -2), (dict(heads=2048), -2), (dict(q=None), -1), (dict(k=None), -1),
    (dict(v=None), -1), (dict(out=None), -1), (dict(q=FAKE + 4), -1), (dict(out=FAKE + 2), -1),
    (dict(ldq=255), -1), (dict(ldq=260), -1), (dict(ldq=248), -1), (dict(ldk=0), -1), (dict(ldv=-128), -1),
    (dict(ldo=250), -1), (dict(eps=-1.0, qn=FAKE), -1), (dict(eps=float("nan"), kn=FAKE), -1),
    (dict(theta=-1.0), -1), (dict(theta=float("inf")), -1), (dict(qn=FAKE + 2), -1)])
def test_append_refusals(lp, over, code):
    assert append(lp, **over) == code, lp.lib.lopa_last_error()


@pytest.mark.parametrize("over,code", [
    (dict(heads=3), -2), (dict(max_rows=-1), -1), (dict(max_len=-1), -1), (dict(max_len=129), -3),
    (dict(block=-1), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(cap=-1.0), -1),
    (dict(cap=float("nan")), -1), (dict(q=None), -1), (dict(out=None), -1), (dict(q=FAKE + 8), -1),
    (dict(ldq=250), -1), (dict(ldo=128), -1)])
def test_attention_refusals(lp, over, code):
    assert attend(lp, **over) == code, lp.lib.lopa_last_error()


def test_attention_workspace(lp):
    """The workspace is asked for where the keys are split, and a smaller one is refused."""
    f = lp.lib.lopa_paged_attention_workspace
    assert f(4, 2, 96, 1, 1, 1, 100) == -2 and f(4, 3, 64, 1, 1, 1, 100) == -2
    assert f(4, 2, 64, -1, 1, 1, 100) == -2 and f(4, 2, 64, 1, 1, -1, 100) == -1
    assert f(4, 2, 64, 1, 1, 1, 1 << 30) == -2
    assert f(4, 2, 64, 0, 0, 0, 0) == 0
    need = f(4, 2, 64, 1, 1, 1, 100000)
    if need:
        p, b = pages(lp, n_pages=10000), batch(lp, n_seq=1, rows=1, table_ld=10000)
        kw = dict(p=p, b=b, max_rows=1, max_len=100000)
        assert attend(lp, size=need - 1, **kw) == -2
        assert attend(lp, size=need, ws=None, **kw) == -1
        assert attend(lp, size=need, ws=FAKE + 4, **kw) == -1


def test_nothing_to_do(lp):
    """No rows or no sequences: fine, and nothing is launched."""
    for b in (batch(lp, rows=0), batch(lp, n_seq=0), batch(lp, rows=0, n_seq=0, table=None, q_start=None)):
        assert append(lp, b=b) == 0 and attend(lp, b=b) == 0
    assert attend(lp, max_rows=0) == 0
    assert logprobs(lp, rows=0) == 0


def logprobs(lp, x=FAKE, dtype=2, ld=100, rows=3, vocab=100, exclude=-1, tokens=FAKE, n=4, lo=FAKE, en=FAKE,
             ids=FAKE, tl=FAKE, ws=FAKE, size=1 << 40):
    return lp.lib.lopa_token_logprobs(x, dtype, ld, rows, vocab, exclude, tokens, n, lo, en, ids, tl, ws, size, None)


@pytest.mark.parametrize("over,code", [
    (dict(x=None), -1), (dict(x=FAKE + 2), -1), (dict(x=FAKE + 1, dtype=0), -1), (dict(dtype=3), -1),
    (dict(dtype=-1), -1), (dict(ld=99), -1), (dict(ld=0), -1), (dict(rows=-1), -2), (dict(vocab=0), -2),
    (dict(vocab=(1 << 24) + 1, ld=1 << 25), -2), (dict(exclude=-2), -1), (dict(exclude=100), -1),
    (dict(n=-1), -2), (dict(n=33), -2), (dict(tokens=None), -1), (dict(lo=None), -1), (dict(ids=None), -1),
    (dict(tl=None), -1), (dict(n=0), -1)])
def test_logprobs_refusals(lp, over, code):
    assert logprobs(lp, **over) == code, lp.lib.lopa_last_error()


def test_logprobs_workspace(lp):
    f = lp.lib.lopa_token_logprobs_workspace
    assert f(-1, 5, 0) == -2 and f(1, 0, 0) == -2 and f(1, 5, 33) == -2 and f(0, 5, 3) == 0
    need = f(1, 152064, 5)
    if need:
        kw = dict(rows=1, vocab=152064, ld=152064, n=5)
        assert logprobs(lp, size=need - 1, **kw) == -2
        assert logprobs(lp, size=need, ws=None, **kw) == -1
        assert logprobs(lp, size=need, ws=FAKE + 8, **kw) == -1


def test_binding_refuses_host_tensors(lp):
    t = torch.zeros
    i = lambda *s: t(s, dtype=torch.int32)
    pool, q = t((2, 1, 16, 64), dtype=torch.bfloat16), t((3, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        lp.lopa_paged_attention(q, pool, pool, i(1, 2), i(2), i(1), 3, 16, 1, 1.0, 0.0, q)
    with pytest.raises(ValueError, match="device tensor"):
        lp.lopa_paged_append(pool, pool, i(1, 2), i(2), i(1), q, q, q, None, None, 0.0, 0.0, q)
    with pytest.raises(ValueError, match="device tensor"):
        lp.lopa_token_logprobs(t((3, 5)), None, -1, entropy=t(3))
    with pytest.raises(lp.LopaError):
        lp.lopa_paged_attention_workspace(4, 3, 64, 1, 1, 1, 1)
    with pytest.raises(lp.LopaError):
        lp.lopa_token_logprobs_workspace(1, 0, 0)
