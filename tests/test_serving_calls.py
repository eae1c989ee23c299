"""Calls of the serving operators that the host refuses or answers without a launch
(pointers here are never dereferenced)."""
import importlib.util
import os
import random

import pytest
import torch

import test_serving_api as api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lp():
    import paper_2512_16229_amd as lp
    return lp


@pytest.mark.parametrize("ids,logprobs", [(None, (3, 4)), ((3, 4), None), ((3, 0), (3, 4)), ((3, 4), (3, 0)),
                                          ((3, 2), (3, 4)), (None, (3, 0))])
def test_binding_takes_the_top_list_whole(lp, ids, logprobs):
    """One array of the top list without the other, or of another width, is no call without a list."""
    ids = None if ids is None else torch.zeros(ids, dtype=torch.int32)
    logprobs = None if logprobs is None else torch.zeros(logprobs)
    with pytest.raises(ValueError, match="top_ids and top_logprobs"):
        lp.lopa_token_logprobs(torch.zeros(3, 5), None, -1, top_ids=ids, top_logprobs=logprobs)


@pytest.mark.parametrize("src", ["paged_append.hip", "paged_attention.hip", "logprobs.hip"])
def test_compiled_with_nan_semantics(src):
    """The kernels hand a NaN on to the rows that see it, so none of their sources is compiled under
    the assumption that there is none."""
    spec = importlib.util.spec_from_file_location(
        "lopa_build", os.path.join(ROOT, "paper_2512_16229_amd", "build.py"))
    b = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(b)
    flags = b.FLAGS + b.EXTRA_FLAGS.get(src, [])
    assert src in b.SOURCES
    assert not {"-ffast-math", "-ffinite-math-only", "-fno-honor-nans", "-Ofast"} & set(flags)


# ------------------------------------------------ grids of 32-bit work-items
def test_attention_of_more_work_than_a_launch_holds(lp):
    """Sequences x K / V heads past 2^24 workgroups of 256 threads: refused before anything is
    enqueued, by the workspace's size as by the call; just below it has a plan."""
    f = lp.lib.lopa_paged_attention_workspace
    assert f(512, 512, 64, 65535, 65535, 1, 100) == -2
    p, b = api.pages(lp, kv_heads=512), api.batch(lp, n_seq=65535, rows=65535)
    assert api.attend(lp, p, b, heads=512, ldq=512 * 64, ldo=512 * 64, max_rows=1) == -2, lp.lib.lopa_last_error()
    assert f(256, 256, 64, 65535, 65535, 1, 100) == 0
    assert f(1024, 1, 64, 65535, 1 << 20, 64, 100) >= 0


def test_attention_splits_keys_within_a_launch(lp):
    """Joining takes a workgroup per row: with 2^24 rows keys are not split."""
    f = lp.lib.lopa_paged_attention_workspace
    assert f(1, 1, 64, 2, (1 << 24) - 1, (1 << 24) - 2, 100000) > 0
    assert f(1, 1, 64, 2, 1 << 24, (1 << 24) - 1, 100000) == 0


def test_logprobs_rows(lp):
    """Fewer than 2^24 rows; the parts of a row leave that many workgroups."""
    f = lp.lib.lopa_token_logprobs_workspace
    assert f(1 << 24, 100, 0) == -2 and api.logprobs(lp, rows=1 << 24) == -2
    assert f((1 << 24) - 1, 100, 0) == 0
    assert f((1 << 22) + 1, 30000, 0) < 12 * (1 << 24)  # 12 bytes a part


# ----------------------------------------------------------------- empty batches
def test_no_rows_need_no_arrays(lp):
    """An empty batch is nothing to do, whichever arrays are null (empty tensors have no address)."""
    none = dict(x=None, tokens=None, lo=None, en=None, ids=None, tl=None, ws=None, size=0)
    assert api.logprobs(lp, rows=0, **none) == 0, lp.lib.lopa_last_error()
    assert api.logprobs(lp, rows=0, ids=None, tl=None) == 0
    empty = dict(q=None, out=None, b=api.batch(lp, rows=0))
    assert api.attend(lp, **empty, ws=None, size=0) == 0 and api.append(lp, **empty, k=None, v=None) == 0
    assert api.logprobs(lp, rows=0, n=33) == -2 and api.logprobs(lp, rows=0, exclude=100) == -1


# ----------------------------------------------------------------- shared memory
# (rows, elements between the starts, row strides): heads of 64 elements, four of them
SHARED = [(5, 0, 256, 256), (5, 128, 256, 256), (5, -128, 256, 256), (5, 4 * 256 + 248, 256, 256),
          (5, 1000, 1024, 1024 + 8), (1, 248, 4096, 256), (3, 2 * 1024, 1024, 1024), (5, 1024 + 248, 512, 512),
          (5, 3 * 512, 512, 2048), (7, -3 * 512 - 8, 2048, 512)]


@pytest.mark.parametrize("rows,shift,ld_a,ld_b", SHARED)
def test_shared_memory_is_refused(lp, rows, shift, ld_a, ld_b):
    """Attention reads q in several workgroups while others write out, and append reads a row's keys
    and values in other wavefronts than those that write its queries."""
    a, b = 0x100000, 0x100000 + 2 * shift
    batch = api.batch(lp, rows=rows)
    kw = dict(b=batch, max_rows=rows)
    assert api.attend(lp, q=a, ldq=ld_a, out=b, ldo=ld_b, **kw) == -1
    assert b"share memory" in lp.lib.lopa_last_error()
    assert api.attend(lp, q=b, ldq=ld_b, out=a, ldo=ld_a, **kw) == -1
    far = dict(heads=4, p=api.pages(lp, kv_heads=4), b=batch)
    x, y, z = 0x10000000, 0x20000000, 0x30000000
    assert api.append(lp, q=x, k=a, ldk=ld_a, v=z, ldv=256, out=b, ldo=ld_b, **far) == -1
    assert b"shares memory" in lp.lib.lopa_last_error()
    assert api.append(lp, q=x, k=y, ldk=256, v=b, ldv=ld_b, out=a, ldo=ld_a, **far) == -1
    if shift or (ld_a != ld_b and rows > 1):
        assert api.append(lp, q=a, ldq=ld_a, k=y, ldk=256, v=z, ldv=256, out=b, ldo=ld_b, **far) == -1


def test_shared_memory_is_refused_anywhere(lp):
    """Views of one buffer at random places, against a search of all pairs of rows."""
    rng, found = random.Random(3), 0
    for _ in range(4000):
        rows, shift = rng.randint(1, 9), 8 * rng.randint(-500, 500)
        ld_a, ld_b = (8 * rng.randint(32, 150) for _ in range(2))
        if rng.random() < 0.5:
            ld_b = ld_a
        if any(abs(i * ld_a - shift - j * ld_b) < 256 for i in range(rows) for j in range(rows)):
            found += 1
            assert api.attend(lp, q=0x100000, ldq=ld_a, out=0x100000 + 2 * shift, ldo=ld_b, max_rows=rows,
                              b=api.batch(lp, rows=rows)) == -1, (rows, shift, ld_a, ld_b)
    assert found > 1000


def test_shared_memory_in_place_with_another_stride(lp):
    assert api.append(lp, q=0x100000, ldq=256, k=0x20000000, v=0x30000000, out=0x100000, ldo=264) == -1


# ----------------------------------------------------------------- scale and cap
@pytest.mark.parametrize("scale,cap", [(2.0 ** 101, 0.0), (-2.5e38, 0.0), (0.1, 2.0 ** 101), (0.1, 3e38),
                                       (0.1, 2.0 ** -101), (0.0, 1e-40), (2.0 ** 60, 2.0 ** -60)])
def test_scores_out_of_range(lp, scale, cap):
    """Factors that leave fp32 made a score of 0 a NaN (0 x infinity)."""
    q, out = 0x100000, 0x200000
    assert api.attend(lp, scale=scale, cap=cap, q=q, out=out) == -1
    assert b"2^100" in lp.lib.lopa_last_error()
