"""Calls of the serving operators that the host refuses or answers without a launch
(pointers here are never dereferenced)."""
import importlib.util
import os

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
