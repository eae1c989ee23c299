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
