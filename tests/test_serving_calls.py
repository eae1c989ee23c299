"""Calls of the serving operators that the host refuses or answers without a launch
(pointers here are never dereferenced)."""
import pytest
import torch

import test_serving_api as api


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
