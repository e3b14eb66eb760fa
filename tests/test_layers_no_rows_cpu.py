"""Calls without rows: what would point to nothing may be null; what is written all the same, and a workspace, may not."""
import pytest
import torch

import paper_1905_10936_amd as ef
from tests.test_layers_cpu import CALLS, call

NULL = ef.EF_ERR_NULL
# what no rows leave empty, by call
EMPTY = {"ef_act_encode": ("x", "act"), "ef_act_decode": ("y", "act"), "ef_norm_forward": ("x", "residual", "h", "y", "act", "rstd"),
         "ef_norm_backward": ("dy", "act", "rstd", "dh", "dx"), "ef_weight_grad": ("dz", "act"), "ef_token_logp": ("logits", "tokens", "logp"),
         "ef_policy_loss": ("logits", "tokens", "advantage", "token_weight", "logp", "losses", "dlogits")}


@pytest.mark.parametrize("name", EMPTY)
def test_null_is_nothing(name):
    assert set(EMPTY[name]) <= set(CALLS[name])
    if torch.cuda.is_available() and "ws" in CALLS[name]:
        pytest.skip("the addresses are made up")
    # those with a workspace look for its device next, and find none here
    assert call(name, rows=0, **{k: None for k in EMPTY[name]}) == (ef.EF_ERR_HIP if "ws" in CALLS[name] else ef.EF_OK)
    assert call(name, rows=-1, **{k: None for k in EMPTY[name]}) in (NULL, ef.EF_ERR_ARG)


@pytest.mark.parametrize("name,arg", [("ef_norm_backward", "ws"), ("ef_weight_grad", "ws"), ("ef_weight_grad", "dw"), ("ef_policy_loss", "ws")])
def test_what_is_needed_without_rows(name, arg):
    assert call(name, rows=0, **{k: None for k in EMPTY[name] + (arg,)}) == NULL


@pytest.mark.parametrize("name", EMPTY)
def test_the_other_arguments_are_checked(name):
    width = "vocab" if "vocab" in CALLS[name] else "width"
    for changes in (dict(type=9), {width: 0}):
        assert call(name, rows=0, **dict({k: None for k in EMPTY[name]}, **changes)) == ef.EF_ERR_ARG
