"""Arrays that are not where the hidden states are, and hidden states that are not on a GPU: the binding refuses them before any launch (no GPU).  Every array in turn is a tensor
of another device, which has no memory."""
import pytest
import torch

import paper_2605_26646_amd as umas
from paper_2605_26646_amd import binding
from tests.test_targets_host import lib, native_ce, native_distill, tensors  # noqa: F401  (a fixture)

B, F, I, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def away(*shape, dtype):
    return torch.empty(*shape, dtype=dtype, device="meta")


TAUGHT = [dict(W=away(40, 16, dtype=B)), dict(rowsel=away(6, dtype=I)), dict(weight=away(6, dtype=F)), dict(tok_role=away(6, dtype=I), n_roles=1), dict(dW=away(40, 16, dtype=F)),
          dict(dH=away(6, 16, dtype=B)), dict(row=away(6, dtype=F)), dict(stats=away(32, dtype=U8)), dict(workspace=away(1 << 20, dtype=U8)), dict(H=away(6, 16, dtype=B))]


@pytest.mark.parametrize("call,kw", [(call, kw) for call in (native_ce, native_distill) for kw in TAUGHT] +
                         [(native_ce, dict(ids=away(6, dtype=I))), (native_distill, dict(top_ids=away(6, 3, dtype=I))), (native_distill, dict(top_logits=away(6, 3, dtype=F))),
                          (native_distill, dict(lse=away(6, dtype=F)))])
def test_an_array_of_another_device(lib, call, kw):  # noqa: F811
    with pytest.raises(ValueError, match="device"):
        call(tensors(**kw))


@pytest.mark.parametrize("call", [native_ce, native_distill])
@pytest.mark.parametrize("workspace", [None, torch.empty(1 << 24, dtype=U8)])
def test_hidden_states_of_the_host(lib, call, workspace):  # noqa: F811
    with pytest.raises(ValueError, match="GPU"):
        call(tensors(workspace=workspace))


def native_top(H=None, W=None, rowsel=None, ids=None, logits=None, lse=None, ws=torch.empty(0, dtype=U8)):
    H, W = torch.zeros(6, 16, dtype=B) if H is None else H, torch.zeros(40, 16, dtype=B) if W is None else W
    return binding._native().top_logits(H, W, 3, rowsel, ids, logits, lse, ws, 0)


def test_largest_logits(lib):  # noqa: F811
    for kw in (dict(H=away(6, 16, dtype=B)), dict(W=away(40, 16, dtype=B)), dict(rowsel=away(6, dtype=I)), dict(ids=away(6, 3, dtype=I)), dict(logits=away(6, 3, dtype=F)),
               dict(lse=away(6, dtype=F)), dict(ws=away(1 << 20, dtype=U8))):
        with pytest.raises(ValueError, match="device"):
            native_top(**kw)
    for ws in (None, torch.empty(1 << 24, dtype=U8)):
        with pytest.raises(ValueError, match="GPU"):
            native_top(ws=ws)
    assert native_top() == -4
