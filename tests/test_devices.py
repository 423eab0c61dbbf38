"""Arrays that are not where the hidden states are, and hidden states that are not on a GPU: the binding refuses them before any launch.  Every array in turn is a tensor
of another device, which has no memory."""
import numpy as np
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


# ------------------------------------------------------------------------------------------------ the calls that were there before
def policy_logprobs(a):
    return binding._native().policy_logprobs(a["H"], a["W"], a["ids"], a["rowsel"], True, a["ws"], 0)


def policy_logprobs_static(a):
    return binding._native().policy_logprobs_static(a["H"], a["W"], a["ids"], a["rowsel"], a["logp"], a["lse"], a["entropy"], 0)


def ppo_loss(a):
    return binding._native().ppo_loss(a["H"], a["W"], a["ids"], a["rowsel"], a["logp_old"], a["adv"], a["role"], 0, 0.2, 0.0, 0.0, False, 0, a["logp_ref"], 0.0, a["dW"], a["dH"],
                                      a["logp"], a["stats"], a["ws"], 0)


def values(a):
    return binding._native().values(a["H"], a["w"], 0.0, a["rowsel"], a["value"], 0)


def value_loss(a):
    return binding._native().value_loss(a["H"], a["w"], 0.0, a["rowsel"], a["value_old"], a["ret"], a["role"], 0, 0.2, False, False, 0, a["dH"], a["dw"], a["db"], a["value"], a["stats"],
                                        a["ws"], 0)


SHAPES = dict(H=((6, 16), B), W=((40, 16), B), ids=((6,), I), rowsel=((6,), I), logp_old=((6,), F), adv=((6,), F), role=((6,), I), logp_ref=((6,), F), dW=((40, 16), F), dH=((6, 16), B),
              logp=((6,), F), lse=((6,), F), entropy=((6,), F), stats=((64,), U8), ws=((1 << 20,), U8), w=((16,), F), value=((6,), F), value_old=((6,), F), ret=((6,), F), dw=((16,), F),
              db=((1,), F))
USED = [(policy_logprobs, "W ids rowsel ws"), (policy_logprobs_static, "W ids rowsel logp lse entropy"), (ppo_loss, "W ids rowsel logp_old adv role logp_ref dW dH logp stats ws"),
        (values, "w rowsel value"), (value_loss, "w rowsel value_old ret role dH dw db value stats ws")]


@pytest.mark.parametrize("call", [call for call, _ in USED])
def test_scores_updates_and_critic_of_the_host(lib, call):  # noqa: F811
    for device in ("meta", "cpu"):
        with pytest.raises(ValueError, match="GPU"):
            call({n: torch.empty(*shape, dtype=t, device=device) for n, (shape, t) in SHAPES.items()})


@pytest.mark.gpu
@pytest.mark.parametrize("call,name", [(call, n) for call, names in USED for n in names.split()])
def test_scores_updates_and_critic(call, name):
    """One array elsewhere, of a device that has no memory."""
    a = {n: torch.zeros(*shape, dtype=t, device="meta" if n == name else "cuda") for n, (shape, t) in SHAPES.items()}
    with pytest.raises(ValueError, match="device"):
        call(a)


def assign(mask, **kw):
    a = dict(n_roles=1, n_models=1, role_to_model=[0], traj_turn_off=[0, 1], turn_role=[0], turn_tok_off=[0, 5], mask=mask, turn_pred_off=None, turn_pred=None, traj_group=None,
             role_reward=None, turn_reward=None, traj_reward=None, w_role=None, w_turn=None, w_traj=None, place_mode=0, norm_eps=1e-6, stream=0)
    return binding._native().assign(*{**a, **kw}.values())


def streams(**kw):
    tensors_ = [torch.zeros(2 if n.endswith("_off") else 5, dtype=torch.int64) for n in STREAMS]
    return umas.Streams(5, 1, 1, *[kw.get(n, t) for n, t in zip(STREAMS, tensors_)])


STREAMS = ["model_tok_off", "perm", "tok_turn", "tok_role", "tok_mask", "tok_reward", "turn_seg_off", "seg_turn", "model_turn_off", "traj_seg_off", "model_trajrun_off", "rowsel",
           "model_rowsel_off", "turn_scalar", "turn_step", "tok_flags"]


def front(native, s, value, arrays):
    x, y, mask, role, out = arrays
    off = np.array([0, 1], np.int32)
    return [lambda: native.advantages(s, value, 1.0, 1.0, 1.0, 0, 0), lambda: native.ready_batch(s, off, 0, 1, None, None, 0), lambda: native.ready_batch(s, off, 1, 1, None, None, 0),
            lambda: native.ready_batch(s, off, 2, 5, None, None, 0), lambda: native.kl_rewards(x, y, y, mask, 0.1, out, 0),
            lambda: native.whiten(x, mask, role, np.array([0, 5]), 1, 1, 1e-8, out, 0)]


def test_routing_rewards_and_batches(lib):  # noqa: F811
    """On the host: refused at the latest for the workspace.  One array elsewhere: by name."""
    native = binding._native()
    five = lambda dtype, dev="cpu": torch.zeros(5, dtype=dtype, device=dev)  # noqa: E731
    host = (five(F), five(F), five(U8), five(I), five(F))
    assert assign(five(U8), role_to_model=np.array([0], np.int32), traj_turn_off=np.array([0, 1], np.int32), turn_role=np.array([0], np.int32), turn_tok_off=np.array([0, 5])) == -4
    for call in front(native, streams(), five(F), host):
        assert call() == -4
    for name in STREAMS:
        for call in front(native, streams(**{name: five(torch.int64, "meta")}), None, host)[:4]:
            with pytest.raises(ValueError, match="device"):
                call()
    with pytest.raises(ValueError, match="device"):
        front(native, streams(), five(F, "meta"), host)[0]()
    for i in range(5):
        arrays = list(host)
        arrays[i] = five(arrays[i].dtype, "meta")
        for q, used in ((4, (0, 1, 2, 4)), (5, (0, 2, 3, 4))):
            if i in used:
                with pytest.raises(ValueError, match="device"):
                    front(native, streams(), None, arrays)[q]()
