"""Workspace queries and refusals of the largest logits, cross entropy and distillation: decided on the host, before any launch (no GPU)."""
import os

import pytest
import torch

import paper_2605_26646_amd as umas
from paper_2605_26646_amd import binding

F32, BF16, NO_DW = 0, 1, -1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(umas.lib_path()):
        import __graft_entry__ as g
        g.build()
    return umas.load_library()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,V", [(0, 64, 300), (1, 64, 300), (64, 2048, 151936), (257, 3584, 1000), (5000, 64, 3001)])
def test_workspaces_grow_from_least_to_full(lib, n, d, V, dtype):
    assert 0 < lib.umas_top_logits_workspace_bytes_min(n, d, V, 40, dtype) <= lib.umas_top_logits_workspace_bytes(n, d, V, 40, dtype)
    for dw in (F32, BF16, NO_DW):
        least, full = (getattr(lib, "umas_cross_entropy_workspace_bytes" + w)(n, d, V, dtype, dw) for w in ("_min", ""))
        assert 0 < least <= full
        for k in (1, 64):
            least_k, full_k = (getattr(lib, "umas_distill_workspace_bytes" + w)(n, d, V, k, dtype, dw) for w in ("_min", ""))
            assert least <= least_k <= full_k and full <= full_k


def test_the_smallest_workspace_does_not_grow_with_the_rows_logits(lib):
    small, large = (lib.umas_cross_entropy_workspace_bytes_min(n, 2048, 151936, BF16, F32) for n in (1000, 16000))
    assert large - small < 0.05 * 2 * 15000 * 151936             # not a bf16 number per row and entry
    small, large = (lib.umas_top_logits_workspace_bytes_min(n, 2048, 151936, 64, BF16) for n in (1000, 100000))
    assert small == large


@pytest.mark.parametrize("n,d,V,k,dw", [(-1, 64, 300, 4, F32), (8, 0, 300, 4, F32), (8, 64, 0, 4, F32), (8, 64, 300, 0, F32), (8, 64, 300, 65, F32), (8, 64, 300, 4, 2),
                                        (8, 64, 300, 4, -2)])
def test_queries_about_impossible_sizes_are_zero(lib, n, d, V, k, dw):
    for w in ("_min", ""):
        assert getattr(lib, "umas_distill_workspace_bytes" + w)(n, d, V, k, BF16, dw) == 0
        if dw == F32:
            assert getattr(lib, "umas_top_logits_workspace_bytes" + w)(n, d, V, k, BF16) == 0


PLENTY = 1 << 40


def top(lib, **kw):
    a = dict(H=256, W=256, dtype=BF16, n_rows=4, d=64, V=300, rowsel=None, n_sel=4, k=4, ids=256, logits=256, lse=256, ws=256, ws_bytes=PLENTY, stream=None)
    return lib.umas_top_logits(*{**a, **kw}.values()), lib.umas_last_error().decode()


def ce(lib, **kw):
    a = dict(H=256, W=256, dtype=BF16, n_rows=4, d=64, V=300, ids=256, rowsel=None, n_sel=4, weight=None, tok_role=None, n_roles=0, z_coef=0.0, accumulate_dW=0,
             norm_rows=0, stats=256, logp=None, dH=256, dW=256, dW_type=F32, ws=256, ws_bytes=PLENTY, stream=None)
    return lib.umas_cross_entropy_fwd_bwd(*{**a, **kw}.values()), lib.umas_last_error().decode()


def distill(lib, **kw):
    a = dict(H=256, W=256, dtype=BF16, n_rows=4, d=64, V=300, ids=256, logits=256, k=4, teacher_lse=None, rowsel=None, n_sel=4, weight=None, tok_role=None, n_roles=0,
             accumulate_dW=0, norm_rows=0, stats=256, kl=None, dH=256, dW=256, dW_type=F32, ws=256, ws_bytes=PLENTY, stream=None)
    return lib.umas_distill_fwd_bwd(*{**a, **kw}.values()), lib.umas_last_error().decode()


SHARED = [(dict(dtype=7), -3, "dtype"), (dict(n_rows=-1), -1, "negative"), (dict(d=0), -2, "positive"), (dict(V=0), -2, "positive"), (dict(d=60), -2, "d % 8"),
          (dict(n_sel=3), -1, "rowsel is NULL"), (dict(n_sel=5, rowsel=256), -1, "exceeds n_rows"), (dict(H=None), -1, "H and ids"), (dict(W=None), -1, "W must not"),
          (dict(H=264), -1, "16-byte"), (dict(ids=None), -1, "H and ids"), (dict(ws=None), -4, "workspace"), (dict(ws=264), -4, "256-byte"), (dict(ws_bytes=64), -4, "hold"),
          (dict(dtype=F32, n_rows=1 << 20, n_sel=1 << 20, d=4096, V=100000), -2, "small shapes"), (dict(n_rows=1 << 28, n_sel=1 << 28, d=8), -2, "4 GiB")]
TAUGHT = [(dict(dH=None), -1, "dH"), (dict(stats=None), -1, "stats"), (dict(n_roles=65, tok_role=256), -2, "n_roles"), (dict(n_roles=2), -1, "tok_role"),
          (dict(dW_type=5), -3, "dW_type"), (dict(dtype=F32, dW_type=BF16), -3, "dW_type"), (dict(dW=None), -1, "dW must be NULL"), (dict(dW_type=NO_DW), -1, "dW must be NULL"),
          (dict(dW=264, dW_type=BF16), -1, "16-byte aligned"), (dict(norm_rows=3), -1, "norm_rows")]


@pytest.mark.parametrize("call", [top, ce, distill])
@pytest.mark.parametrize("kw,code,needle", SHARED)
def test_shared_arguments(lib, call, kw, code, needle):
    status, message = call(lib, **kw)
    assert status == code and needle in message, message


@pytest.mark.parametrize("call", [ce, distill])
@pytest.mark.parametrize("kw,code,needle", TAUGHT)
def test_arguments_of_the_taught_head(lib, call, kw, code, needle):
    status, message = call(lib, **kw)
    assert status == code and needle in message, message


@pytest.mark.parametrize("call,kw,code,needle", [(top, dict(k=0), -2, "k=0"), (top, dict(k=65), -2, "k=65"), (top, dict(logits=None), -1, "top_logits"), (top, dict(lse=None), -1, "lse"),
                                                 (distill, dict(k=0), -2, "k=0"), (distill, dict(k=65), -2, "k=65"), (distill, dict(logits=None), -1, "top_logits"),
                                                 (ce, dict(z_coef=-1.0), -1, "z_coef"), (ce, dict(z_coef=float("nan")), -1, "z_coef"), (ce, dict(z_coef=float("inf")), -1, "z_coef")])
def test_arguments_of_their_own(lib, call, kw, code, needle):
    status, message = call(lib, **kw)
    assert status == code and needle in message, message


# ------------------------------------------------------------------------------------------------ the binding's own checks, on host tensors
def tensors(**kw):
    n, d, V, k = 6, 16, 40, 3
    a = dict(H=torch.zeros(n, d, dtype=torch.bfloat16), W=torch.zeros(V, d, dtype=torch.bfloat16), ids=torch.zeros(n, dtype=torch.int32),
             top_ids=torch.zeros(n, k, dtype=torch.int32), top_logits=torch.zeros(n, k), lse=None, rowsel=None, z_coef=0.0, weight=None, tok_role=None, n_roles=0,
             train_head=True, accumulate_dW=False, norm_rows=0, dW=None, dH=None, row=None, stats=None, workspace=torch.empty(0, dtype=torch.uint8))
    return {**a, **kw}


def native_ce(a):
    return binding._native().cross_entropy(a["H"], a["W"], a["ids"], a["rowsel"], a["z_coef"], a["weight"], a["tok_role"], a["n_roles"], a["train_head"], a["accumulate_dW"],
                                           a["norm_rows"], a["dW"], a["dH"], a["row"], a["stats"], a["workspace"], 0)


def native_distill(a):
    return binding._native().distill(a["H"], a["W"], a["top_ids"], a["top_logits"], a["lse"], a["rowsel"], a["weight"], a["tok_role"], a["n_roles"], a["train_head"],
                                     a["accumulate_dW"], a["norm_rows"], a["dW"], a["dH"], a["row"], a["stats"], a["workspace"], 0)


F, I, B = torch.float32, torch.int32, torch.bfloat16
WRONG = [(dict(W=torch.zeros(40, 24, dtype=B)), ValueError), (dict(W=torch.zeros(40, 16)), ValueError), (dict(W=torch.zeros(16, 40, dtype=B).T), ValueError),
         (dict(H=torch.zeros(6, 32, dtype=B)[:, ::2]), ValueError), (dict(rowsel=torch.zeros(3, dtype=torch.int64)), TypeError), (dict(rowsel=torch.zeros(6, dtype=I)[::2]), TypeError),
         (dict(weight=torch.zeros(5)), ValueError), (dict(weight=torch.zeros(6, dtype=torch.float64)), TypeError), (dict(tok_role=torch.zeros(7, dtype=I), n_roles=2), ValueError),
         (dict(tok_role=torch.zeros(6), n_roles=2), TypeError), (dict(dH=torch.zeros(6, 16)), ValueError), (dict(dH=torch.zeros(5, 16, dtype=B)), ValueError),
         (dict(row=torch.zeros(5)), ValueError), (dict(row=torch.zeros(6, dtype=B)), ValueError), (dict(stats=torch.zeros(31, dtype=torch.uint8)), ValueError),
         (dict(stats=torch.zeros(32, dtype=torch.uint8), n_roles=1, tok_role=torch.zeros(6, dtype=I)), ValueError), (dict(accumulate_dW=True), ValueError),
         (dict(dW=torch.zeros(40, 16, dtype=torch.float64)), TypeError), (dict(dW=torch.zeros(39, 16)), ValueError), (dict(dW=torch.zeros(16, 40).T), ValueError)]


@pytest.mark.parametrize("call", [native_ce, native_distill])
@pytest.mark.parametrize("kw,kind", WRONG)
def test_tensors_that_do_not_fit(lib, call, kw, kind):
    with pytest.raises(kind):
        call(tensors(**kw))


@pytest.mark.parametrize("call,kw,kind", [(native_ce, dict(ids=torch.zeros(6, dtype=torch.int64)), TypeError), (native_ce, dict(ids=torch.zeros(5, dtype=I)), ValueError),
                                          (native_distill, dict(top_ids=torch.zeros(6, 3, dtype=torch.int64)), TypeError), (native_distill, dict(top_logits=torch.zeros(6, 2)), ValueError),
                                          (native_distill, dict(top_logits=torch.zeros(3, 6).T), ValueError), (native_distill, dict(lse=torch.zeros(5)), ValueError)])
def test_targets_that_do_not_fit(lib, call, kw, kind):
    with pytest.raises(kind):
        call(tensors(**kw))


@pytest.mark.parametrize("call", [native_ce, native_distill])
def test_what_fits_gets_as_far_as_the_workspace(lib, call):
    for kw in (dict(), dict(train_head=False), dict(dW=torch.zeros(40, 16)), dict(dW=torch.zeros(40, 16, dtype=B), accumulate_dW=True),
               dict(weight=torch.zeros(6), tok_role=torch.zeros(6, dtype=I), n_roles=2, rowsel=torch.zeros(4, dtype=I), dH=torch.zeros(6, 16, dtype=B), row=torch.zeros(6),
                    stats=torch.zeros(96, dtype=torch.uint8))):
        assert call(tensors(**kw)) == -4 and "workspace" in lib.umas_last_error().decode()


@pytest.mark.parametrize("kw,kind", [(dict(W=torch.zeros(40, 24, dtype=B)), ValueError), (dict(rowsel=torch.zeros(3, dtype=torch.int64)), TypeError),
                                     (dict(ids=torch.zeros(6, 3, dtype=torch.int64)), ValueError), (dict(ids=torch.zeros(6, 2, dtype=I)), ValueError),
                                     (dict(logits=torch.zeros(6, 4)), ValueError), (dict(lse=torch.zeros(5)), ValueError)])
def test_outputs_of_the_largest_logits_that_do_not_fit(lib, kw, kind):
    a = {**dict(H=torch.zeros(6, 16, dtype=B), W=torch.zeros(40, 16, dtype=B), rowsel=None, ids=None, logits=None, lse=None, ws=torch.empty(0, dtype=torch.uint8)), **kw}
    call = lambda a: binding._native().top_logits(a["H"], a["W"], 3, a["rowsel"], a["ids"], a["logits"], a["lse"], a["ws"], 0)
    with pytest.raises(kind):
        call(a)
    assert call({**a, **dict(W=torch.zeros(40, 16, dtype=B), rowsel=None, ids=None, logits=None, lse=None)}) == -4
