"""The example's step: the gradients that reach its optimizer are those of the loss, clipped to a common norm.

Hidden states, gain, head and dH are bf16.  A rounding is 2^-8 of a value at most; on the way to a gradient lie those of h, the gain, H, W, the kept numerators, dH and dh: seven, and as
random signs they add up to about 2^-8 sqrt(7) / sqrt(3) = 0.006 of a gradient's norm, at most 7 * 2^-8 = 0.027 where all agree, which is the bound."""
import importlib.util
import os

import pytest
import torch

import paper_2605_26646_amd as umas

pytestmark = pytest.mark.gpu


def test_gradients_of_the_solver():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "teach_role.py")
    spec = importlib.util.spec_from_file_location("teach_role", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    gen = torch.Generator("cuda").manual_seed(7)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    n, context, V = 300, 96, 501
    x, said = randn(n, context), torch.randint(0, V, (n,), device="cuda", generator=gen, dtype=torch.int32)
    params = [randn(context, 128) / context ** 0.5, 1 + 0.1 * randn(128), 0.2 * randn(V, 128)]
    rows = torch.arange(0, n, 2, device="cuda", dtype=torch.int32)
    parts = [rows[:70].contiguous(), rows[70:].contiguous()]

    class Idle:
        def step(self):
            pass

    loss = example.train(x, params, Idle(), parts, len(rows), lambda H, W, r, **kw: umas.umas_cross_entropy_fwd_bwd(H, W, said, r, **kw))
    A, gain, W = (p.double().cpu().requires_grad_() for p in params)
    h = x.double().cpu()[::2] @ A
    H = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6) * gain
    want = torch.nn.functional.cross_entropy(H @ W.T, said.long().cpu()[::2])
    grads = torch.autograd.grad(want, (A, gain, W))
    norm = float(sum(g.square().sum() for g in grads).sqrt())
    scale = min(1.0, 1.0 / norm)
    assert abs(loss - float(want.detach())) < 0.02 * float(want.detach())
    for p, g in zip(params, grads):
        assert float((p.grad.double().cpu() - g * scale).norm()) <= (7 * 2.0 ** -8 + 7 * 2.0 ** -8 * (scale < 1)) * scale * float(g.norm())
    assert float(sum(p.grad.double().square().sum() for p in params).sqrt()) <= 1 + 1e-5
