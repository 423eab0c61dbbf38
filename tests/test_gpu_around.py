"""The norm in front of a head, the draw of a token and the clipping of gradients on the GPU against the oracle, at the sizes where pieces, wavefronts and units end
and on inputs whose masks leave something empty.

Tolerances, from the arithmetic; f = 2^-24, u = 2^-8 (a rounding to bf16; 0 for float32).
  norm      a sum of squares of d numbers, at most d/64 + 16 of them one after the other: 1/rms is off by c = f ((d/64 + 16)/2 + 4) of itself, y by c + 2 f and
            its rounding, u.  The reference starts from the sum as the device has stored it, which is x + r to u (float32: f).
  8 bits    the scale is off by c + 3 f; a quotient, off by c + 5 f of itself, is rounded to a half of the step at its size: 2^-4 of it, 2^-10 below 2^-6
  backward  dx: f (8 i |a| + 8 i |s m|) + f (d/64 + 24) i |s| (i^2/d) sum |a s|, f |dhidden| and the rounding, u |dx|; dgain: f (n + 8) sum |dy s i|
  draws     tokens are equal.  logq is a float64 number rounded once, of a mass whose units are at least 2^-39: f |logq| + 1e-6 V 2^-39; logp has a sum of float32
            exponentials, each off by (|x| + 2) 2^-22 of itself, in float64: sum p (|x| + 2) 2^-22 + f |logp|
  clipping  the norm f of itself, numbers 2 f and their rounding, u"""
import math

import numpy as np
import pytest
import torch

import paper_2605_26646_amd as umas
from oracle import umas_oracle as orc

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
F, U = 2.0 ** -24, {"bf16": 2.0 ** -8, "f32": 0.0}
TINY = 1e-37


def device(x, dtype):
    """The array on the device in a type, and the values it has there."""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DT[dtype])
    return t.cuda(), t.double().numpy()


def host(t):
    return t.double().cpu().numpy()


# ------------------------------------------------------------------------------------------------ norm
WIDTHS = {"bf16": [8, 64, 504, 512, 520, 1024, 1544, 2048, 3584, 4096, 4104, 8192, 16384],
          "f32": [1, 3, 4, 5, 63, 255, 256, 257, 1023, 1024, 1025, 2048, 2051, 4099, 8191, 16383, 16384]}
NORM = [(dtype, d, n) for dtype in WIDTHS for i, d in enumerate(WIDTHS[dtype]) for n in ((1, 7, 2500) if i % 4 == 1 else (1, 6))]


def close(got, want, tol, name):
    off = np.abs(got - want) - tol
    assert not (off > 0).any(), (name, float(off.max()), np.argwhere(off > 0)[:3].tolist())


def rel_of(d):
    return F * ((d / 64 + 16) / 2 + 4)


@pytest.mark.parametrize("dtype,d,n", NORM)
@pytest.mark.parametrize("residual", [False, True])
def test_rms_norm(dtype, d, n, residual):
    rng = np.random.default_rng([5, d, n, residual])
    x, xh = device(rng.normal(size=(n, d)) * np.exp(rng.normal(size=(n, 1))), dtype)
    g, gh = device(1 + rng.normal(size=d) * 0.3, dtype)
    r, rh = device(rng.normal(size=(n, d)) * 3, dtype) if residual else (None, None)
    eps = 1e-6
    y, hidden, inv = umas.umas_rms_norm(x, g, r, eps=eps)
    assert y.dtype == DT[dtype] and hidden.dtype == DT[dtype] and inv.dtype == torch.float32
    if residual:
        close(host(hidden), xh + rh, max(U[dtype], F) * (1 + 2.0 ** -14) * np.abs(xh + rh) + TINY, "hidden")
    else:
        assert hidden is x
    want, inv_o = orc.rms_norm(host(hidden), gh, eps)
    c = rel_of(d)
    close(host(inv), inv_o, c * inv_o, "inv_rms")
    close(host(y), want, (U[dtype] + c + 3 * F) * 1.001 * np.abs(want) + TINY, "y")
    q, scale, hidden8, inv8 = umas.umas_rms_norm_quantized(x, g, r, eps=eps)
    assert q.dtype == torch.float8_e4m3fn and torch.equal(hidden8, hidden) and torch.equal(inv8, inv)
    big = np.abs(want).max(1) / 448
    big[big == 0] = 1
    close(host(scale), big, (c + 3 * F) * big, "scale")
    q, t = q.float().double().cpu().numpy(), want / big[:, None]
    close(q, t, np.maximum(2.0 ** -4 * np.abs(t), 2.0 ** -10) * 1.0001 + (c + 5 * F) * np.abs(t), "q")
    assert np.abs(q).max() <= 448


def test_rms_norm_of_zeros_infinities_and_no_numbers():
    for dtype, d in (("bf16", 64), ("bf16", 4096), ("f32", 33)):
        x = torch.randn(6, d, device="cuda").to(DT[dtype])
        x[1] = 0
        x[2, 5] = float("nan")
        x[3, 7] = float("inf")
        x[4] = torch.finfo(DT[dtype]).tiny
        g = torch.ones(d, device="cuda", dtype=DT[dtype])
        y, _, inv = umas.umas_rms_norm(x, g, eps=1e-5)
        assert not y[1].any() and float(inv[1]) == pytest.approx(1e-5 ** -0.5, rel=1e-6)
        assert y[2].isnan().all() and y[0].isfinite().all() and y[5].isfinite().all()
        assert float(inv[3]) == 0.0 and y[3, 7].isnan() and not y[3, :7].any()
        q, scale, _, _ = umas.umas_rms_norm_quantized(x, g, eps=1e-5)
        assert float(scale[1]) == 1.0 and not q[1].float().any()
        assert scale[2].isnan() and q[2].float().isnan().all() and scale[3].isnan() and q[3].float().isnan().all()
        for i in (0, 5):
            assert float(q[i].float().abs().max()) == 448
    # an eps of 0 and a row of zeros: 0 times infinity
    y, _, inv = umas.umas_rms_norm(torch.zeros(1, 8, device="cuda"), torch.ones(8, device="cuda"), eps=0.0)
    assert float(inv[0]) == math.inf and y.isnan().all()


def test_rms_norm_into_its_own_arrays():
    x, r, g = (torch.randn(*s, device="cuda").bfloat16() for s in ((3000, 512), (3000, 512), (512,)))
    y, hidden, inv = umas.umas_rms_norm(x, g, r)
    x2, r2 = x.clone(), r.clone()
    got = umas.umas_rms_norm(x2, g, r2, hidden=r2, y=x2)
    assert got[0] is x2 and got[1] is r2 and torch.equal(x2, y) and torch.equal(r2, hidden) and torch.equal(got[2], inv)
    x3 = x.clone()
    assert torch.equal(umas.umas_rms_norm(x3, g, y=x3)[0], umas.umas_rms_norm(x, g)[0])
    guard = torch.full((5, 512), 7.0, device="cuda").bfloat16()      # rows behind the last one stay as they were
    umas.umas_rms_norm(x[:3], g, y=guard[:3])
    assert (guard[3:] == 7).all()


@pytest.mark.parametrize("dtype,d,n", NORM)
@pytest.mark.parametrize("through", [False, True])
def test_rms_norm_backward(dtype, d, n, through):
    rng = np.random.default_rng([6, d, n, through])
    s, sh = device(rng.normal(size=(n, d)) * np.exp(rng.normal(size=(n, 1))), dtype)
    g, gh = device(1 + rng.normal(size=d) * 0.3, dtype)
    dy = rng.normal(size=(n, d)) * (rng.random((n, 1)) > 0.3)
    dy, dyh = device(dy, dtype)
    ds, dsh = device(rng.normal(size=(n, d)), dtype) if through else (None, None)
    _, _, inv = umas.umas_rms_norm(s, g)
    i = host(inv)
    dx, dgain = umas.umas_rms_norm_bwd(dy, s, g, inv, ds)
    dx_o, dg_o = orc.rms_norm_backward(dyh, sh, gh, i, dsh)
    a = np.abs(dyh * gh)
    m = np.abs(i ** 2 / d * (dyh * gh * sh).sum(1))[:, None]
    tol = F * 8 * i[:, None] * (a + np.abs(sh) * m) + F * (d / 64 + 24) * (i[:, None] * np.abs(sh)) * (i ** 2 / d * (a * np.abs(sh)).sum(1))[:, None]
    if through:
        tol += F * np.abs(dsh)
    close(host(dx), dx_o, 1.01 * (tol + (U[dtype] + F) * np.abs(dx_o)) + TINY, "dx")
    close(host(dgain), dg_o, F * (n + 8) * (np.abs(dyh * sh) * i[:, None]).sum(0) + TINY, "dgain")
    more = dgain.clone()
    umas.umas_rms_norm_bwd(dy, s, g, inv, ds, accumulate_dgain=True, dgain=more)
    assert torch.equal(more, dgain + dgain)
    into = dy.clone()                                               # in place of dy
    assert torch.equal(umas.umas_rms_norm_bwd(into, s, g, inv, ds, dx=into)[0], dx)


@pytest.mark.parametrize("dtype,d", [("bf16", 256), ("bf16", 8192), ("f32", 77)])
def test_rows_without_a_gradient_add_nothing_whatever_they_hold(dtype, d):
    n = 40
    s, dy, ds = (torch.randn(n, d, device="cuda").to(DT[dtype]) for _ in range(3))
    g = torch.randn(d, device="cuda").to(DT[dtype])
    idle = torch.arange(n, device="cuda") % 3 == 1
    dy[idle] = 0
    _, _, inv = umas.umas_rms_norm(s, g)
    want = umas.umas_rms_norm_bwd(dy, s, g, inv, ds)
    s[idle] = float("nan")
    inv[idle] = float("nan")
    got = umas.umas_rms_norm_bwd(dy, s, g, inv, ds)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[0][idle], ds[idle])
    got = umas.umas_rms_norm_bwd(dy, s, g, inv)
    assert not got[0][idle].any() and got[0].isfinite().all() and torch.equal(got[1], want[1])
    dx, dgain = umas.umas_rms_norm_bwd(dy[:0], s[:0], g, inv[:0])
    assert dx.shape == (0, d) and not dgain.any()


def test_rms_norm_backward_against_differences():
    n, d, eps, h = 5, 48, 1e-3, 2e-3
    torch.manual_seed(3)
    x, r, v = (torch.randn(n, d, device="cuda") for _ in range(3))
    g = torch.randn(d, device="cuda")
    value = lambda x, g: float((umas.umas_rms_norm(x, g, r, eps=eps)[0].double() * v.double()).sum())  # noqa: E731
    y, hidden, inv = umas.umas_rms_norm(x, g, r, eps=eps)
    dx, dgain = umas.umas_rms_norm_bwd(v, hidden, g, inv)
    for _ in range(10):
        e, eg = torch.randn(n, d, device="cuda"), torch.randn(d, device="cuda")
        # h^2 times third derivatives of order one, and d float32 roundings over 2 h: below 1e-3 of sums of about ten
        slope = (value(x + h * e, g) - value(x - h * e, g)) / (2 * h)
        assert abs(slope - float((dx * e).sum())) < 2e-2
        slope = (value(x, g + h * eg) - value(x, g - h * eg)) / (2 * h)
        assert abs(slope - float((dgain * eg).sum())) < 2e-2


# ------------------------------------------------------------------------------------------------ draws
def check_draws(z, u, settings, got, V):
    """z: the logits as float64 numpy [n, V]; settings: dict of numbers or arrays."""
    ids, logp, logq = (x.cpu().numpy() for x in got)
    for i in range(len(z)):
        s = {k: (v[i].item() if np.ndim(v) else v) for k, v in settings.items()}
        id_o, logp_o, logq_o = orc.sample(z[i], float(u[i]), **s)
        assert ids[i] == id_o, (i, s, float(u[i]), int(ids[i]), id_o)
        if id_o < 0:
            assert logp[i] == 0 and logq[i] == 0
            continue
        zi = np.where(np.isnan(z[i]), -np.inf, z[i])
        x = np.where(zi == zi.max(), 0.0, zi - zi.max())
        p = np.exp(x) / np.exp(x).sum()
        p, x = p[p > 0], x[p > 0]
        assert abs(logp[i] - logp_o) <= (p * (np.abs(x) + 2)).sum() * 2.0 ** -22 + F * abs(logp_o), (i, logp[i], logp_o)
        assert abs(logq[i] - logq_o) <= F * abs(logq_o) + 1e-6 * V * 2.0 ** -39 + 1e-12, (i, logq[i], logq_o)


def row_settings(rng, n, V):
    return {"temperature": np.where(rng.random(n) < 0.15, 0.0, 0.2 + 1.5 * rng.random(n)).astype(np.float32),
            "top_k": np.where(rng.random(n) < 0.4, 0, np.exp(rng.random(n) * np.log(V + 2))).astype(np.int32),
            "top_p": np.where(rng.random(n) < 0.3, 1.0, rng.random(n)).astype(np.float32),
            "min_p": np.where(rng.random(n) < 0.5, 0.0, 0.3 * rng.random(n)).astype(np.float32)}


def on_device(settings):
    return {k: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for k, v in settings.items()}


SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.6, top_k=1), dict(top_k=7), dict(temperature=1.3, top_p=0.9), dict(min_p=0.1), dict(top_k=40, top_p=0.8, min_p=0.02),
            dict(temperature=0.05, top_p=0.5), dict(temperature=100.0, top_p=0.3), dict(top_p=0.0), dict(top_k=10 ** 9, min_p=1.0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 255, 1000, 1023, 1024, 1025, 2049, 4096, 5003, 20011])
def test_sample_logits(V, dtype):
    rng = np.random.default_rng([8, V])
    n = 24
    for j, scale in enumerate((0.0, 1.0, 4.0)):
        z, zh = device(rng.normal(size=(n, V)) * scale, dtype)
        u = rng.random(n).astype(np.float32)
        for s in SETTINGS if V <= 1100 or j == 1 else SETTINGS[3:7]:
            check_draws(zh, u, s, umas.umas_sample_logits(z, torch.from_numpy(u).cuda(), **s), V)
        s = row_settings(rng, n, V)
        check_draws(zh, u, s, umas.umas_sample_logits(z, torch.from_numpy(u).cuda(), **on_device(s)), V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,pad,shift", [(1000, 1, 0), (1000, 3, 5), (1025, 7, 1), (4099, 0, 1), (5000, 13, 3)])
def test_sample_logits_of_a_padded_vocabulary(V, pad, shift, dtype):
    rng = np.random.default_rng([9, V, pad])
    n = 9
    buf, bufh = device(rng.normal(size=(n * (V + pad) + shift)) * 3, dtype)
    z = buf[shift:].view(n, V + pad)[:, :V]
    zh = bufh[shift:].reshape(n, V + pad)[:, :V]
    u = rng.random(n).astype(np.float32)
    for s in (dict(), dict(top_p=0.7), dict(top_k=20, min_p=0.01)):
        check_draws(zh, u, s, umas.umas_sample_logits(z, torch.from_numpy(u).cuda(), **s), V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [5, 700, 3000])
def test_masked_and_infinite_logits(V, dtype):
    low, inf, nan = torch.finfo(DT[dtype]).min, math.inf, math.nan
    rng = np.random.default_rng([10, V])
    z = rng.normal(size=(12, V)) * 2
    z[0] = -inf                                                     # nothing
    z[1] = nan
    z[2] = low                                                      # all masked by the lowest number: as likely as each other
    z[3, 1:] = -inf                                                 # one left
    z[4, 1:] = low
    z[5, rng.random(V) < 0.5] = nan
    z[6, rng.random(V) < 0.9] = -inf
    z[7, [1, 3]] = inf                                              # two that are infinitely likely
    z[8, 2] = inf
    z[9] = 0.0
    z[10, ::2] = -0.0
    z[10, 1::2] = 0.0
    z[11, :-1] = low
    z[11, -1] = -torch.finfo(DT[dtype]).max / 2
    z, zh = device(z, dtype)
    for u in (0.0, 0.3, 0.5, 0.999, 1.0 - 2.0 ** -24):
        uu = np.full(12, u, np.float32)
        for s in (dict(), dict(top_k=3), dict(top_p=0.6), dict(min_p=0.5), dict(temperature=0.0), dict(temperature=0.5, top_k=2, top_p=0.9)):
            check_draws(zh, uu, s, umas.umas_sample_logits(z, torch.from_numpy(uu).cuda(), **s), V)


def test_uniform_numbers_out_of_range_and_at_borders():
    V = 8
    z = torch.zeros(9, V, device="cuda")
    u = torch.tensor([0.0, 0.125, 0.25, 0.5 - 2.0 ** -25, 0.5, 1.0, 7.0, -3.0, math.nan], device="cuda")
    for s in (dict(), dict(top_k=8), dict(top_p=1.0, min_p=1.0)):
        ids, logp, logq = umas.umas_sample_logits(z, u, **s)
        assert ids.tolist() == [0, 1, 2, 3, 4, 7, 7, 0, 0]
        assert torch.allclose(logp, torch.full_like(logp, -math.log(8))) and torch.allclose(logq, logp)
    ids, _, logq = umas.umas_sample_logits(z, u, top_p=0.5)          # the first four of equal ones
    assert ids.tolist() == [0, 0, 1, 1, 2, 3, 3, 0, 0] and torch.allclose(logq, torch.full_like(logq, -math.log(4)))
    ids, _, logq = umas.umas_sample_logits(z, u, top_k=2, top_p=0.75)
    assert ids.tolist() == [0, 0, 0, 0, 1, 1, 1, 0, 0] and torch.allclose(logq, torch.full_like(logq, -math.log(2)))


def test_settings_of_rows_out_of_range_are_taken_in():
    z = torch.randn(8, 500, device="cuda")
    u = torch.rand(8, device="cuda")
    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))  # noqa: E731
    full = lambda v, t=torch.float32: torch.full((8,), v, dtype=t, device="cuda")  # noqa: E731
    for kw, as_if in ((dict(temperature=full(-1.0)), dict(temperature=0.0)), (dict(temperature=full(math.nan)), dict(temperature=0.0)), (dict(top_p=full(1.5)), dict(top_p=1.0)),
                      (dict(top_p=full(math.nan)), dict(top_p=1.0)), (dict(top_p=full(-0.5)), dict(top_p=0.0)), (dict(min_p=full(2.0)), dict(min_p=1.0)),
                      (dict(min_p=full(-1.0)), dict(min_p=0.0)), (dict(min_p=full(math.nan)), dict(min_p=0.0)), (dict(top_k=full(-5, torch.int32)), dict(top_k=0)),
                      (dict(top_k=full(2 ** 31 - 1, torch.int32)), dict())):
        assert same(umas.umas_sample_logits(z, u, **kw), umas.umas_sample_logits(z, u, **as_if)), kw
    ids, _, _ = umas.umas_sample_logits(z, u, temperature=math.inf)  # uniform
    assert torch.equal(ids.long(), (u.double() * 500).long())


def plain_tokens(H, W):
    return H.double().cpu().numpy() @ W.double().cpu().numpy().T


@pytest.mark.parametrize("n,d,V,dtype", [(1, 64, 300, "bf16"), (3, 2048, 4001, "bf16"), (40, 72, 1025, "bf16"), (64, 512, 2048, "bf16"), (65, 264, 3001, "bf16"), (128, 64, 769, "bf16"),
                                         (129, 136, 1000, "bf16"), (300, 64, 2049, "bf16"), (5, 33, 777, "f32"), (70, 64, 2500, "f32")])
def test_sample_tokens(n, d, V, dtype):
    rng = np.random.default_rng([11, n, V])
    for select in (False, True):
        # a grid on which every product and sum is exact in float32, so that logits are equal
        H, _ = device(np.round(rng.normal(size=(n, d)) * 4) / 4, dtype)
        W, _ = device(np.round(rng.normal(size=(V, d)) * (64 / math.sqrt(d))) / 32, dtype)
        rows = np.sort(rng.permutation(n)[:max(1, 3 * n // 4)]) if select else np.arange(n)
        sel = torch.from_numpy(rows.astype(np.int32)).cuda() if select else None
        z, u = plain_tokens(H, W), rng.random(n).astype(np.float32)
        ud = torch.from_numpy(u).cuda()
        for s in (dict(), dict(temperature=0.0), dict(temperature=0.7, top_k=20, top_p=0.9), dict(top_p=0.95, min_p=0.01), row_settings(rng, n, V)):
            got = umas.umas_sample_tokens(H, W, ud, sel, **on_device(s))
            check_draws(z[rows], u[rows], {k: v[rows] if np.ndim(v) else v for k, v in s.items()}, [x[torch.from_numpy(rows).cuda()] for x in got], V)
            rest = torch.ones(n, dtype=torch.bool)
            rest[rows] = False
            assert (got[0].cpu()[rest] == -1).all() and not got[1].cpu()[rest].any() and not got[2].cpu()[rest].any()


def test_tokens_do_not_depend_on_the_workspace_or_on_other_rows():
    n, d, V = 700, 64, 3000
    H, _ = device(np.round(np.random.default_rng(1).normal(size=(n, d)) * 4) / 4, "bf16")
    W, _ = device(np.round(np.random.default_rng(2).normal(size=(V, d)) * 8) / 32, "bf16")
    u = torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(4))
    lib = umas.load_library()
    least, full = (getattr(lib, "umas_sample_tokens_workspace_bytes" + w)(n, d, V, 1) for w in ("_min", ""))
    assert least < full
    for s in (dict(), dict(top_p=0.8), dict(temperature=0.5, top_k=30)):
        want = umas.umas_sample_tokens(H, W, u, **s)
        for b in (least, (least + full) // 2, full):
            ws = torch.full((b,), 0xFF, dtype=torch.uint8, device="cuda")
            assert all(torch.equal(a, c) for a, c in zip(umas.umas_sample_tokens(H, W, u, workspace=ws, **s), want))
        for rows in ([5], list(range(100, 160)), list(range(0, 700, 3))):
            sel = torch.tensor(rows, dtype=torch.int32, device="cuda")
            got = umas.umas_sample_tokens(H, W, u, sel, **s)
            assert all(torch.equal(a[rows], c[rows]) for a, c in zip(got, want))
    same = umas.umas_sample_logits((H.float() @ W.float().T), u, top_p=0.8)
    want = umas.umas_sample_tokens(H, W, u, top_p=0.8)
    assert all(torch.equal(a, b) for a, b in zip(same, want))
    logp = umas.umas_policy_logprobs(H, W, want[0])[0]
    assert (logp - want[1]).abs().max() < 2e-5


# ------------------------------------------------------------------------------------------------ clipping
def gradients(rng, sizes):
    out, values = [], []
    for i, n in enumerate(sizes):
        dtype = "bf16" if i % 3 else "f32"
        t, v = device(rng.normal(size=n) * 10.0 ** rng.integers(-3, 2), dtype)
        out.append(t)
        values.append(v)
    return out, values


SIZES = [[1], [7, 8, 9], [8191, 8192, 8193], [0, 5, 0, 16384, 0], [100003], list(range(1, 97)), list(range(200, 300)), [3] * 500 + [70001]]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("share", [0.1, 1.5, math.inf])
def test_clip_gradients(sizes, share):
    rng = np.random.default_rng([12, len(sizes), sum(sizes)])
    grads, values = gradients(rng, sizes)
    norm = orc.clip(values, math.inf)[0]
    norm_o, c, _, want = orc.clip(values, share * norm)
    keep = [g.clone() for g in grads]
    out = [torch.full_like(g, 7) for g in grads]
    stats, got = umas.umas_clip_gradients(grads, share * norm, out=out)
    s = umas.read_clip_stats(stats)[0]
    assert abs(s["norm"] - norm_o) <= F * norm_o * 1.01 and abs(s["scale"] - c) <= F * 1.01 * c and s["n_not_finite"] == 0
    assert all(a is b for a, b in zip(got, out)) and all(torch.equal(a, b) for a, b in zip(grads, keep))
    for o, w in zip(out, want):
        u = U["bf16" if o.dtype == torch.bfloat16 else "f32"]
        close(host(o), w, (u + 2.01 * F) * np.abs(w) + TINY, "out")
    stats2, got = umas.umas_clip_gradients(grads, share * norm)
    assert torch.equal(stats2, stats) and all(a is b for a, b in zip(got, grads)) and all(torch.equal(a, b) for a, b in zip(grads, out))


def test_clip_gradients_in_views_at_any_offset():
    rng = np.random.default_rng(13)
    for dtype in ("bf16", "f32"):
        flat, _ = device(rng.normal(size=70000), dtype)
        into = torch.full_like(flat, 5.0)
        at, views, outs = 1, [], []
        for n in (1, 3, 9001, 17, 8192, 33333, 2):
            views.append(flat[at:at + n])
            outs.append(into[at + 2:at + 2 + n])
            at += n + 3
        want = orc.clip([host(v) for v in views], 3.0)
        stats, _ = umas.umas_clip_gradients(views, 3.0, out=outs)
        for o, w in zip(outs, want[3]):
            close(host(o), w, (U[dtype] + 2.01 * F) * np.abs(w) + TINY, "out")
        written = sum(len(o) for o in outs)
        assert int((into == 5.0).sum()) >= len(into) - written       # what lies between the views is as it was
        before = flat.clone()
        umas.umas_clip_gradients(views, 3.0)
        assert all(torch.equal(v, o) for v, o in zip(views, outs))
        inside = torch.zeros(len(flat), dtype=torch.bool, device="cuda")
        at = 1
        for v in views:
            inside[at:at + len(v)] = True
            at += len(v) + 3
        assert torch.equal(flat[~inside], before[~inside])


def test_gradients_that_are_no_numbers_scale_nothing():
    for bad, count in ((math.nan, 1), (math.inf, 2), (-math.inf, 3)):
        g = [torch.randn(9000, device="cuda"), torch.randn(20001, device="cuda").bfloat16()]
        g[1][5:5 + count] = bad
        keep = [x.clone() for x in g]
        stats, _ = umas.umas_clip_gradients(g, 0.5)
        s = umas.read_clip_stats(stats)[0]
        assert s["scale"] == 1.0 and s["n_not_finite"] == count and not np.isfinite(s["norm"])
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(g, keep))
    g = [torch.full((1000,), 3e30, device="cuda")]                   # a square beyond float32
    stats, _ = umas.umas_clip_gradients(g, 1.0)
    s = umas.read_clip_stats(stats)[0]
    assert abs(s["norm"] / (3e30 * 1000 ** 0.5) - 1) < 1e-6 and s["n_not_finite"] == 0 and abs(float(g[0].norm()) - 1) < 1e-5
    g = [torch.zeros(100, device="cuda"), torch.zeros(0, device="cuda")]
    s = umas.read_clip_stats(umas.umas_clip_gradients(g, 1.0)[0])[0]
    assert s["norm"] == 0 and s["scale"] == 1 and not g[0].any()
