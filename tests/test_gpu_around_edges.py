"""The norm, the draws and the clipping where a call is large, repeated, recorded or joined with others: vocabularies in full width, rows whose filters end far behind the front, more
rows than one chunk, offsets past 32 bits, graphs, streams, and a step from the norm to the clipped gradients.

Tolerances, from the arithmetic; f = 2^-24.
  draws     tokens are equal to those of float64 weights.  A weight is off by 2.2e-12 of itself and by half a unit of 2^-s, s = min(51, 62 - ceil log2 V), and a mass is at least
            the largest weight, 1: logq is off by e = 5e-12 + V 2^-s, and rounded once, f |logq|.  logp as for the small sizes: sum p (|x| + 2) 2^-22 + f |logp|.
  step      float32 throughout.  Every value on the way is a sum of at most d + V + n products, each rounded once and each sum rounded once per term: off by (d + V + n) f = 2.4e-5
            of the sum of magnitudes, which for sums of random signs is at most 16 times the largest result here; four of them follow one another: 1.6e-3 of the largest entry.
  the rest  compares bits"""
import math

import numpy as np
import pytest
import torch

import paper_2605_26646_amd as umas

pytestmark = pytest.mark.gpu
F = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def same(a, b):
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


# ------------------------------------------------------------------------------------------------ draws
def draw64(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """ids, logp, logq of float64 logits on the device, all rows under one setting with a temperature above 0."""
    top = z.max(1, keepdim=True).values
    p = torch.exp(z - top)
    s, order = torch.sort(z, dim=1, descending=True, stable=True)
    w = torch.exp((s - top) / temperature)
    if 0 < top_k < z.shape[1]:
        w[:, top_k:] = 0
    w[w < min_p] = 0
    if top_p < 1:
        run = torch.cumsum(w, 1)
        ahead = torch.cat([torch.zeros_like(run[:, :1]), run[:, :-1]], 1)
        w[:, 1:][(ahead >= top_p * run[:, -1:])[:, 1:]] = 0
    kept = torch.zeros_like(w).scatter_(1, order, w)
    run = torch.cumsum(kept, 1)
    last = torch.where(kept > 0, torch.arange(z.shape[1], device=z.device), 0).max(1).values
    ids = torch.minimum((run <= u.double()[:, None] * run[:, -1:]).sum(1), last)
    at = ids[:, None]
    return ids, torch.log(p.gather(1, at)[:, 0] / p.sum(1)), torch.log(kept.gather(1, at)[:, 0] / run[:, -1]), torch.where(p > 0, p / p.sum(1, keepdim=True) * ((z - top).abs() + 2), 0).sum(1)


def check(z, u, got, **s):
    ids, logp, logq, e = draw64(z.double(), u, **s)
    bad = (got[0].long() != ids).nonzero().flatten().tolist()
    assert not bad, (s, [(i, int(got[0][i]), int(ids[i]), float(u[i])) for i in bad])
    V = z.shape[1]
    unit = 2.0 ** -min(51, 62 - max(V - 1, 0).bit_length())
    assert ((got[1].double() - logp).abs() <= e * 2.0 ** -22 + F * logp.abs()).all(), s
    assert ((got[2].double() - logq).abs() <= F * logq.abs() + 5e-12 + V * unit).all(), s


def logits_of(kind, n, V, dtype, gen):
    z = torch.randn(n, V, device="cuda", generator=gen)
    z = {"flat": lambda: z * 1e-3, "wide": lambda: z, "peaked": lambda: z * 4, "ties": lambda: (z * 2).round() / 2, "equal": lambda: z * 0,
         "rising": lambda: (z * 2).sort(1).values, "falling": lambda: (z * 2).sort(1, descending=True).values,
         "two": lambda: torch.where(z > 1, 0.0, -3.0)}[kind]()
    return z.to(DT[dtype])


FAR = [dict(top_p=0.9), dict(top_p=0.5, temperature=0.7), dict(top_p=0.99, temperature=3.0), dict(top_k=5000), dict(top_k=60000), dict(min_p=1e-4), dict(min_p=0.02),
       dict(top_k=20000, top_p=0.7, min_p=1e-5), dict(top_k=300), dict(top_k=2, top_p=0.999)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["flat", "wide", "peaked", "ties", "equal", "rising", "falling", "two"])
@pytest.mark.parametrize("V", [33001, 151936])
def test_filters_that_end_far_behind_the_front(V, kind, dtype):
    """One row (whose workgroup does all of it), two and many (spread over the chip) give the same."""
    gen = torch.Generator("cuda").manual_seed(V + len(kind))
    n = 10
    z, u = logits_of(kind, n, V, dtype, gen), torch.rand(n, device="cuda", generator=gen)
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -24
    for s in FAR + [dict()]:
        got = umas.umas_sample_logits(z, u, **s)
        check(z, u, got, **s)
        for rows in (1, 2):
            few = [umas.umas_sample_logits(z[a:a + rows], u[a:a + rows], **s) for a in range(0, n, rows)]
            assert same(got, [torch.cat(x) for x in zip(*few)]), s


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["flat", "wide", "peaked", "ties", "equal", "rising", "two"])
@pytest.mark.parametrize("V", [128, 129, 300, 511, 512, 513])
def test_rows_of_as_many_tokens_as_one_list_holds(V, kind, dtype):
    gen = torch.Generator("cuda").manual_seed(V + len(kind))
    n = 12
    z, u = logits_of(kind, n, V, dtype, gen), torch.rand(n, device="cuda", generator=gen)
    z[3, :V // 3] = -math.inf
    z[4, V // 4:] = torch.finfo(z.dtype).min
    z[5, 2:] = -1e30
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -24
    for s in (dict(top_k=1), dict(top_k=V // 2), dict(top_k=V - 1, top_p=0.9), dict(top_p=0.6), dict(top_p=0.999, min_p=0.1), dict(top_k=140, min_p=0.05, top_p=0.5, temperature=2.0),
              dict(min_p=1.0), dict(top_p=0.0), dict(top_p=0.8, temperature=1e-3)):
        got = umas.umas_sample_logits(z, u, **s)
        check(z, u, got, **s)
        assert same(got, [torch.cat(x) for x in zip(*[umas.umas_sample_logits(z[a:a + 3], u[a:a + 3], **s) for a in range(0, n, 3)])]), s


@pytest.mark.parametrize("min_p", [0.3, 0.1, 0.03, 0.01])
def test_some_hundreds_of_tokens_above_a_border_of_min_p(min_p):
    gen = torch.Generator("cuda").manual_seed(5)
    n, V = 48, 50000
    z = torch.randn(n, V, device="cuda", generator=gen) * torch.linspace(0.3, 3, n, device="cuda")[:, None]
    u = torch.rand(n, device="cuda", generator=gen)
    for s in (dict(), dict(top_p=0.9), dict(top_k=200), dict(top_k=150, top_p=0.5)):
        check(z, u, umas.umas_sample_logits(z, u, min_p=min_p, **s), min_p=min_p, **s)


@pytest.mark.parametrize("n", [1, 6])
def test_the_widest_vocabulary(n):
    V = 1 << 20
    gen = torch.Generator("cuda").manual_seed(n)
    z, u = torch.randn(n, V, device="cuda", generator=gen) * 2, torch.rand(n, device="cuda", generator=gen)
    for s in (dict(), dict(top_p=0.95), dict(top_k=100000, temperature=0.5), dict(min_p=1e-3)):
        check(z, u, umas.umas_sample_logits(z, u, **s), **s)


@pytest.mark.parametrize("V,n", [(1500, 2500), (5000, 1029)])
def test_more_rows_than_a_chunk(V, n):
    gen = torch.Generator("cuda").manual_seed(V)
    z, u = torch.randn(n, V, device="cuda", generator=gen) * 2, torch.rand(n, device="cuda", generator=gen)
    for s in (dict(), dict(top_p=0.9), dict(top_k=700), dict(top_k=8, temperature=0.8)):
        check(z, u, umas.umas_sample_logits(z, u, **s), **s)
    t = 0.3 + torch.rand(n, device="cuda", generator=gen)
    k = torch.randint(0, V, (n,), device="cuda", generator=gen, dtype=torch.int32)
    got = umas.umas_sample_logits(z, u, temperature=t, top_k=k)
    for a in (0, 1023, 1024, n - 1):
        check(z[a:a + 1], u[a:a + 1], [x[a:a + 1] for x in got], temperature=float(t[a]), top_k=int(k[a]))


def test_rows_of_logits_far_apart():
    """Row offsets past 2^31 numbers and 2^32 bytes."""
    V, stride = 3001, 2 ** 31 + 5
    buf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((3, V), (stride, 1))
    z.copy_(torch.randn(3, V, device="cuda"))
    u = torch.tensor([0.2, 0.5, 0.9], device="cuda")
    for s in (dict(), dict(top_p=0.8), dict(top_k=20)):
        got = umas.umas_sample_logits(z, u, **s)
        assert same(got, umas.umas_sample_logits(z.contiguous(), u, **s))
        check(z.contiguous(), u, got, **s)


def test_rows_that_are_selected_twice_and_in_any_order():
    n, d, V = 50, 64, 3000
    H, W, u = torch.randn(n, d, device="cuda").bfloat16(), torch.randn(V, d, device="cuda").bfloat16(), torch.rand(n, device="cuda")
    for s in (dict(), dict(top_p=0.9), dict(top_k=500)):
        want = umas.umas_sample_tokens(H, W, u, **s)
        sel = torch.randperm(n, device="cuda")[:30].to(torch.int32)
        got = umas.umas_sample_tokens(H, W, u, torch.cat([sel, sel[:12], sel[:1]]), **s)
        assert same([x[sel.long()] for x in got], [x[sel.long()] for x in want])
    none = umas.umas_sample_tokens(H, W, u, sel[:0])
    assert (none[0] == -1).all() and not none[1].any() and not none[2].any()
    assert [x.shape for x in umas.umas_sample_tokens(H[:0], W, u[:0], top_k=3)] == [(0,)] * 3 == [x.shape for x in umas.umas_sample_logits(H[:0], u[:0])]


# ------------------------------------------------------------------------------------------------ sizes
def test_a_norm_over_more_than_32_bits_of_numbers():
    n, d = 131072 + 300, 16384
    x = torch.empty(n, d, dtype=torch.bfloat16, device="cuda").fill_(1.0)
    tail = torch.randn(7, d, device="cuda").bfloat16()
    x[-7:] = tail
    g = torch.randn(d, device="cuda").bfloat16()
    y, _, inv = umas.umas_rms_norm(x, g)
    want = umas.umas_rms_norm(tail, g)
    assert same((y[-7:], inv[-7:]), (want[0], want[2]))
    assert torch.equal(y[0], y[n - 8]) and torch.equal(y[0], y[n // 2])
    q, scale, _, _ = umas.umas_rms_norm_quantized(x, g)
    want = umas.umas_rms_norm_quantized(tail, g)
    assert same((q[-7:], scale[-7:]), want[:2])
    del q
    y.zero_()
    y[-7:] = dy = torch.randn(7, d, device="cuda").bfloat16()         # nothing but the last rows
    want = umas.umas_rms_norm_bwd(dy, tail, g, inv[-7:].clone())
    dx, dgain = umas.umas_rms_norm_bwd(y, x, g, inv, dx=y)
    assert same((dx[-7:],), (want[0],)) and not dx[:-7].any()
    # seven terms each, in another order
    assert ((dgain - want[1]).abs() <= 16 * F * (dy.float() * tail.float() * inv[-7:, None]).abs().sum(0)).all()


def test_a_norm_of_more_rows_than_a_launch_counts():
    n, d = (1 << 25) + 77, 8                                          # a wavefront to a row: threads past 2^31
    x = torch.ones(n, d, dtype=torch.bfloat16, device="cuda")
    x[-5:] = torch.randn(5, d, device="cuda").bfloat16()
    g = torch.randn(d, device="cuda").bfloat16()
    y, _, inv = umas.umas_rms_norm(x, g)
    want = umas.umas_rms_norm(x[-5:].clone(), g)
    assert same((y[-5:], inv[-5:]), (want[0], want[2]))
    first = umas.umas_rms_norm(x[:1].clone(), g)
    assert (y[:-5] == first[0]).all() and (inv[:-5] == first[2]).all()


def test_a_gradient_of_more_than_32_bits_of_numbers():
    n = 2 ** 31 + 12345
    a = torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    b = torch.full((3,), 2.0, device="cuda")
    norm = math.sqrt(n * 2.0 ** -20 + 12)
    stats, _ = umas.umas_clip_gradients([a, b], norm / 2)
    s = umas.read_clip_stats(stats)[0]
    assert abs(s["norm"] - norm) <= 2 * F * norm and abs(s["scale"] - 0.5) <= 2 * F and s["n_not_finite"] == 0
    assert (a == 2.0 ** -11).all() and ((b - 1).abs() <= 2.0 ** -22).all()


# ------------------------------------------------------------------------------------------------ graphs, streams
def training(x, r, g, dy, ws):
    y, hidden, inv = umas.umas_rms_norm(x, g, r)
    q = umas.umas_rms_norm_quantized(x, g, r)
    dx, dgain = umas.umas_rms_norm_bwd(dy, hidden, g, inv, dy, workspace=ws[0])
    stats, clipped = umas.umas_clip_gradients([dx, dgain] + [y[i] for i in range(100)], 3.0, out=[torch.empty_like(dx), torch.empty_like(dgain)] + [torch.empty_like(y[i]) for i in range(100)],
                                              workspace=ws[1])
    umas.umas_clip_gradients([dgain, dx], 2.0, workspace=ws[1])
    return [y, hidden, inv, *q, dx, dgain, stats, *clipped]


def answering(H, W, u, ws):
    out = []
    for s in (dict(), dict(top_k=20), dict(top_p=0.9), dict(top_k=900, min_p=1e-3), dict(temperature=0.0)):
        out += umas.umas_sample_tokens(H, W, u, workspace=ws, **s)
    return out + [*umas.umas_sample_logits(H, u, top_p=0.7)]


def test_recorded_calls_give_at_every_replay_what_eager_ones_give():
    n, d, V = 130, 512, 3000
    lib = umas.load_library()
    new = lambda *s: torch.randn(*s, device="cuda").bfloat16()  # noqa: E731
    x, r, g, dy, W, u = new(n, d), new(n, d), new(d), new(n, d), new(V, d) / 8, torch.rand(n, device="cuda")
    room = lambda b: torch.empty(b, dtype=torch.uint8, device="cuda")  # noqa: E731
    ws = [room(lib.umas_rms_norm_workspace_bytes(n, d)), room(lib.umas_clip_workspace_bytes(102))]
    draws = room(lib.umas_sample_tokens_workspace_bytes(n, d, V, 1))   # both graphs use it, one after the other
    few = room(lib.umas_sample_tokens_workspace_bytes(3, d, V, 1))
    training(x, r, g, dy, ws)
    answering(x, W, u, draws)
    answering(x[:3], W, u[:3], few)
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    with torch.cuda.graph(graphs[0]):
        outs.append(training(x, r, g, dy, ws) + answering(x, W, u, draws))
    with torch.cuda.graph(graphs[1]):
        outs.append(answering(r, W, u, draws) + answering(x[:3], W, u[:3], few))
    for _ in range(4):
        for t in (x, r, dy):
            t.copy_(new(n, d))
        u.copy_(torch.rand(n, device="cuda"))
        for group in outs:
            for o in group:
                o.view(torch.uint8).fill_(0x55)
        draws.fill_(0xFF)
        umas.umas_sample_logits(torch.randn(7, 5000, device="cuda"), torch.rand(7, device="cuda"), top_p=0.5)   # other work between the replays
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert same(outs[0], training(x, r, g, dy, ws) + answering(x, W, u, draws))
        assert same(outs[1], answering(r, W, u, draws) + answering(x[:3], W, u[:3], few))


def test_calls_on_two_streams_at_once():
    n, d, V = 40, 256, 20000
    new = lambda *s: torch.randn(*s, device="cuda").bfloat16()  # noqa: E731
    x, r, g, dy, W, u = new(2, 200, d), new(2, 200, d), new(d), new(2, 200, d), new(V, d) / 8, torch.rand(2, n, device="cuda")
    work = lambda i: training(x[i], r[i], g, dy[i], (None, None)) + answering(x[i][:n].contiguous(), W, u[i], None)  # noqa: E731
    want = [work(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(work(i))
    torch.cuda.synchronize()
    for i in range(2):
        for outputs in got[i]:
            assert same(outputs, want[i])


# ------------------------------------------------------------------------------------------------ together
def step64(x, r, g, W, said, rows, eps, coef):
    """The loss and gradients of cross entropy behind the norm, hidden going on past it with coefficient coef, in float64."""
    x, r, g, W, coef = (t.double().cpu() for t in (x, r, g, W, coef))
    leaves = [t.requires_grad_() for t in (x, g, W)]
    s = x[rows] + r[rows]
    H = s * torch.rsqrt(s.square().mean(1, keepdim=True) + eps) * g
    loss = torch.nn.functional.cross_entropy(H @ W.T, said[rows].long().cpu())
    return [loss.detach()] + list(torch.autograd.grad(loss + (s * coef[rows]).sum(), leaves))


@pytest.mark.parametrize("n,d,V", [(37, 96, 257), (1, 8, 5), (130, 64, 200)])
def test_a_step_from_the_norm_to_clipped_gradients(n, d, V):
    """Tokens drawn from the head behind the norm are what it is taught, in rows that a padded batch selects; the rows behind hold no numbers."""
    gen = torch.Generator("cuda").manual_seed(n)
    new = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    pad, eps = 5, 1e-5
    x, r, g, W = new(n + pad, d), new(n + pad, d), 1 + 0.1 * new(d), new(V, d) * 0.3
    coef = new(n + pad, d) * 1e-2
    x[n:], coef[n:] = math.nan, 0.0
    rows = torch.arange(n, dtype=torch.int32, device="cuda")
    u = torch.rand(n + pad, device="cuda", generator=gen)
    y, hidden, inv = umas.umas_rms_norm(x, g, r, eps=eps)
    ids, logp, _ = umas.umas_sample_tokens(y, W, u, rows, top_p=0.9)
    assert (ids[n:] == -1).all() and ((ids[:n] >= 0) & (ids[:n] < V)).all()
    again = umas.umas_policy_logprobs(y, W, ids, rows)[0]
    assert ((again - logp)[:n].abs() <= 1e-5 * (1 + logp[:n].abs())).all()
    stats, _, dH, dW = umas.umas_cross_entropy_fwd_bwd(y, W, ids, rows)
    dx, dgain = umas.umas_rms_norm_bwd(dH, hidden, g, inv, coef)
    loss_o, dx_o, dg_o, dW_o = step64(x, r, g, W, ids, torch.arange(n), eps, coef)
    assert abs(float(umas.read_target_stats(stats)["loss"][0]) - float(loss_o)) <= 1e-5 * (1 + float(loss_o))
    for got, want, name in ((dx, dx_o, "dx"), (dgain, dg_o, "dgain"), (dW, dW_o, "dW")):
        assert float((got.double().cpu() - want).abs().max()) <= 1.6e-3 * float(want.abs().max()), name
    assert not dx[n:].any()
    norm = math.sqrt(sum(float(t.double().square().sum()) for t in (dx, dgain, dW)))
    want = [t * 0.5 for t in (dx, dgain, dW)]
    cstats, clipped = umas.umas_clip_gradients([dx, dgain, dW], norm / 2)
    s = umas.read_clip_stats(cstats)[0]
    assert abs(s["norm"] - norm) <= 2 * F * norm and s["n_not_finite"] == 0
    for a, b in zip(clipped, want):
        assert ((a - b).abs() <= 4 * F * b.abs() + 1e-37).all()
