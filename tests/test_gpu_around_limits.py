"""The draws, the norm and the clipping at the ends of what their numbers hold: temperatures close to 0, logits of many binades, borders on which sums that are
taken in another order fall to the other side, infinite gains, factors below float32's normal numbers.

Tolerances, from the arithmetic; f = 2^-24.
  draws     as in check_draws: tokens are equal, logp and logq are off by what their sums are"""
import math

import numpy as np
import pytest
import torch

import paper_2605_26646_amd as umas
from tests.test_gpu_around import DT, check_draws, device
from tests.test_gpu_around_edges import check, same

pytestmark = pytest.mark.gpu
F = 2.0 ** -24


# ------------------------------------------------------------------------------------------------ draws
def close_logits(tops, V, dtype, rng):
    """A row for each largest logit: it stands at up to three places, some of the numbers next below it at others, the rest is far below, masked by -infinity or by the
    lowest number.  Every unit of 1024 tokens but the last starts with masked ones, and one holds nothing else."""
    step = 1 if dtype == "f32" else 1 << 16                          # of float32's bits from one number to the next
    z = np.empty((len(tops), V), np.float32)
    for i, top in enumerate(np.float32(tops)):
        z[i] = -np.inf if i % 2 else torch.finfo(DT[dtype]).min
        some = rng.permutation(np.arange(V // 3, V))
        z[i, some[:V // 4]] = top - np.abs(top) * (1 + rng.random(V // 4)) - 1
        bits = np.full(V // 8, top, np.float32).view(np.int32)
        below = rng.integers(1, 12, V // 8) * step
        z[i, some[V // 4:V // 4 + V // 8]] = (bits + np.where(top > 0, -below, below)).astype(np.int32).view(np.float32)
        z[i, some[-1 - i % 3:]] = top
    return z


def without_dust(z, t):
    """Weights below 1e-290 count as none, which a float64 oracle holds on to down to 1e-323: tokens around there become -infinity."""
    with np.errstate(over="ignore"):
        gap = (z - z.max(1, keepdims=True)) / np.asarray(t, np.float64).reshape(-1, 1)
    return np.where((gap < -600) & (gap > -780), -np.inf, z)


TOPS = [s * 1.37 * 2.0 ** e for e in range(-3, 17) for s in (1, -1)] + [1.0, -2.0, 20.0, 2.0 ** 31 * 1.1, 2.0 ** 31 * 1.9, -(2.0 ** 32) * 0.7, 2.0 ** 40]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [7, 1100, 2100])
def test_temperatures_close_to_0_beside_largest_logits_of_many_binades(V, dtype):
    rng = np.random.default_rng([21, V])
    n = len(TOPS)
    _, rows = device(close_logits(TOPS, V, dtype, rng), dtype)
    for t in [1.0] + [10.0 ** -e for e in range(3, 13)]:
        t = float(np.float32(t * (1 + 0.5 * rng.random())))
        z, zh = device(without_dust(rows, t), dtype)
        for u in (np.zeros(n, np.float32), rng.random(n).astype(np.float32), np.full(n, 1 - F, np.float32)):
            check_draws(zh, u, dict(temperature=t), umas.umas_sample_logits(z, torch.from_numpy(u).cuda(), temperature=t), V)
        u = 0.01 + 0.98 * rng.random(n).astype(np.float32)
        for s in (dict(top_p=0.7), dict(top_k=2), dict(min_p=0.5), dict(temperature=torch.full((n,), t, device="cuda"))):
            plain = {k: v for k, v in s.items() if k != "temperature"}
            check_draws(zh, u, dict(temperature=t, **plain), umas.umas_sample_logits(z, torch.from_numpy(u).cuda(), **{"temperature": t, **s}), V)


def test_a_cold_draw_of_a_wide_vocabulary_is_the_largest_logit():
    n, V = 40, 151936
    gen = torch.Generator("cuda").manual_seed(3)
    z, u = torch.randn(n, V, device="cuda", generator=gen) * 5, torch.rand(n, device="cuda", generator=gen)
    best = z.max(1)
    logp = torch.log_softmax(z.double(), 1).gather(1, best.indices[:, None])[:, 0]
    for t in (1e-6, 1e-7, 1e-8, 1e-9, 1e-10):
        for s in (dict(), dict(top_p=0.9)):
            ids, got, logq = umas.umas_sample_logits(z, u, temperature=t, **s)
            # the second largest logit is 1e-4 below and more, but for a chance of 1e-3 a row; that one is a draw between two
            sure = z.topk(2, 1).values.diff(dim=1).abs()[:, 0] > 800 * t
            assert sure.sum() > n // 2 and torch.equal(ids[sure], best.indices[sure].int()) and not logq[sure].any()
            assert ((got.double() - logp)[sure].abs() <= 40 * 2.0 ** -22 + F * logp[sure].abs()).all()   # |x| + 2 <= 40 where p counts
            assert (ids >= 0).all() and got.isfinite().all()


@pytest.mark.parametrize("scale,min_p,most", [(4.0, 0.05, 60), (1.0, 0.2, 500)])
def test_rows_of_which_min_p_leaves_fewer_tokens_than_top_k(scale, min_p, most):
    """They are decided by the list of what is left: no launch for spread rows gets one.  Its lists, 4096 places a row, are the last that lies in the workspace."""
    n, V = 60, 50000
    gen = torch.Generator("cuda").manual_seed(7)
    z, u = torch.randn(n, V, device="cuda", generator=gen) * scale, torch.rand(n, device="cuda", generator=gen)
    left = (z >= z.max(1, keepdim=True).values + math.log(min_p)).sum(1)
    z, u = z[left <= most], u[left <= most]
    n = len(z)
    assert n >= 20
    lib = umas.load_library()
    ws = torch.full((lib.umas_sample_logits_workspace_bytes(n, V),), 0x5A, dtype=torch.uint8, device="cuda")
    k = most + 1
    for s in (dict(top_k=k), dict(top_k=k, top_p=0.8), dict(top_k=20000), dict(top_k=20000, top_p=0.8)):
        got = umas.umas_sample_logits(z, u, min_p=min_p, workspace=ws, **s)
        check(z, u, got, min_p=min_p, **s)
        assert (ws[-n * 4096 * 4:] == 0x5A).all(), s
        one = [umas.umas_sample_logits(z[i:i + 1], u[i:i + 1], min_p=min_p, **s) for i in range(n)]
        assert same(got, [torch.cat(x) for x in zip(*one)]), s
        k_of = torch.full((n,), s["top_k"], device="cuda", dtype=torch.int32)
        assert same(got, umas.umas_sample_logits(z, u, **{**s, "top_k": k_of}, min_p=min_p, workspace=ws)) and (ws[-n * 4096 * 4:] == 0x5A).all(), s
    if most <= 64:                                                   # a top_k that is held to be decided by the front, by one workgroup a row
        check(z, u, umas.umas_sample_logits(z, u, min_p=min_p, top_k=64), min_p=min_p, top_k=64)


@pytest.mark.parametrize("n", [1, 2, 5])
def test_a_border_of_top_p_among_equal_logits_beside_weights_that_are_no_whole_number(n):
    """One token of weight 1, 3000 equal ones of 64 units (2^-46 of it each), and 30 000 of 0.45 units, which count in the mass that top_p is of and else as nothing.  u = 1 draws the last token
    that is kept: the border's.  A row alone lists the equal ones; among others a workgroup finds more of them than it has room for, and they are gone through by bits."""
    V, at, many = 33001, 4096, 3000
    z = torch.full((V,), -math.log(2) * (46 - math.log2(0.45)))
    z[at:at + many] = -40 * math.log(2)
    z[0] = 0
    w = torch.exp(z.double())
    assert abs(w[at] * 2.0 ** 46 - 64) < 1e-3 and 0.44 < w[1] * 2.0 ** 46 < 0.46
    z, u = z.cuda().expand(n, V).contiguous(), torch.ones(n, device="cuda")
    all_of = float(w.sum())
    for reach, last in ((1 + 1500.5 * float(w[at]), at + 1500), (1 + 0.5 * float(w[at]), at), (1 + 2999.5 * float(w[at]), at + 2999),
                        (all_of - 5000 * 2.0 ** -46, at + many - 1)):        # ... beyond all whole numbers: what has one is kept
        ids, _, logq = umas.umas_sample_logits(z, u, top_p=reach / all_of)
        assert ids.tolist() == [last] * n, (reach, ids.tolist())
        assert (logq + 40 * math.log(2)).abs().max() <= 1e-5                 # 2 f of 28, and the mass, which is 1 to 3e-9


@pytest.mark.parametrize("V", [1000, 1024, 5000, 600000])
def test_borders_that_rounding_decides_fall_the_same_way_alone_and_among_others(V):
    """A row of two or four equal parts: at u = 1/4, 1/2 and 3/4 the running mass and what it has to pass are the same number, but for the order of sums."""
    n = 60 if V < 10000 else 12
    gen = torch.Generator("cuda").manual_seed(V)
    z = torch.cat([torch.randn(n // 2, V // p, device="cuda", generator=gen).repeat(1, p) for p in (2, 4)])
    n = len(z)
    for j, t in ((1, 1.0), (2, 0.7), (3, 1.9)):
        u, t_of = torch.full((n,), j / 4, device="cuda"), torch.full((n,), t, device="cuda")
        got = umas.umas_sample_logits(z, u, temperature=t_of)
        one = [umas.umas_sample_logits(z[i:i + 1], u[i:i + 1], temperature=t_of[i:i + 1]) for i in range(n)]
        assert same(got, [torch.cat(x) for x in zip(*one)]), t
        assert same(got, umas.umas_sample_logits(z, u, temperature=float(t_of[0]))), t
        k_of = torch.zeros(n, dtype=torch.int32, device="cuda")
        assert same(got, umas.umas_sample_logits(z, u, temperature=float(t_of[0]), top_k=k_of)), t
        rows = slice(0 if j == 2 else n // 2, n)                     # whose parts end there: the last token of one or the first of the next
        assert ((got[0][rows].long() - V // 4 * j).abs() <= 1).all()


# ------------------------------------------------------------------------------------------------ norm
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 4096), ("f32", 33), ("f32", 3000)])
def test_a_row_whose_norm_is_infinite_in_places_is_no_number_in_8_bits(dtype, d):
    for big in (math.inf, -math.inf, torch.finfo(DT[dtype]).max):      # the last: a normalised 2 times the largest number is beyond it
        x = torch.randn(9, d, device="cuda").to(DT[dtype])
        x[:, 3] = 0
        x[::2, 3] = 2 * math.sqrt(d)                                   # normalised 1.7 to 2: sqrt(d (4 d) / (4 d + d))
        gain = torch.ones(d, device="cuda").to(DT[dtype])
        gain[3] = big
        y = umas.umas_rms_norm(x, gain)[0]
        q, scale, _, _ = umas.umas_rms_norm_quantized(x, gain)
        assert y[::2, 3].isinf().all() and scale[::2].isnan().all() and q[::2].float().isnan().all()
        if math.isfinite(big):
            assert (scale[1::2] > 0).all() and scale.isfinite()[1::2].all() and q[1::2].float().isfinite().all()
        else:
            assert scale[1::2].isnan().all() and q[1::2].float().isnan().all()   # 0 times infinity


@pytest.mark.parametrize("d", [64, 512, 1024, 2048, 3584, 8192])
def test_quotients_on_a_border_of_8_bits_go_to_the_even_side_in_any_call(d):
    """448 s gain / max |s gain|: products of two bf16 numbers have 16 bits, so float64 has the quotient to 2^-53, and what lies on no border lies 2^-24 of itself and more from each."""
    n = 2100                                                           # more rows than those that a workgroup each takes
    torch.manual_seed(d)
    x, r = torch.randn(n, d).bfloat16(), (torch.randn(n, d) * (0.5 + 4 * torch.rand(n, 1))).bfloat16()
    gain = (1 + 0.3 * torch.randn(d)).bfloat16()
    x, r, g = x.cuda(), r.cuda(), gain.cuda()
    q, scale, hidden, inv = umas.umas_rms_norm_quantized(x, g, r)
    t = hidden.cpu().double() * gain.double()
    t = 448 * t / t.abs().max(1, keepdim=True).values
    bits = torch.arange(127, dtype=torch.uint8)
    value = bits.view(torch.float8_e4m3fn).double()
    border = (value[1:] + value[:-1]) / 2
    at = torch.bucketize(t.abs(), border)                              # the nearest one's bits; of what lies on a border the lower one's
    on = border[at.clamp(max=125)] == t.abs()
    assert on.sum() > n * d / 20000                                    # they do not lie there by chance alone
    at = torch.where(on & (at % 2 == 1), at + 1, at)
    got = q.cpu().view(torch.uint8)
    assert torch.equal((got & 127).long(), at) and torch.equal((got & 127 != 0) & (got > 127), (at != 0) & (t < 0))
    for rows in (1, 5, 300):
        few = umas.umas_rms_norm_quantized(x[:rows], g, r[:rows])
        assert torch.equal(few[0].view(torch.uint8), q[:rows].view(torch.uint8))


# ------------------------------------------------------------------------------------------------ clipping
@pytest.mark.parametrize("max_norm", [1.0, 1e-4, 1e-20, 1e-30])
def test_factors_below_the_normal_numbers_of_32_bits(max_norm):
    """Norms of 1e38 and more over a small bound: out is c g to 2 f and its rounding, whatever float32 has for c."""
    for size, big in ((1, 3e38), (9001, 3e38), (20000, 1e37), (5000, 2e30)):
        grads = [(big * (0.5 + 0.5 * torch.rand(size, device="cuda"))), -(big * (0.5 + 0.5 * torch.rand(size + 3, device="cuda"))).bfloat16(), torch.ones(5, device="cuda")]
        norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
        c = max_norm / norm
        out = [torch.full_like(g, 7) for g in grads]
        stats, _ = umas.umas_clip_gradients(grads, max_norm, out=out)
        s = umas.read_clip_stats(stats)[0]
        assert s["n_not_finite"] == 0 and (s["norm"] == np.inf if norm > 3.5e38 else abs(s["norm"] / norm - 1) < 2 * F)
        assert abs(float(s["scale"]) - c) <= 2 * F * c + 2.0 ** -149
        for o, g in zip(out, grads):
            want, u = g.double() * c, 2.0 ** -8 if g.dtype == torch.bfloat16 else 0.0
            # half a step of the smallest numbers, which bf16's are of 2^-133
            assert ((o.double() - want).abs() <= (u + 3 * F) * want.abs() + (2.0 ** -134 if u else 2.0 ** -150)).all(), (size, big)
        umas.umas_clip_gradients(grads, max_norm)
        assert same(grads, out)
