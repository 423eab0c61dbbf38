"""Largest logits, cross entropy and distillation on the GPU against the oracle, at the sizes where tiles, wavefronts and chunks end and on inputs whose
masks leave something empty.

Tolerances, from the arithmetic.  u = 2^-8 (a rounding to bf16), f = 2^-24.  Logits are float32 sums of exact products, lse a float32 logarithm of a sum of V
terms: p = exp(z - lse) has the relative error d = 4 f (|z| + |lse|) + 8 f (two exponentials, the sum's own rounding).  An entry of dz is rounded to bf16 once,
as a numerator or as a target's entry; for dW the scaled row of H is rounded as well and, where dW is bf16, the sum:
  |dH - dH_o| <= 1.05 [(u + V 2^-23) |dz| |W| + D |W| + u |dH_o|],   |dW - dW_o| <= 1.05 [(2 u + u^2 + n 2^-23) |dz|^T |H| + D^T |H| + u |dW_o|]
where D is what d does to the entries, d |g| a' p everywhere, and at a target also the float32 rounding of a difference of a' p and t, 8 f |g| (a' p + t).
Norm-wise both arrays meet 1e-2, the bar of bf16 gradients here.  The float32 path sums in float64: 1e-5.  Log-probs, divergences, logsumexps: 2e-2 absolute
is the bar of bf16 scores; these meet d |z| + 1e-5 in float32 sums, and that is asked for."""
import numpy as np
import pytest
import torch

import paper_2605_26646_amd as umas
from oracle import umas_oracle as orc
from paper_2605_26646_amd import binding
from tests import parity as P

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def arrays(seed, n, d, V, dtype, scale=1.0, grid=False):
    """Hidden states and head as float64 numpy (the values the device has) and on the device."""
    rng = np.random.default_rng([77, seed])
    H, W = rng.normal(size=(n, d)), rng.normal(size=(V, d)) * scale / max(np.sqrt(d), 1)
    if grid:                                                  # every product and sum is exact in float32
        H, W = np.round(H * 4) / 4, np.round(W * 64) / 64
    out = []
    for X in (H, W):
        t = torch.from_numpy(X.astype(np.float32)).to(DT[dtype])
        out += [t.double().numpy(), t.cuda()]
    return out[0], out[2], out[1], out[3], rng


def selection(rng, n, kind):
    if kind == "all":
        return None, None
    rows = np.sort(rng.permutation(n)[:max(1, (3 * n) // 4)]) if kind == "some" else rng.permutation(n)
    return rows, torch.from_numpy(rows.astype(np.int32)).cuda()


def cuda(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x).astype(dtype))).cuda()


# ------------------------------------------------------------------------------------------------ largest logits
SIZES = [(1, 8, 1, 1), (1, 64, 5, 8), (2, 24, 63, 64), (3, 72, 64, 64), (5, 64, 255, 20), (16, 128, 256, 64), (17, 64, 257, 33), (33, 512, 1000, 10),
         (64, 200, 3001, 64), (65, 64, 3001, 5), (127, 136, 512, 64), (128, 64, 769, 1), (129, 64, 1025, 50), (255, 64, 300, 64), (257, 72, 2049, 64),
         (520, 64, 5000, 7)]


def check_top(H, W, k, rows, got, exact):
    ids_o, top_o, lse_o = orc.top_logits(H, W, k, rows)
    ids, top, lse = (x.cpu().numpy() for x in got)
    if exact:
        assert np.array_equal(ids, ids_o) and np.array_equal(top, top_o.astype(np.float32))
    else:                                                     # equal to rounding: the tokens are distinct, carry their logits, and nothing larger is left out
        tol = 1e-5 * (1 + np.abs(top_o[np.isfinite(top_o)]).max(initial=0))
        fin = np.isfinite(top_o)
        assert np.array_equal(fin, np.isfinite(top)) and np.abs(top[fin] - top_o[fin]).max(initial=0) <= tol
        for i in range(len(ids)):
            have = ids[i][ids[i] >= 0]
            assert len(set(have)) == len(have) and (np.diff(top[i][:len(have)]) <= 0).all()
            if len(have):
                assert np.abs(W[have] @ H[i] - top[i][:len(have)]).max() <= tol
    assert np.abs(lse - lse_o).max() <= 1e-5 * (1 + np.abs(lse_o).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("grid", [True, False])
@pytest.mark.parametrize("n,d,V,k", SIZES)
def test_top_logits(n, d, V, k, grid, dtype):
    for kind in ("all", "some", "order"):
        H, W, Hd, Wd, rng = arrays(n + V + k, n, d, V, dtype, grid=grid)
        rows, sel = selection(rng, n, kind)
        check_top(H, W, k, rows, umas.umas_top_logits(Hd, Wd, k, sel), grid)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["rising", "falling", "equal"])
@pytest.mark.parametrize("n,V", [(1, 4000), (40, 4000), (200, 6001), (700, 3000)])
def test_top_logits_of_sorted_and_equal_logits(n, V, order, dtype):
    """Every logit beats all before it, none does, all are the same."""
    d, k = 8, 64
    W = np.zeros((V, d))
    v = np.arange(V)
    if order != "equal":                                      # 64 a + b with a, b < 128: exact in bf16
        W[:, 0], W[:, 1] = v // 64, v % 64
    H = np.zeros((n, d))
    H[:, 0], H[:, 1] = 64, 1
    if order == "falling":
        H = -H
    Hd, Wd = cuda(H, np.float32).to(DT[dtype]), cuda(W, np.float32).to(DT[dtype])
    ids, top, _ = umas.umas_top_logits(Hd, Wd, k)
    z = W @ H[0]
    want = np.lexsort((v, -z))[:k]
    assert (ids.cpu().numpy() == want).all() and (top.cpu().numpy() == z[want]).all()


def test_top_logits_that_are_no_numbers_are_not_listed():
    H, W, Hd, Wd, rng = arrays(5, 140, 64, 700, "bf16", grid=True)
    bad_row, inf_tok, nan_tok = 7, 11, 400
    Wd[nan_tok] = float("nan")
    Hd[:, 0] = 1.0
    Wd[:, 0] = 0.0
    Wd[inf_tok, 0] = -float("inf")
    Hd[bad_row] = float("nan")
    H, W = Hd.double().cpu().numpy(), Wd.double().cpu().numpy()
    for n in (3, 40, 140):
        ids, top, lse = umas.umas_top_logits(Hd[:n].contiguous(), Wd, 64)
        z = H[:n] @ np.where(np.isfinite(W), W, 0).T
        z[:, [inf_tok, nan_tok]] = -np.inf
        for i in range(n):
            if i == bad_row:
                assert (ids[i] == -1).all() and (top[i] == -np.inf).all()
            else:
                want = np.lexsort((np.arange(700), -z[i]))[:64]
                assert (ids[i].cpu().numpy() == want).all()


def test_top_logits_do_not_depend_on_the_workspace_or_on_other_rows():
    H, W, Hd, Wd, rng = arrays(6, 900, 64, 3000, "bf16", grid=True)
    lib = umas.load_library()
    sizes = [getattr(lib, "umas_top_logits_workspace_bytes" + w)(900, 64, 3000, 40, 1) for w in ("_min", "")]
    want = umas.umas_top_logits(Hd, Wd, 40)
    for b in (sizes[0], (sizes[0] + sizes[1]) // 2, sizes[1]):
        ws = torch.full((b,), 0xFF, dtype=torch.uint8, device="cuda")
        got = umas.umas_top_logits(Hd, Wd, 40, workspace=ws)
        assert all(torch.equal(a, c) for a, c in zip(got[:2], want[:2])) and (got[2] - want[2]).abs().max() < 1e-5
    for rows in ([5], [899], list(range(100, 160))):
        sel = torch.tensor(rows, dtype=torch.int32, device="cuda")
        got = umas.umas_top_logits(Hd, Wd, 40, sel)
        assert torch.equal(got[0][rows], want[0][rows]) and torch.equal(got[1][rows], want[1][rows])
        rest = torch.ones(900, dtype=torch.bool, device="cuda")
        rest[rows] = False
        assert (got[0][rest] == -1).all() and not got[1][rest].any() and not got[2][rest].any()


@pytest.mark.parametrize("n,d,V,k", [(1, 2048, 50001, 64), (24, 3584, 30001, 50), (60, 2048, 20001, 20), (300, 1544, 50001, 32), (2500, 264, 40001, 64)])
def test_top_logits_of_large_heads(n, d, V, k):
    g = torch.Generator(device="cuda").manual_seed(n)
    H = torch.round(torch.randn(n, d, device="cuda", generator=g) * 8).div_(8).bfloat16()
    W = torch.round(torch.randn(V, d, device="cuda", generator=g) * 8).div_(256).bfloat16()
    z = H.double() @ W.double().T
    key = (z * 2.0 ** 12).round().long() * 2 ** 20 + torch.arange(V - 1, -1, -1, device="cuda")
    want = V - 1 - (key.topk(k, dim=1).values & (2 ** 20 - 1))
    ids, top, lse = umas.umas_top_logits(H, W, k)
    assert torch.equal(ids.long(), want) and torch.equal(top.double(), z.gather(1, want))
    assert (lse - torch.logsumexp(z, 1)).abs().max() < 1e-4


# ------------------------------------------------------------------------------------------------ targets
def stats_of(r, role, n_roles, norm):
    out = []
    for k in range(1 + n_roles):
        q = np.ones(len(r["rows"]), bool) if k == 0 else role[r["rows"]] == k - 1
        taught = q & (r["mass"] > 0)
        out.append((r["row_loss"][q].sum() / (norm if k == 0 else max(q.sum(), 1)), r["w"][q].mean() if q.any() else 0,
                    r["entropy"][taught].mean() if taught.any() else 0, r["lse"][taught].mean() if taught.any() else 0, q.sum(), (q & ~taught).sum()))
    return out


def check_taught(r, H, W, ids, masses, got, dtype, dW_dtype, role, n_roles, norm, z_coef, dW_before=None):
    """The call's outputs against the oracle's dict r."""
    stats, row, dH, dW = got
    rows, n, V = r["rows"], len(H), len(W)
    z = np.asarray(H)[rows] @ np.asarray(W).T if len(rows) else np.zeros((0, V))
    z[r["mass"] <= 0] = 0
    f = 2.0 ** -24
    zl = np.abs(z).max(initial=0) + np.abs(r["lse"]).max(initial=0)
    tol_row = 1e-5 * (1 + np.abs(r["row"]).max(initial=0)) + (8 * f * zl if dtype == "bf16" else 0)
    assert np.abs(row.cpu().numpy() - r["row"]).max(initial=0) <= tol_row
    s = umas.read_target_stats(stats)
    r["row_loss"] = np.where(r["w"] != 0, r["w"] * ((-1 if masses is None else 1) * r["row"][rows] + z_coef * r["lse"] ** 2), 0) if len(rows) else np.zeros(0)
    for k, (loss, wm, ent, lse, cnt, ign) in enumerate(stats_of(r, role, n_roles, norm)):
        big = np.abs(r["row_loss"]).max(initial=0) * max(1, cnt / norm)
        assert abs(s["loss"][k] - loss) <= 1e-5 * (1 + big) + 8 * f * zl and abs(s["weight_mean"][k] - wm) <= 1e-6 * (1 + abs(wm))
        assert abs(s["entropy_mean"][k] - ent) <= 1e-5 * (1 + abs(ent)) + 16 * f * zl * (1 + zl) and abs(s["lse_mean"][k] - lse) <= 1e-5 * (1 + abs(lse))
        assert s["n_scored"][k] == cnt and s["n_ignored"][k] == ign
    assert dH.dtype == DT[dtype]
    dH = dH.double().cpu().numpy()
    idle = np.ones(n, bool)
    idle[rows[(r["w"] != 0) & (r["mass"] > 0)]] = False
    assert not dH[idle].any()
    want_W = r["dW"] + (0 if dW_before is None else dW_before)
    if dtype == "f32":
        P.close(dH, r["dH"], 1e-5, "dH")
        if dW is not None:
            P.close(dW.cpu().numpy(), want_W, 1e-5, "dW")
        return
    u, A = 2.0 ** -8, np.abs(r["dz"])
    p = np.exp(z - r["lse"][:, None]) * (r["mass"] > 0)[:, None]
    ga = np.abs(r["w"] / norm * (r["mass"] + 2 * z_coef * r["lse"]))[:, None] * p
    D = ga * (4 * f * (np.abs(z) + np.abs(r["lse"])[:, None]) + 8 * f)
    for q, i in enumerate(rows):
        t = [1.0] if masses is None else masses[i]
        for j, v in enumerate(np.atleast_1d(ids[i])):
            if r["mass"][q] > 0 and t[j] > 0:
                D[q, v] += 8 * f * (ga[q, v] + abs(r["w"][q]) / norm * t[j])
    bound = np.zeros(dH.shape)
    Wa, Ha = np.abs(W), np.abs(np.where(np.isfinite(H), H, 0))[rows]
    bound[rows] = 1.05 * ((u + V * 2.0 ** -23) * (A @ Wa) + D @ Wa + u * np.abs(r["dH"][rows])) + 1e-30
    P.close_bounded(dH[rows], r["dH"][rows], bound[rows], 1e-2, "dH")
    if dW is None:
        return
    assert dW.dtype == DT[dW_dtype]
    bound = 1.05 * ((2 * u + u * u + len(rows) * 2.0 ** -23) * (A.T @ Ha) + D.T @ Ha + (u if dW_dtype == "bf16" else 2 * f) * np.abs(want_W)) + 1e-30
    P.close_bounded(dW.double().cpu().numpy(), want_W, bound, 1e-2, "dW")


def lean(H, W, ids, rng, by=6.0):
    """Hidden states that lean towards a token, so that rows are of every degree of confidence."""
    v = np.where((ids >= 0) & (ids < len(W)), ids, 0)
    w = W[v]
    return H + by * rng.random((len(H), 1)) * w / np.maximum((w * w).sum(1, keepdims=True), 1e-3)


TAUGHT = [(1, 8, 1, 1), (1, 64, 300, 7), (3, 24, 63, 3), (30, 72, 256, 64), (64, 64, 257, 20), (65, 136, 1000, 10), (128, 64, 511, 33), (129, 64, 512, 2),
          (200, 264, 3001, 16), (256, 64, 769, 64), (257, 72, 2049, 5), (600, 200, 1500, 12)]


@pytest.mark.parametrize("dtype,dW_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("n,d,V,k", TAUGHT)
@pytest.mark.parametrize("kind", ["ce", "renormalised", "tail"])
def test_targets(n, d, V, k, kind, dtype, dW_dtype):
    for seed, sel_kind in enumerate(("all", "some", "order")):
        H, W, _, Wd, rng = arrays(n + V + seed, n, d, V, dtype, scale=2.0)
        rows, sel = selection(rng, n, sel_kind)
        k_ = 1 if kind == "ce" else min(k, V)
        ids = np.stack([rng.permutation(V)[:k_] for _ in range(n)])
        Hd = cuda(lean(H, W, ids[:, 0], rng), np.float32).to(DT[dtype])
        H = Hd.double().cpu().numpy()
        gone = rng.random((n, k_)) < 0.15                     # places that do not count, in some rows all of them
        gone |= (rng.random((n, 1)) < 0.1)
        ids = np.where(gone, rng.choice([-1, -100, V, 2 ** 31 - 1], size=ids.shape), ids)
        weight = (rng.normal(size=n) * (rng.random(n) > 0.2)).astype(np.float32)
        role = rng.integers(-1, 3, n)
        norm = (len(rows) if rows is not None else n) + (17 if seed == 2 else 0)
        kw = dict(norm_rows=norm if seed == 2 else 0)
        z_coef = 0.0 if seed == 0 else 0.05
        before = None
        if seed == 1:                                         # added to
            before = rng.normal(size=(V, d)).astype(np.float32) * 0.01
            kw.update(dW=cuda(before, np.float32).to(DT[dW_dtype]), accumulate_dW=True)
            before = kw["dW"].double().cpu().numpy()
        elif dW_dtype != dtype:
            kw.update(dW=torch.full((V, d), float("nan"), device="cuda"))
        args = (sel, cuda(weight, np.float32), cuda(role, np.int32), 2)
        if kind == "ce":
            ids = ids[:, 0]
            r = orc.cross_entropy(H, W, ids, rows, weight, z_coef, norm)
            got = umas.umas_cross_entropy_fwd_bwd(Hd, Wd, cuda(ids, np.int32), *args, z_coef=z_coef, **kw)
            masses = None
        else:
            z_coef = 0.0
            l = rng.normal(size=ids.shape).astype(np.float32) * 2
            l[rng.random(ids.shape) < 0.05] = -np.inf
            l = np.where(gone, np.nan, l).astype(np.float32)
            lse = None if kind == "renormalised" else (3.0 + rng.random(n) * 4).astype(np.float32)
            masses = orc.teacher_masses(ids, l, lse, V)
            r = orc.distill(H, W, ids, l, lse, rows, weight, norm)
            got = umas.umas_distill_fwd_bwd(Hd, Wd, cuda(ids, np.int32), cuda(l, np.float32), None if lse is None else cuda(lse, np.float32), *args, **kw)
        check_taught(r, H, W, ids, masses, got, dtype, dW_dtype, role, 2, norm, z_coef, before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_token_in_several_places(dtype):
    n, d, V = 70, 64, 300
    H, W, Hd, Wd, rng = arrays(3, n, d, V, dtype)
    ids = rng.integers(0, 6, (n, 9))
    l = rng.normal(size=(n, 9)).astype(np.float32)
    r = orc.distill(H, W, ids, l)
    got = umas.umas_distill_fwd_bwd(Hd, Wd, cuda(ids, np.int32), cuda(l, np.float32))
    check_taught(r, H, W, ids, orc.teacher_masses(ids, l, None, V), got, dtype, dtype, np.zeros(n), 0, n, 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [40, 200, 600])
def test_rows_that_teach_nothing_may_hold_anything(n, dtype):
    """Ignored rows and rows of weight 0 whose hidden states are infinities and no numbers, the last row among them."""
    d, V = 64, 700
    H, W, Hd, Wd, rng = arrays(n, n, d, V, dtype)
    ids = rng.integers(0, V, n)
    weight = np.ones(n, np.float32)
    ids[[0, 5, n - 1]] = -100
    weight[[3, n - 2]] = 0
    for i, x in ((0, np.nan), (5, np.inf), (n - 1, np.nan), (3, np.nan), (n - 2, -np.inf)):
        Hd[i] = x
    clean = H.copy()
    clean[[0, 5, n - 1, 3, n - 2]] = 0
    r = orc.cross_entropy(clean, W, ids, None, weight)
    stats, logp, dH, dW = umas.umas_cross_entropy_fwd_bwd(Hd, Wd, cuda(ids, np.int32), None, cuda(weight, np.float32))
    assert torch.isfinite(dH.float()).all() and torch.isfinite(dW.float()).all()
    assert abs(umas.read_target_stats(stats)["loss"][0] - r["loss"]) < 1e-5 * (1 + r["loss"])
    tol = 1e-5 if dtype == "f32" else 1e-2
    for x, o in ((dH, r["dH"]), (dW, r["dW"])):
        x = x.double().cpu().numpy()
        assert np.linalg.norm(x - o) <= tol * np.linalg.norm(o)
    good = np.setdiff1d(np.arange(n), [3, n - 2])
    assert np.abs(logp.cpu().numpy() - r["row"])[good].max() < 1e-4


@pytest.mark.parametrize("n", [40, 300])
def test_logits_far_above_the_targets_are_computed_once_more(n):
    """Rows whose targets have probabilities of e^-80 and less: their numerators would not serve."""
    d, V, k = 64, 900, 4
    H, W, Hd, Wd, rng = arrays(9, n, d, V, "bf16")
    ids = np.stack([rng.permutation(V)[:k] for _ in range(n)])
    for i in (2, n - 3):
        Hd[i] = Hd[i] * 60
    H = Hd.double().cpu().numpy()
    z = H @ W.T
    for i in (2, n - 3):
        ids[i] = np.argsort(z[i])[:k]
        assert z[i].max() - z[i][ids[i]].max() > 60
    l = rng.normal(size=(n, k)).astype(np.float32)
    weight = np.ones(n, np.float32)
    weight[5] = 0
    r = orc.distill(H, W, ids, l, None, None, weight)
    got = umas.umas_distill_fwd_bwd(Hd, Wd, cuda(ids, np.int32), cuda(l, np.float32), None, None, cuda(weight, np.float32))
    check_taught(r, H, W, ids, orc.teacher_masses(ids, l, None, V), got, "bf16", "bf16", np.zeros(n), 0, n, 0.0)


@pytest.mark.parametrize("dtype,dW_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("accumulate", [False, True])
def test_chunks_of_a_small_workspace(dtype, dW_dtype, accumulate):
    n, d, V = 900, 72, 1100
    H, W, Hd, Wd, rng = arrays(4, n, d, V, dtype)
    ids = rng.integers(0, V, n)
    code = {"bf16": 1, "f32": 0}
    lib = umas.load_library()
    least, full = (getattr(lib, "umas_cross_entropy_workspace_bytes" + w)(n, d, V, code[dtype], code[dW_dtype]) for w in ("_min", ""))
    before = cuda(rng.normal(size=(V, d)) * 1e-3, np.float32).to(DT[dW_dtype])
    r = orc.cross_entropy(H, W, ids)
    for b in (least, (least + full) // 2, max(least, full)):
        dW = before.clone()
        ws = torch.full((b,), 0xFF, dtype=torch.uint8, device="cuda")
        got = umas.umas_cross_entropy_fwd_bwd(Hd, Wd, cuda(ids, np.int32), dW=dW, accumulate_dW=accumulate, workspace=ws)
        check_taught(r, H, W, ids, None, got, dtype, dW_dtype, np.zeros(n), 0, n, 0.0, before.double().cpu().numpy() if accumulate else None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [20, 300])
def test_a_frozen_head_leaves_out_one_product_only(n, dtype):
    H, W, Hd, Wd, rng = arrays(8, n, 64, 1000, dtype)
    ids = cuda(rng.integers(0, 1000, n), np.int32)
    a = umas.umas_cross_entropy_fwd_bwd(Hd, Wd, ids)
    b = umas.umas_cross_entropy_fwd_bwd(Hd, Wd, ids, train_head=False)
    assert b[3] is None and torch.equal(a[1], b[1]) and torch.equal(a[0], b[0])
    x, y = a[2].double(), b[2].double()
    assert (x - y).norm() <= (2.0 ** -8 if dtype == "bf16" else 1e-6) * x.norm()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_selected_and_no_rows(dtype):
    H, W, Hd, Wd, rng = arrays(2, 20, 64, 300, dtype)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    ids = torch.zeros(20, dtype=torch.int32, device="cuda")
    l = torch.zeros(20, 3, device="cuda")
    stats, row, dH, dW = umas.umas_cross_entropy_fwd_bwd(Hd, Wd, ids, none)
    assert not row.any() and not dH.any() and not dW.any() and umas.read_target_stats(stats)["loss"][0] == 0
    dW.fill_(1.0)
    stats, row, dH, dW2 = umas.umas_distill_fwd_bwd(Hd, Wd, ids[:, None].repeat(1, 3), l, None, none, dW=dW, accumulate_dW=True)
    assert not row.any() and not dH.any() and (dW2 == 1).all() and umas.read_target_stats(stats)["n_scored"][0] == 0
    t, v, lse = umas.umas_top_logits(Hd, Wd, 3, none)
    assert (t == -1).all() and not v.any() and not lse.any()
    empty = torch.empty(0, 64, dtype=DT[dtype], device="cuda")
    stats, row, dH, dW = umas.umas_cross_entropy_fwd_bwd(empty, Wd, ids[:0])
    assert row.numel() == 0 and dH.numel() == 0 and not dW.any()
    assert [x.shape[0] for x in umas.umas_top_logits(empty, Wd, 3)] == [0, 0, 0]


def test_micro_batches_add_up():
    n, d, V, k = 500, 128, 2000, 8
    H, W, Hd, Wd, rng = arrays(12, n, d, V, "bf16")
    ids = np.stack([rng.permutation(V)[:k] for _ in range(n)])
    l = rng.normal(size=(n, k)).astype(np.float32)
    r = orc.distill(H, W, ids, l)
    dW = torch.zeros(V, d, device="cuda")
    loss, dH = 0.0, torch.zeros(n, d, device="cuda")
    for part in np.array_split(rng.permutation(n), 3):
        stats, _, h, _ = umas.umas_distill_fwd_bwd(Hd, Wd, cuda(ids, np.int32), cuda(l, np.float32), None, cuda(part, np.int32), dW=dW, accumulate_dW=True,
                                                   norm_rows=n)
        loss += umas.read_target_stats(stats)["loss"][0]
        dH += h.float()
    assert abs(loss - r["loss"]) < 1e-5 * (1 + r["loss"])
    for x, o in ((dH, r["dH"]), (dW, r["dW"])):
        assert np.linalg.norm(x.double().cpu().numpy() - o) <= 1e-2 * np.linalg.norm(o)


def test_gradient_against_differences_of_the_loss():
    """Of the call's own loss in float32, along random directions."""
    n, d, V, k = 60, 48, 400, 6
    H, W, Hd, Wd, rng = arrays(13, n, d, V, "f32")
    ids = cuda(np.stack([rng.permutation(V)[:k] for _ in range(n)]), np.int32)
    l, lse = cuda(rng.normal(size=(n, k)), np.float32), cuda(2 + rng.random(n), np.float32)

    def row_sums(H_, W_, which):                              # the rows' own outputs, summed in float64: the loss's float32 would not do
        if which == "ce":
            s, row, dH, dW = umas.umas_cross_entropy_fwd_bwd(H_, W_, ids[:, 0].contiguous())
            return -row.double().mean().item(), dH.double(), dW.double()
        s, row, dH, dW = umas.umas_distill_fwd_bwd(H_, W_, ids, l, lse)
        return row.double().mean().item(), dH.double(), dW.double()

    for which in ("ce", "distill"):
        _, dH, dW = row_sums(Hd, Wd, which)
        for X, D, put in ((Hd, dH, lambda x: (x, Wd)), (Wd, dW, lambda x: (Hd, x))):
            a = torch.from_numpy(rng.normal(size=tuple(X.shape))).cuda()
            e = 1e-2
            up, down = (row_sums(*put((X.double() + s * e * a).float()), which)[0] for s in (1, -1))
            # second differences are O(e^2), rows are float32: 1e-7 of a loss of about 6 over 2 e
            assert abs((up - down) / (2 * e) - (D * a).sum().item()) <= 2e-4 * (1 + (D * a).abs().sum().item())


@pytest.mark.parametrize("n", [40, 300])
def test_recorded_into_a_graph(n):
    d, V, k = 64, 3000, 8
    H, W, Hd, Wd, rng = arrays(20, n, d, V, "bf16", grid=True)
    ids = cuda(np.stack([rng.permutation(V)[:k] for _ in range(n)]), np.int32)
    l = cuda(rng.normal(size=(n, k)), np.float32)
    y = ids[:, 0].contiguous()
    lib = umas.load_library()
    ws = [torch.empty(b, dtype=torch.uint8, device="cuda") for b in (lib.umas_top_logits_workspace_bytes(n, d, V, k, 1),
                                                                     lib.umas_cross_entropy_workspace_bytes(n, d, V, 1, 1), lib.umas_distill_workspace_bytes(n, d, V, k, 1, 1))]

    def outputs():
        e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        return [e(n, k, t=torch.int32), e(n, k), e(n)] + [e(32, t=torch.uint8), e(n), torch.empty_like(Hd), torch.empty_like(Wd)] + \
               [e(32, t=torch.uint8), e(n), torch.empty_like(Hd), torch.empty_like(Wd)]

    def step(o):
        umas.umas_top_logits(Hd, Wd, k, ids=o[0], logits=o[1], lse=o[2], workspace=ws[0])
        umas.umas_cross_entropy_fwd_bwd(Hd, Wd, y, stats=o[3], logp=o[4], dH=o[5], dW=o[6], workspace=ws[1])
        umas.umas_distill_fwd_bwd(Hd, Wd, ids, l, stats=o[7], kl=o[8], dH=o[9], dW=o[10], workspace=ws[2])

    o = outputs()
    step(o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(o)
    torch.cuda.synchronize()
    for factor in (1.0, -1.0, 0.5):
        Hd.copy_(cuda(H * factor, np.float32))
        l.copy_(cuda(rng.normal(size=(n, k)), np.float32))
        for x in o:
            x.view(torch.uint8).fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        eager = outputs()
        step(eager)
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(o, eager)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i


def test_on_another_stream_and_the_same_bits_every_time():
    n, d, V, k = 400, 256, 5000, 16
    H, W, Hd, Wd, rng = arrays(21, n, d, V, "bf16")
    ids, l = cuda(np.stack([rng.permutation(V)[:k] for _ in range(n)]), np.int32), cuda(rng.normal(size=(n, k)), np.float32)
    torch.cuda.synchronize()
    want = umas.umas_distill_fwd_bwd(Hd, Wd, ids, l), umas.umas_top_logits(Hd, Wd, k)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            got = umas.umas_distill_fwd_bwd(Hd, Wd, ids, l), umas.umas_top_logits(Hd, Wd, k)
    torch.cuda.synchronize()
    for a, b in zip(want[0] + want[1], got[0] + got[1]):
        assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals():
    n, d, V, k = 10, 64, 300, 4
    H, W, Hd, Wd, rng = arrays(1, n, d, V, "bf16")
    ids, l = torch.zeros(n, k, dtype=torch.int32, device="cuda"), torch.zeros(n, k, device="cuda")
    y = ids[:, 0].contiguous()
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    refused = [(-2, lambda: umas.umas_top_logits(Hd, Wd, 0)), (-2, lambda: umas.umas_top_logits(Hd, Wd, 65)), (-4, lambda: umas.umas_top_logits(Hd, Wd, 4, workspace=ws)),
               (-4, lambda: umas.umas_cross_entropy_fwd_bwd(Hd, Wd, y, workspace=ws)), (-1, lambda: umas.umas_cross_entropy_fwd_bwd(Hd, Wd, y, z_coef=-1.0)),
               (-1, lambda: umas.umas_cross_entropy_fwd_bwd(Hd, Wd, y, z_coef=float("nan"))), (-1, lambda: umas.umas_cross_entropy_fwd_bwd(Hd, Wd, y, norm_rows=3)),
               (-1, lambda: umas.umas_cross_entropy_fwd_bwd(Hd, Wd, y, None, None, None, 2)), (-2, lambda: umas.umas_cross_entropy_fwd_bwd(Hd, Wd, y, None, None, y, 65)),
               (-2, lambda: umas.umas_distill_fwd_bwd(Hd, Wd, ids.repeat(1, 17), l.repeat(1, 17))),
               (-1, lambda: umas.umas_cross_entropy_fwd_bwd(Hd, Wd, y, torch.tensor([n], dtype=torch.int32, device="cuda"))),
               (-2, lambda: umas.umas_top_logits(Hd[:, :60].contiguous(), Wd[:, :60].contiguous(), 4))]
    for code, call in refused:
        with pytest.raises(umas.UmasError) as e:
            call()
        assert e.value.code == code, str(e.value)
    for kind, call in [(ValueError, lambda: umas.umas_top_logits(Hd[:, ::2], Wd, 4)), (ValueError, lambda: umas.umas_cross_entropy_fwd_bwd(Hd, Wd.float(), y)),
                       (TypeError, lambda: umas.umas_cross_entropy_fwd_bwd(Hd, Wd, y.long())), (ValueError, lambda: umas.umas_cross_entropy_fwd_bwd(Hd, Wd, y[:5])),
                       (ValueError, lambda: umas.umas_distill_fwd_bwd(Hd, Wd, ids, l[:, :3])), (TypeError, lambda: umas.umas_distill_fwd_bwd(Hd, Wd, ids, l.double())),
                       (ValueError, lambda: umas.umas_distill_fwd_bwd(Hd, Wd, ids.T.contiguous().T, l)), (TypeError, lambda: umas.umas_cross_entropy_fwd_bwd(Hd, Wd, y, dW=Wd.double())),
                       (ValueError, lambda: umas.umas_cross_entropy_fwd_bwd(Hd, Wd, y, dW=Wd[:5]))]:
        with pytest.raises(kind):
            call()
    assert binding.TARGET_STATS_DTYPE.itemsize == 32
