"""Largest logits, cross entropy and distillation on inputs that show what a kernel assumes: large logits gathered in few tokens, masks of a type's lowest value,
infinities in rows that are taught, rows of weight 0, teachers that give next to nothing to their places.  Inputs and tolerances as in test_gpu_targets."""
import numpy as np
import pytest
import torch

import paper_2605_26646_amd as umas
from oracle import umas_oracle as orc
from tests.test_gpu_targets import DT, arrays, check_taught, cuda

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ largest logits
def largest64(H, W, k):
    """Tokens and logits in float64, ties to the lowest token; logits are multiples of 1/256."""
    ids, top, V = [], [], len(W)
    for h in H.split(500):
        z = h.double() @ W.double().T
        key = (z * 256).round().long() * 2 ** 20 + torch.arange(V - 1, -1, -1, device="cuda")
        ids.append(V - 1 - (key.topk(k, dim=1).values & (2 ** 20 - 1)))
        top.append(z.gather(1, ids[-1]))
    return torch.cat(ids), torch.cat(top)


@pytest.mark.parametrize("kind", ["raised", "falling"])
@pytest.mark.parametrize("n,V,k", [(1300, 151936, 8), (2100, 32001, 2), (2100, 32001, 20), (2100, 50001, 20), (4200, 32001, 8), (4200, 50001, 20), (4200, 50001, 2)])
def test_large_logits_that_share_a_few_tiles(n, V, k, kind):
    """Frequent tokens first, as in a trained head: the k largest lie in one tile or two, and single tokens behind them come close.  Whatever is not written
    on the way holds a large number here, which must not be taken for a logit."""
    g = torch.Generator(device="cuda").manual_seed(n + V + k)
    d = 64
    H = torch.randint(-4, 5, (n, d), device="cuda", generator=g, dtype=torch.float32).div_(4)
    W = torch.randint(-8, 9, (V, d), device="cuda", generator=g, dtype=torch.float32).div_(64)
    v = torch.arange(V, device="cuda")
    H[:, 0] = 1
    W[:, 0] = (v < 256) * 8.0 if kind == "raised" else torch.round(-(1.0 + v).log() * 16).div_(16)
    H, W = H.bfloat16(), W.bfloat16()
    want, top = largest64(H, W, k)
    lib = umas.load_library()
    for which in ("", "_min"):
        bytes_ = getattr(lib, "umas_top_logits_workspace_bytes" + which)(n, d, V, k, 1)
        got = umas.umas_top_logits(H, W, k, workspace=torch.full((bytes_,), 0x7F, dtype=torch.uint8, device="cuda"))
        assert torch.equal(got[0].long(), want) and torch.equal(got[1].double(), top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d", [(3, 64), (40, 64), (100, 64), (300, 64)])
@pytest.mark.parametrize("V,k", [(700, 20), (1025, 12), (1025, 64), (3001, 64)])
def test_tokens_masked_by_the_lowest_number(n, d, V, k, dtype):
    """A mask of the type's lowest value in a column of its own: these logits are numbers, which come behind all others, in rising order of tokens.  In one row nothing
    but masked tokens is left."""
    H, W, Hd, Wd, rng = arrays(n + V + k, n, d, V, dtype, grid=True)
    lowest = torch.finfo(torch.bfloat16).min
    open_ = np.sort(rng.permutation(V)[:10])
    masked = np.ones(V, bool)
    masked[open_] = False
    W[masked] = 0
    W[:, :2] = 0
    W[masked, 0], W[:, 1] = lowest, lowest
    H[:, 0], H[:, 1] = 1, 0
    empty = n // 2
    H[empty] = 0
    H[empty, 1] = 1
    ids, top, lse = (x.cpu().numpy() for x in umas.umas_top_logits(cuda(H, np.float32).to(DT[dtype]), cuda(W, np.float32).to(DT[dtype]), k))
    z = H @ W.T
    for i in range(n):
        want = np.lexsort((np.arange(V), -z[i]))[:k]
        assert (ids[i] == want).all() and (top[i] == z[i][want].astype(np.float32)).all()
        m = z[i].max()
        want_lse = m + np.log(np.exp(z[i] - m).sum())
        assert abs(lse[i] - want_lse) <= 1e-5 * (1 + abs(want_lse))


@pytest.mark.parametrize("n", [3, 40, 100, 300])
@pytest.mark.parametrize("V", [256, 300, 1025])
def test_a_row_without_any_logit_has_no_mass(n, V):
    """Every logit is -infinity: nothing is listed, and the sum of exponentials is 0."""
    d = 64
    H, W = torch.zeros(n, d, device="cuda"), torch.zeros(V, d, device="cuda")
    H[:, 0], W[:, 0] = 1, -float("inf")
    ids, top, lse = umas.umas_top_logits(H.bfloat16(), W.bfloat16(), 5)
    assert (ids == -1).all() and (top == -float("inf")).all() and (lse == -float("inf")).all()


# ------------------------------------------------------------------------------------------------ targets
def teach(kind, Hd, Wd, ids, weight, n_roles=0, role=None):
    w = None if weight is None else cuda(weight, np.float32)
    r = None if role is None else cuda(role, np.int32)
    if kind == "ce":
        return umas.umas_cross_entropy_fwd_bwd(Hd, Wd, cuda(ids, np.int32), None, w, r, n_roles)
    return umas.umas_distill_fwd_bwd(Hd, Wd, cuda(ids[:, None], np.int32), torch.zeros(len(ids), 1, device="cuda"), None, None, w, r, n_roles)


@pytest.mark.parametrize("kind", ["ce", "distill"])
@pytest.mark.parametrize("n,dtype", [(40, "bf16"), (200, "bf16"), (300, "bf16"), (40, "f32"), (300, "f32")])
def test_an_overflow_in_a_taught_row_is_seen(n, dtype, kind):
    """The row's logits are all +infinity: its loss is no number however many rows there are, and nothing takes it for a row that is ignored."""
    H, W, Hd, Wd, rng = arrays(n, n, 64, 700, dtype)
    ids = rng.integers(0, 700, n)
    Wd[:, 0] = 1.0
    Hd[n // 3, 0] = float("inf")
    stats, row, dH, dW = teach(kind, Hd, Wd, ids, None)
    s = umas.read_target_stats(stats)
    assert not np.isfinite(s["loss"][0]) and s["n_ignored"][0] == 0
    bad = ~torch.isfinite(row)
    assert bad[n // 3] and int(bad.sum()) == 1
    assert not torch.isfinite(dH[n // 3].float()).any()


@pytest.mark.parametrize("n", [40, 300])
def test_a_targets_logit_that_overflows_is_seen(n):
    H, W, Hd, Wd, rng = arrays(n + 1, n, 64, 700, "bf16")
    ids = rng.integers(1, 700, n)
    bad, y = n // 3, 0
    ids[bad] = y
    Hd[:, 0], Wd[:, 0] = 0.0, 0.0
    Hd[bad, 0], Wd[y, 0] = 2.0 ** 100, 2.0 ** 30
    stats, logp, dH, dW = teach("ce", Hd, Wd, ids, None)
    assert not np.isfinite(umas.read_target_stats(stats)["loss"][0])
    no = ~torch.isfinite(logp)
    assert no[bad] and int(no.sum()) == 1


@pytest.mark.parametrize("kind", ["ce", "distill"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [40, 200, 600])
def test_statistics_next_to_rows_of_weight_0_that_hold_anything(n, dtype, kind):
    """Their entropies and logsumexps are no numbers and are left out; those of a row of weight 0 that are numbers count.  (Tolerances as in check_taught: 2^-24 of the
    logits and of their squares.)"""
    V = 700
    H, W, Hd, Wd, rng = arrays(n + 2, n, 64, V, dtype)
    ids, role = rng.integers(0, V, n), rng.integers(0, 2, n)
    weight = np.ones(n, np.float32)
    bad = np.array([3, n // 2, n - 2])
    weight[bad], weight[7] = 0, 0
    role[bad[0]] = 0
    role[bad[1]] = 1
    for i, x in zip(bad, (np.nan, np.inf, -np.inf)):
        Hd[i] = x
    clean = H.copy()
    clean[bad] = 0
    r = orc.cross_entropy(clean, W, ids, None, weight)
    s = umas.read_target_stats(teach(kind, Hd, Wd, ids, weight, 2, role)[0])
    good = np.ones(n, bool)
    good[bad] = False
    zl = np.abs(H @ W.T).max() + np.abs(r["lse"]).max()
    for k in range(3):
        q = good if k == 0 else good & (role == k - 1)
        for name in ("entropy", "lse"):
            want = r[name][q].mean()
            assert abs(s[name + "_mean"][k] - want) <= 1e-5 * (1 + abs(want)) + (16 * 2.0 ** -24 * zl * (1 + zl) if name == "entropy" else 0)
        assert s["n_scored"][k] == (n if k == 0 else (role == k - 1).sum()) and s["n_ignored"][k] == 0


@pytest.mark.parametrize("dtype,dW_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("n", [30, 200, 300])
@pytest.mark.parametrize("gap", [20.0, 28.0, 40.0])
def test_a_teacher_that_gives_next_to_nothing_to_its_places(n, dtype, dW_dtype, gap):
    """Masses of e^-20 and less: dz = g (T p - t) still sums to 0 over the vocabulary."""
    d, V, k = 64, 300, 5
    H, W, Hd, Wd, rng = arrays(int(n + gap), n, d, V, dtype, scale=2.0)
    ids = np.stack([rng.permutation(V)[:k] for _ in range(n)])
    l = rng.normal(size=(n, k)).astype(np.float32)
    lse = (l.max(1) + gap).astype(np.float32)
    masses = orc.teacher_masses(ids, l, lse, V)
    r = orc.distill(H, W, ids, l, lse)
    kw = {} if dW_dtype == dtype else dict(dW=torch.full((V, d), float("nan"), device="cuda"))
    got = umas.umas_distill_fwd_bwd(Hd, Wd, cuda(ids, np.int32), cuda(l, np.float32), cuda(lse, np.float32), **kw)
    check_taught(r, H, W, ids, masses, got, dtype, dW_dtype, np.zeros(n), 0, n, 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [30, 300])
def test_a_penalty_that_cancels_the_dense_part(n, dtype):
    """1 + 2 c lse is 0, or as near as float32 comes: the one-hot part stands by itself.  Norm-wise bars: what is left of the dense part is rounding."""
    V = 300
    H, W, _, _, rng = arrays(n + 3, 1, 64, V, dtype)
    H, W = np.repeat(H, n, 0), W.copy()
    H[:, 0], W[:, 0] = 1.0, -12.0
    ids = rng.integers(0, V, n)
    z = H[0] @ W.T
    lse = z.max() + np.log(np.exp(z - z.max()).sum())
    assert lse < -2
    c = float(np.float32(-0.5 / lse))
    r = orc.cross_entropy(H, W, ids, z_coef=c)
    stats, logp, dH, dW = umas.umas_cross_entropy_fwd_bwd(cuda(H, np.float32).to(DT[dtype]), cuda(W, np.float32).to(DT[dtype]), cuda(ids, np.int32), z_coef=c)
    assert abs(umas.read_target_stats(stats)["loss"][0] - r["loss"]) <= 1e-5 * (1 + abs(r["loss"]))
    for x, o in ((dH, r["dH"]), (dW, r["dW"])):
        x = x.double().cpu().numpy()
        assert np.isfinite(x).all() and np.linalg.norm(x - o) <= (1e-2 if dtype == "bf16" else 1e-5) * np.linalg.norm(o)


@pytest.mark.parametrize("n,dW_dtype", [(20, "bf16"), (64, "bf16"), (120, "bf16"), (200, "bf16"), (200, "f32")])
def test_roundings_of_a_head_taught_by_few_rows(n, dW_dtype):
    """Every target is a token of its own, so that a row of dW is one entry times one hidden state: up to 256 rows it carries the rounding of the entry and, in bf16, that of the result.  Independent
    roundings add by their squares; one is what the exact dW is off by when it is rounded.  A tenth more is let pass."""
    d, V, k = 256, 20001, 64
    H, W, Hd, Wd, rng = arrays(n, n, d, V, "bf16")
    ids = rng.permutation(V)[:n * k].reshape(n, k)
    l = rng.normal(size=(n, k)).astype(np.float32) * 0.3          # no target much larger than the others
    r = orc.distill(H, W, ids, l)
    kw = {} if dW_dtype == "bf16" else dict(dW=torch.empty(V, d, device="cuda"))
    _, _, dH, dW = umas.umas_distill_fwd_bwd(Hd, Wd, cuda(ids, np.int32), cuda(l, np.float32), **kw)
    off = lambda x, o: np.linalg.norm(x.double().cpu().numpy() - o) / np.linalg.norm(o)  # noqa: E731
    one = lambda o: off(torch.from_numpy(o).bfloat16(), o)  # noqa: E731
    assert off(dW, r["dW"]) <= 1.1 * one(r["dW"]) * (2 ** 0.5 if dW_dtype == "bf16" else 1)
    assert off(dH, r["dH"]) <= 1.1 * one(r["dH"]) * 2 ** 0.5


@pytest.mark.parametrize("kind", ["ce", "distill"])
@pytest.mark.parametrize("n,dtype", [(3, "bf16"), (60, "bf16"), (100, "bf16"), (200, "bf16"), (300, "bf16"), (100, "f32")])
def test_targets_beside_tokens_masked_by_the_lowest_number(n, dtype, kind):
    """Tokens that a column of its own masks have no probability and no gradient; the others are what they are without them.  Norm-wise bars as everywhere."""
    V, d = 1025, 64
    H, W, _, _, rng = arrays(n + 4, n, d, V, dtype)
    masked = rng.random(V) < 0.6
    masked[[0, V - 1]] = False, True
    open_ = np.flatnonzero(~masked)
    W[masked], W[:, 0] = 0, 0
    H[:, 0] = 1
    ids = rng.choice(open_, n)
    r = orc.cross_entropy(H, W[open_], np.searchsorted(open_, ids))
    W[masked, 0] = torch.finfo(torch.bfloat16).min
    stats, row, dH, dW = teach(kind, cuda(H, np.float32).to(DT[dtype]), cuda(W, np.float32).to(DT[dtype]), ids, None)
    s = umas.read_target_stats(stats)
    assert abs(s["loss"][0] - r["loss"]) <= 1e-5 * (1 + r["loss"]) and abs(s["entropy_mean"][0] - r["entropy"].mean()) <= 1e-4 * (1 + r["entropy"].mean())
    assert not dW[torch.from_numpy(masked).cuda()].any()
    tol = 1e-2 if dtype == "bf16" else 1e-5
    for x, o in ((dH.double().cpu().numpy(), r["dH"]), (dW.double().cpu().numpy()[open_], r["dW"])):
        assert np.isfinite(x).all() and np.linalg.norm(x - o) <= tol * np.linalg.norm(o)
