"""Cases of the operators directly around a head: the norm in front of it (with the residual's addition, its backward pass, an output in
8 bits), the draw of a token from its logits, and the global norm and clipping of the gradients behind it.

A case is a dict of plain values.  `listed()` names the fixed ones, `draw(rng)` gives another one of the same ranges,
`prepare(case, seed)` makes what a caller has in hand before the call (on the GPU, from the seed alone), `run(state)` is one
pass, `work(case)` the bytes and operations it cannot do without, `exact(case, seed)` the outputs in 64 bits.  With `own` set a
pass calls the framework's operators, else it computes them in their plain form, in elementary operations.

Kinds of case and the range each stands for:
  sample    a token for every row of given logits: temperature, top-k, min-p, top-p, one uniform number a row (1 to 1024 rows, 1000 to
            160 000 tokens, bf16 or float32, rows of a padded vocabulary, tokens masked by -infinity or the lowest number)
  tokens    the same from hidden states and a head (1 to 512 rows)
  norm      root-mean-square norm of x + residual (1 to 40 000 rows of 64 to 8192 columns), or with its output in 8 bits
  norm_bwd  its backward pass, with the gradient that reaches the sum by itself and the gain's gradient
  clip      global norm over a list of gradients of several types and sizes, scaled in place or into other arrays (1e4 to 8e8 numbers)
"""
import math

import torch

own = False

HEAD_3B = (2048, 151936)   # d, V of the repository's pipeline configuration
HEAD_7B = (3584, 152064)   # ... and of its coder / second shared model
EPS = 1e-6


def listed():
    return [
        # serving: the next token of one sequence, from float32 logits
        dict(name="sample_one", kind="sample", rows=1, V=HEAD_3B[1], pad=0, dtype="f32", params="one", temperature=0.7, top_k=0, top_p=0.9, min_p=0.0),
        # serving: a batch of sequences that each bring settings of their own, bf16 logits (many of them equal)
        dict(name="sample_batch_settings", kind="sample", rows=256, V=HEAD_7B[1], pad=0, dtype="bf16", params="rows", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0),
        # a rollout at temperature 1 without filters, an odd vocabulary in padded rows
        dict(name="sample_rollout_odd", kind="sample", rows=777, V=50001, pad=47, dtype="f32", params="one", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0),
        # serving: two dozen sequences that decode together, the wider head, a few candidates
        dict(name="tokens_decode_batch", kind="tokens", rows=24, select=False, d=HEAD_7B[0], V=HEAD_7B[1], dtype="bf16", params="one", temperature=0.8, top_k=20, top_p=0.95, min_p=0.0),
        # a rollout's step over many sequences, some of them ended
        dict(name="tokens_rollout", kind="tokens", rows=400, select=True, d=HEAD_3B[0], V=HEAD_3B[1], dtype="bf16", params="one", temperature=1.0, top_k=0, top_p=0.95, min_p=0.02),
        # serving: one token of a few sequences
        dict(name="norm_decode", kind="norm", rows=4, d=HEAD_3B[0], dtype="bf16", residual=True, quantized=False),
        # the hidden states of a whole batch in front of the head
        dict(name="norm_batch", kind="norm", rows=39224, d=HEAD_3B[0], dtype="bf16", residual=True, quantized=False),
        # a part of a rollout whose next product is one of 8 bits, the wider model
        dict(name="norm_quantized", kind="norm", rows=8192, d=HEAD_7B[0], dtype="bf16", residual=True, quantized=True),
        # float32, an odd width, no residual gradient: one trajectory
        dict(name="norm_bwd_odd", kind="norm_bwd", rows=777, d=1545, dtype="f32", through=False),
        # the batch's backward pass
        dict(name="norm_bwd_batch", kind="norm_bwd", rows=39224, d=HEAD_3B[0], dtype="bf16", through=True),
        # a small model's gradients, in place, below the bound: the norm alone
        dict(name="clip_below", kind="clip", blocks=6, d=512, V=4001, dtype="bf16", into=False, over=False),
        # a part of a large model's gradients with its head, over the bound, into the optimizer's array
        dict(name="clip_over", kind="clip", blocks=6, d=2048, V=HEAD_3B[1], dtype="bf16", into=True, over=True),
    ]


# ------------------------------------------------------------------------------------------------ drawn cases
def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_settings(rng):
    if rng.random() < 0.4:
        return dict(params="rows", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    return dict(params="one", temperature=rng.choice([1.0, 1.0, 0.6, round(rng.uniform(0.3, 1.5), 2)]),
                top_k=rng.choice([0, 0, _log_int(rng, 1, 60), _log_int(rng, 60, 1000)]), top_p=rng.choice([1.0, 0.9, round(rng.uniform(0.5, 0.99), 2)]),
                min_p=rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.2), 2)]))


def draw(rng):
    kind = rng.choice(["sample", "tokens", "norm", "norm_bwd", "clip"])
    if kind == "sample":
        V, rows = rng.choice([HEAD_3B[1], HEAD_7B[1], _log_int(rng, 1000, 160000) | 1]), _log_int(rng, 1, 1024)
        while rows * V > 3.8e7:
            rows = rows * 2 // 3
        return dict(kind=kind, rows=rows, V=V, pad=rng.choice([0, 0, rng.randint(1, 255)]), dtype=rng.choice(["bf16", "f32"]), **_draw_settings(rng))
    if kind == "tokens":
        if rng.random() < 0.15:                                # float32: small heads
            rows, d, V, dtype = _log_int(rng, 1, 200), _log_int(rng, 32, 256), _log_int(rng, 300, 4096), "f32"
        else:
            d, V = rng.choice([HEAD_3B, HEAD_7B, (64 * rng.randint(8, 47), _log_int(rng, 20000, 160000) | 1), (8 * rng.randint(64, 380), _log_int(rng, 20000, 160000) | 1)])
            rows, dtype = _log_int(rng, 1, 400), "bf16"
            while rows * float(d) * V > 1.2e11:
                rows = rows * 2 // 3
        return dict(kind=kind, rows=rows, select=rng.random() < 0.5, d=d, V=V, dtype=dtype, **_draw_settings(rng))
    if kind in ("norm", "norm_bwd"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        d = rng.choice([HEAD_3B[0], HEAD_7B[0], 8 * _log_int(rng, 8, 1024)]) if dtype == "bf16" else _log_int(rng, 64, 8192)
        rows = _log_int(rng, 1, 40000)
        while rows * d * (1 if dtype == "bf16" else 2) > 8.0e7:
            rows = rows * 2 // 3
        if kind == "norm":
            return dict(kind=kind, rows=rows, d=d, dtype=dtype, residual=rng.random() < 0.7, quantized=rng.random() < 0.3)
        return dict(kind=kind, rows=rows, d=d, dtype=dtype, through=rng.random() < 0.5)
    d, blocks, V = 8 * _log_int(rng, 4, 256), rng.randint(0, 8), _log_int(rng, 500, 150000)
    dtype = rng.choice(["bf16", "f32"])
    while blocks * 14 * d * d + V * d > (6.0e8 if dtype == "bf16" else 3.0e8):
        blocks, V = blocks // 2, V // 2
    return dict(kind=kind, blocks=blocks, d=d, V=V | 1, dtype=dtype, into=rng.random() < 0.5, over=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _settings(s, case, n, gen):
    """The call's sampling settings: numbers for all rows, or arrays with one for each."""
    u = torch.rand(n, device="cuda", generator=gen)
    s["u"] = u
    if case["params"] == "one":
        s["settings"] = {k: case[k] for k in ("temperature", "top_k", "top_p", "min_p")}
        return
    r = torch.rand(7, n, device="cuda", generator=gen)
    most = math.log(case["V"])
    s["settings"] = {
        "temperature": torch.where(r[0] < 0.1, 0.0, 0.3 + 1.2 * r[1]),                          # one in ten is greedy
        "top_k": torch.where(r[2] < 0.4, 0.0, (r[3] * most).exp()).int(),
        "top_p": torch.where(r[4] < 0.3, 1.0, 0.5 + 0.49 * r[4]),
        "min_p": torch.where(r[5] < 0.5, 0.0, 0.2 * r[6]),
    }


def _clip_shapes(case):
    """A head, and for every block its products and the two gains in front of them (float32, as gains' gradients are)."""
    d, V = case["d"], case["V"]
    shapes = [(V * d, case["dtype"]), (d, "f32")]
    for b in range(case["blocks"]):
        shapes += [(d * (d + d // 4), case["dtype"]), (d * d, case["dtype"]), (8 * d * d, case["dtype"]), (4 * d * d - b, case["dtype"]), (d, "f32"), (d + 1, "f32")]
    return shapes


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    rand = lambda *shape: torch.rand(*shape, device="cuda", generator=gen)  # noqa: E731
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    s = {"case": case}
    if kind == "sample":
        rows, V = case["rows"], case["V"]
        # background of the whole vocabulary, and some dozen tokens that the context speaks for, more or less sure of them
        z = randn(rows, V + case["pad"]).mul_(2.0)
        at = (rand(rows, 48) * V).long()
        z.scatter_reduce_(1, at, 10.0 + 4.0 * rand(rows, 1) + 2.0 * randn(rows, 48), "amax")   # some places come twice
        banned = rand(rows, 64).mul_(V).long()                  # a grammar's mask in one row of four
        z.scatter_(1, banned, torch.where(rand(rows, 1) < 0.25, -math.inf if seed % 2 else torch.finfo(dtype).min, z.gather(1, banned)))
        s["logits"] = z.to(dtype)[:, :V]
        _settings(s, case, rows, gen)
        return s
    if kind == "tokens":
        rows, d, V = case["rows"], case["d"], case["V"]
        n = rows + rows // 4 + 1 if case["select"] else rows
        # Hidden states and head on a grid (steps of 1/64 and 1/512, finer than bf16 where values are large): every product and sum is exact in
        # 32 bits in any order, so that two correct programs have the same logits, equal ones among them, and draw the same tokens.
        W = torch.round(randn(V, d).mul_(0.02 * 512)).div_(512).to(torch.bfloat16).to(dtype)
        y = (rand(n).square() * V).long().clamp_(max=V - 1)
        lean = 8.0 * torch.ceil(rand(n, 1) * max(1, min(3, round(3 * 2048 / d))))
        s["H"] = (torch.round(randn(n, d) * 16).div_(16) + lean * W[y].float()).to(torch.bfloat16).to(dtype)
        s["W"], s["rowsel"] = W, None
        if case["select"]:
            s["rowsel"] = torch.randperm(n, device="cuda", generator=gen)[:rows].sort().values.int()
        _settings(s, case, n, gen)
        return s
    if kind in ("norm", "norm_bwd"):
        n, d = case["rows"], case["d"]
        s["gain"] = (1.0 + 0.3 * randn(d)).to(dtype)
        # a residual stream: rows of different size, a few columns far above the others
        stream = randn(n, d) * (0.5 + 4.0 * rand(n, 1)) * torch.where(rand(d) < 0.005, 12.0, 1.0)
        if kind == "norm":
            s["x"] = randn(n, d).to(dtype) if case["residual"] else stream.to(dtype)
            s["residual"] = stream.to(dtype) if case["residual"] else None
            return s
        s["hidden"] = stream.to(dtype)
        s["inv_rms"] = torch.rsqrt(s["hidden"].float().square().mean(1) + EPS)
        s["dy"] = (0.01 * randn(n, d) * (rand(n, 1) > 0.2)).to(dtype)             # one row in five has no gradient
        s["dhidden"] = (0.01 * randn(n, d)).to(dtype) if case["through"] else None
        return s
    shapes = _clip_shapes(case)
    s["grads"] = [(1e-3 * (0.2 + 2.0 * rand(1)) * randn(n)).to(DTYPES[t]) for n, t in shapes]
    norm = math.sqrt(sum(float(g.double().square().sum()) if g.numel() < 1e6 else float(g.float().square().sum()) for g in s["grads"]))
    s["max_norm"] = norm / 3.0 if case["over"] else norm * 3.0
    s["out"] = None
    # what is over the bound in place would be below it in the next pass: it goes to arrays of its own, one behind the other
    if case["into"] or case["over"]:
        s["flat"] = {t: torch.empty(sum(n for n, u in shapes if u == t), dtype=DTYPES[t], device="cuda") for t in {u for _, u in shapes}}
        at, s["out"] = dict.fromkeys(s["flat"], 0), []
        for n, t in shapes:
            s["out"].append(s["flat"][t][at[t]:at[t] + n])
            at[t] += n
    return s


# ------------------------------------------------------------------------------------------------ a pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _clip_result(s, norm):
    return {"norm": norm, "out": dict(s["flat"]) if s["out"] else list(s["grads"])}


def _run_own(s):
    import paper_2605_26646_amd as umas
    case, kind = s["case"], s["case"]["kind"]
    if kind == "sample":
        ids, logp, logq = umas.umas_sample_logits(s["logits"], s["u"], **s["settings"])
        return {"ids": ids, "logp": logp, "logq": logq}
    if kind == "tokens":
        ids, logp, logq = umas.umas_sample_tokens(s["H"], s["W"], s["u"], s["rowsel"], **s["settings"])
        return {"ids": ids, "logp": logp, "logq": logq}
    if kind == "norm" and case["quantized"]:
        q, scale, hidden, inv_rms = umas.umas_rms_norm_quantized(s["x"], s["gain"], s["residual"], eps=EPS)
        return {"q": q, "scale": scale, "hidden": hidden, "inv_rms": inv_rms}
    if kind == "norm":
        y, hidden, inv_rms = umas.umas_rms_norm(s["x"], s["gain"], s["residual"], eps=EPS)
        return {"y": y, "hidden": hidden, "inv_rms": inv_rms}
    if kind == "norm_bwd":
        dx, dgain = umas.umas_rms_norm_bwd(s["dy"], s["hidden"], s["gain"], s["inv_rms"], s["dhidden"])
        return {"dx": dx, "dgain": dgain}
    stats, _ = umas.umas_clip_gradients(s["grads"], s["max_norm"], out=s["out"])
    return _clip_result(s, stats.view(torch.float32)[0])


def _of_rows(x, rowsel):
    return x if rowsel is None or not isinstance(x, torch.Tensor) else x[rowsel.long()]


def _scatter(x, s, fill):
    if s.get("rowsel") is None:
        return x
    out = torch.full((s["H"].shape[0],), fill, dtype=x.dtype, device=x.device)
    out[s["rowsel"].long()] = x
    return out


def _column(x, dtype):
    """A setting as one number a row, in a column."""
    return x.to(dtype)[:, None] if isinstance(x, torch.Tensor) else x


def _run_plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind in ("sample", "tokens"):
        sel = s.get("rowsel")
        z = s["logits"].float() if kind == "sample" else _of_rows(s["H"], sel).float() @ s["W"].float().T
        u = _of_rows(s["u"], sel).double()[:, None]
        t, k, p, m = (_of_rows(s["settings"][name], sel) for name in ("temperature", "top_k", "top_p", "min_p"))
        t, k, p, m = _column(t, torch.float64), _column(k, torch.int64), _column(p, torch.float64), _column(m, torch.float64)
        n, V = z.shape
        top = z.amax(1, keepdim=True).double()
        # differences of 0 are told apart from the others, so that a temperature of 0 leaves the largest logits alone
        tt = t if isinstance(t, torch.Tensor) else torch.full((n, 1), t, dtype=torch.float64, device=z.device)
        weight = lambda x: torch.where(x == top, 1.0, torch.where(tt > 0, ((x - top) / tt.clamp(min=1e-30)).exp(), 0.0))  # noqa: E731
        falling, order = z.sort(dim=1, descending=True, stable=True)
        w = weight(falling.double())
        rank = torch.arange(V, device=z.device)
        kk = k if isinstance(k, torch.Tensor) else torch.full((n, 1), k, device=z.device)
        keep = ((kk <= 0) | (rank < kk)) & (w >= m) & ((tt > 0) | (rank < 1)) & (w > 0)
        w = torch.where(keep, w, 0.0)
        ahead = w.cumsum(1)
        mass = ahead[:, -1:].clone()
        pp = p if isinstance(p, torch.Tensor) else torch.full((n, 1), p, dtype=torch.float64, device=z.device)
        keep &= (pp >= 1) | (ahead - w < pp * mass)
        w = torch.where(keep, w, 0.0)
        w = torch.zeros_like(w).scatter_(1, order, w)          # in the order of the tokens again
        run_ = w.cumsum(1)
        mass = run_[:, -1:].clone()
        ids = (run_ <= u * mass).sum(1, keepdim=True)
        last = V - 1 - w.flip(1).ne(0).int().argmax(1, keepdim=True)
        ids = torch.minimum(ids, last)
        logq = (w.gather(1, ids) / mass).log()[:, 0]
        zi = z.gather(1, ids).double()
        logp = (zi - top - (z.double() - top).exp_().sum(1, keepdim=True).log())[:, 0]
        return {"ids": _scatter(ids[:, 0].int(), s, -1), "logp": _scatter(logp.float(), s, 0), "logq": _scatter(logq.float(), s, 0)}
    if kind == "norm":
        dtype = s["x"].dtype
        hidden = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(dtype)
        h = hidden.float()
        inv_rms = torch.rsqrt(h.square().mean(1) + EPS)
        y = h * inv_rms[:, None] * s["gain"].float()
        if not case["quantized"]:
            return {"y": y.to(dtype), "hidden": hidden, "inv_rms": inv_rms}
        scale = y.abs().amax(1) / 448.0
        scale = torch.where(scale > 0, scale, 1.0)
        return {"q": (y / scale[:, None]).to(torch.float8_e4m3fn), "scale": scale, "hidden": hidden, "inv_rms": inv_rms}
    if kind == "norm_bwd":
        dtype, d = s["dy"].dtype, case["d"]
        dy, h, i = s["dy"].float(), s["hidden"].float(), s["inv_rms"][:, None]
        a = dy * s["gain"].float()
        dx = i * (a - h * ((a * h).sum(1, keepdim=True) * i * i / d))
        if s["dhidden"] is not None:
            dx = dx + s["dhidden"].float()
        return {"dx": dx.to(dtype), "dgain": (dy * h * i).sum(0)}
    total = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum()
    norm = total.sqrt()
    scale = (s["max_norm"] / norm).clamp(max=1.0).float()
    for g, o in zip(s["grads"], s["out"] or s["grads"]):
        o.copy_(g.float() * scale)
    return _clip_result(s, norm.float())


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind, size = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind == "sample":                                       # a difference, an exponential and a sum a logit
        return {"bytes": case["rows"] * (case["V"] * size + 16), "flops": 4.0 * case["rows"] * case["V"]}
    if kind == "tokens":
        rows, d, V = case["rows"], case["d"], case["V"]
        return {"bytes": V * d * size + rows * (d * size + 16), "flops": 2.0 * rows * d * V}
    n = case.get("rows", 0) * case.get("d", 0)
    if kind == "norm":
        return {"bytes": n * size * (3 if case["residual"] else 1) + n * (1 if case["quantized"] else size) + 8 * case["rows"], "flops": 6.0 * n}
    if kind == "norm_bwd":
        return {"bytes": n * size * (4 if case["through"] else 3) + 4 * case["rows"] + 4 * case["d"], "flops": 10.0 * n}
    read = sum(m * (2 if t == "bf16" else 4) for m, t in _clip_shapes(case))
    return {"bytes": read * (1 + (case["into"] or case["over"])), "flops": 3.0 * sum(m for m, _ in _clip_shapes(case))}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_draw(z, u, t, k, p, m):
    """One row by its definition: (log-prob of the token under the softmax, under what it was drawn from)."""
    z = z.double()
    logp = torch.log_softmax(z, 0)
    rank = torch.sort(z, descending=True, stable=True).indices
    if t <= 0:
        return logp[rank[0]], 0.0
    if k > 0:
        rank = rank[:k]
    q = torch.softmax(z[rank] / t, 0)
    q = q[q >= m * q[0]]
    q = q / q.sum()
    if p < 1:
        q = q[:1 + int((q.cumsum(0)[:-1] < p).sum())]
    kept, at = rank[:len(q)].sort()
    q = (q / q.sum())[at]
    j = min(int((q.cumsum(0) <= u).sum()), len(q) - 1)
    return logp[kept[j]], q[j].log()


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("sample", "tokens"):
        n = case["rows"] if kind == "sample" else s["H"].shape[0]
        rows = range(n) if s.get("rowsel") is None else s["rowsel"].tolist()
        logp, logq = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
        one = {k: v.tolist() if isinstance(v, torch.Tensor) else [v] * n for k, v in s["settings"].items()}
        u, W = s["u"].tolist(), s["W"].double() if kind == "tokens" else None
        for i in rows:
            z = s["logits"][i] if kind == "sample" else W @ s["H"][i].double()
            logp[i], logq[i] = _exact_draw(z, u[i], one["temperature"][i], one["top_k"][i], one["top_p"][i], one["min_p"][i])
        return {"ids": None, "logp": logp, "logq": logq}
    if kind == "norm":
        x, g = s["x"].double(), s["gain"].double()
        total = x if s["residual"] is None else x + s["residual"].double()
        h = total.to(s["x"].dtype).double()                    # the norm is of the sum as it is stored
        i = (h.pow(2).sum(1) / case["d"] + EPS).pow(-0.5)
        y = h * (i[:, None] * g)
        if not case["quantized"]:
            return {"y": y, "hidden": total, "inv_rms": i}
        scale = y.abs().max(1).values / 448
        scale[scale == 0] = 1.0
        return {"q": y / scale[:, None], "scale": scale, "hidden": total, "inv_rms": i}
    if kind == "norm_bwd":
        # the derivative of y = h i g by h, and by g: d i / d h = - i^3 h / d
        dy, h, g, i = s["dy"].double(), s["hidden"].double(), s["gain"].double(), s["inv_rms"].double()
        dot = (dy * g * h).sum(1)
        dx = dy * g * i[:, None] - h * (dot * i ** 3 / case["d"])[:, None]
        return {"dx": dx if s["dhidden"] is None else dx + s["dhidden"].double(), "dgain": (dy * h).T @ i}
    squares = sum(float(g.double().pow(2).sum()) for g in s["grads"])
    scale = min(1.0, s["max_norm"] / math.sqrt(squares))
    out = [g.double() * scale for g in s["grads"]]
    if s["out"]:
        types = [t for _, t in _clip_shapes(case)]
        out = {t: torch.cat([o for o, u in zip(out, types) if u == t]) for t in s["flat"]}
    return {"norm": torch.tensor(math.sqrt(squares), dtype=torch.float64), "out": out}
