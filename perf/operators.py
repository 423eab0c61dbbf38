"""Cases of the operators that teach a head from targets: the largest logits of a head (a teacher's side, or the candidates of
a next token), the softmax cross entropy of given tokens with its gradient, and distillation from a teacher's largest logits
with its gradient.

A case is a dict of plain values.  `listed()` names the fixed ones, `draw(rng)` gives another one of the same ranges,
`prepare(case, seed)` makes what a caller has in hand before the call (on the GPU, from the seed alone), `run(state)` is one
pass, `work(case)` the bytes and operations it cannot do without, `exact(case, seed)` the outputs in 64 bits.  With `own` set a
pass calls the framework's operators, else it computes them in their plain form, in elementary operations of 32 bits.

Kinds of case and the range each stands for:
  top      logsumexp and the k largest logits of selected rows, ties to the lowest token (1 to 8192 rows, k up to 64)
  ce       cross entropy with weights, ignored tokens and the penalty on the logsumexp, its gradient to hidden states and head
           (20 to 16384 rows; float32 heads are small ones)
  distill  divergence from a teacher's distribution over its k largest tokens, the gradient as above (20 to 16384 rows, k up to 64)

Hidden states have about unit RMS and lean towards the row's own tokens, as those of a trained model do; heads are N(0, 0.02),
tokens follow a truncated Zipf(1.1) law.
"""
import math

import torch

own = False

HEAD_3B = (2048, 151936)   # d, V of the repository's pipeline configuration
HEAD_7B = (3584, 152064)   # ... and of its coder / second shared model


def listed():
    return [
        # serving: the candidates of the next token of one sequence
        dict(name="top_one_token", kind="top", rows=1, k=20, select=False, d=HEAD_3B[0], V=HEAD_3B[1], dtype="bf16"),
        # serving: two dozen sequences that decode together, the wider head
        dict(name="top_decode_batch", kind="top", rows=24, k=50, select=False, d=HEAD_7B[0], V=HEAD_7B[1], dtype="bf16"),
        # a teacher with another vocabulary and an odd width, the scored rows of a few trajectories
        dict(name="top_odd_head", kind="top", rows=777, k=32, select=True, d=1544, V=50001, dtype="bf16"),
        # a teacher over a part of a rollout: every row, as many places as there are
        dict(name="top_teacher_rollout", kind="top", rows=8192, k=64, select=False, d=HEAD_3B[0], V=HEAD_3B[1], dtype="bf16"),
        # the float32 option: the small configuration that is used to check a set-up
        dict(name="ce_float32", kind="ce", rows=768, select=False, head=True, z=0.0, d=64, V=512, dtype="f32"),
        # supervised steps on one short trajectory, the wider head
        dict(name="ce_one_trajectory", kind="ce", rows=203, select=True, head=True, z=0.0, d=HEAD_7B[0], V=HEAD_7B[1], dtype="bf16"),
        # the head is frozen (adapters in the body are trained), an odd vocabulary
        dict(name="ce_frozen_head", kind="ce", rows=2900, select=True, head=False, z=1e-4, d=1536, V=100279, dtype="bf16"),
        # a supervised step on the scored rows of a batch, the largest case
        dict(name="ce_batch", kind="ce", rows=16384, select=False, head=True, z=1e-4, d=HEAD_3B[0], V=HEAD_3B[1], dtype="bf16"),
        # one answer of a teacher, renormalised over few places
        dict(name="distill_one_turn", kind="distill", rows=60, k=10, tail=False, select=False, head=True, d=HEAD_3B[0], V=HEAD_3B[1], dtype="bf16"),
        # a narrow student with an odd vocabulary; the teacher's logsumexp is given
        dict(name="distill_odd_head", kind="distill", rows=1111, k=32, tail=True, select=True, head=True, d=1096, V=50001, dtype="bf16"),
        # an ordinary step of distillation
        dict(name="distill_step", kind="distill", rows=4096, k=64, tail=True, select=False, head=True, d=HEAD_3B[0], V=HEAD_3B[1], dtype="bf16"),
        # the wider student
        dict(name="distill_wide", kind="distill", rows=7000, k=20, tail=False, select=True, head=True, d=HEAD_7B[0], V=HEAD_7B[1], dtype="bf16"),
    ]


# ------------------------------------------------------------------------------------------------ drawn cases
def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_head(rng):
    """Mostly the two heads of the configurations; else any width the bf16 path takes and an odd vocabulary."""
    x = rng.random()
    if x < 0.35:
        return HEAD_3B
    if x < 0.5:
        return HEAD_7B
    d = 64 * rng.randint(8, 47) if rng.random() < 0.7 else 8 * rng.randint(64, 380)
    return d, _log_int(rng, 20000, 160000) | 1


def draw(rng):
    kind = rng.choice(["top", "ce", "distill"])
    case = dict(kind=kind, select=rng.random() < 0.5)
    if rng.random() < 0.15:    # float32: small heads
        case.update(rows=_log_int(rng, 20, 1000), d=_log_int(rng, 32, 512), V=_log_int(rng, 300, 8192), dtype="f32")
        while case["rows"] * float(case["d"]) * case["V"] > 2.0 ** 30:
            case["rows"] = case["rows"] * 2 // 3
    else:
        d, V = _draw_head(rng)
        rows = _log_int(rng, 1, 8192) if kind == "top" else _log_int(rng, 20, 16384)
        while rows * float(d) * V > 5.0e12:
            rows = rows * 2 // 3
        case.update(rows=rows, d=d, V=V, dtype="bf16")
    if case["rows"] > 2000:
        case["rows"] |= 1                                      # ragged as rollouts are
    if kind == "ce":
        case.update(head=rng.random() < 0.7, z=rng.choice([0.0, 1e-4]))
    else:
        case.update(k=_log_int(rng, 1, 64))
    if kind == "distill":
        case.update(head=rng.random() < 0.7, tail=rng.random() < 0.5)
    return case


# ------------------------------------------------------------------------------------------------ inputs
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _zipf(shape, V, gen):
    """Tokens by the law P(id = r - 1) ~ r^-1.1, from the continuous distribution's inverse."""
    u = torch.rand(shape, device="cuda", generator=gen)
    r = (1.0 - u * (1.0 - (V + 1.0) ** -0.1)) ** -10.0
    return (r.long() - 1).clamp_(0, V - 1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, d, V, dtype = case["rows"], case["d"], case["V"], DTYPES[case["dtype"]]
    randn = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    n = rows + rows // 4 + 1 if case["select"] else rows       # rows of the hidden states, a fifth of them not scored
    y = _zipf((n,), V, gen)
    if case["kind"] == "top":
        # Hidden states and head on a grid (steps of 1/64 and 1/512, finer than bf16 where values are large): every product and
        # sum is exact in 32 bits in any order, so that two correct programs agree on every token, equal logits among them.
        W = torch.round(randn(V, d) * (0.02 * 512)).div_(512).to(dtype)
        H = (torch.round(randn(n, d) * 16).div_(16) + 8 * W[y].float()).to(torch.bfloat16).to(dtype)
    else:
        W = (0.02 * randn(V, d)).to(dtype)
        # a token's logit gains lean * |W_y|^2: about lean * d * 0.0004
        lean = 6.0 + 10.0 * torch.rand(n, 1, device="cuda", generator=gen)
        H = (randn(n, d) + lean * min(1.0, 2048 / d) * W[y].float()).to(dtype)
    s = {"case": case, "H": H, "W": W, "rowsel": None}
    if case["select"]:
        s["rowsel"] = torch.randperm(n, device="cuda", generator=gen)[:rows].sort().values.int()
    if case["kind"] == "top":
        return s
    # weights: most rows 1, one in twenty left out by a weight of 0; one row in fifty has no target
    s["weight"] = (0.5 + torch.rand(n, device="cuda", generator=gen)) * (torch.rand(n, device="cuda", generator=gen) > 0.05)
    none = torch.rand(n, device="cuda", generator=gen) < 0.02
    if case["kind"] == "ce":
        s["ids"] = torch.where(none, -100, y).int()
        return s
    # the teacher's places: the row's token first, then distinct ones, every other one among the frequent tokens
    k = case["k"]
    start = torch.rand(n, 2, device="cuda", generator=gen)
    j = torch.arange(k, device="cuda")
    front = max(V // 16, k)
    a = (start[:, :1] * front).long() + (j // 2) * max(front // k, 1)
    b = (start[:, 1:] * (V - front)).long() + (j // 2) * ((V - front) // k)
    ids = torch.where(j % 2 == 0, a % front, front + b % (V - front))
    ids[:, 0] = torch.where((ids[:, 1:] == y[:, None]).any(1), ids[:, 0], y)
    logits = 12.0 - torch.rand(n, k, device="cuda", generator=gen).mul_(6.0 / math.sqrt(k)).cumsum(1)
    s["teacher_lse"] = None
    if case["tail"]:           # what the teacher gives to other tokens: up to a third
        s["teacher_lse"] = torch.logsumexp(logits, 1) - torch.log1p(-torch.rand(n, device="cuda", generator=gen) / 3)
    # one row in ten has fewer places, one in fifty none; what lies in a place that does not count is no number
    have = torch.where(torch.rand(n, device="cuda", generator=gen) < 0.1, (torch.rand(n, device="cuda", generator=gen) * k).long() + 1, k)
    gone = (j >= have[:, None]) | none[:, None]
    s["ids"] = torch.where(gone, -1, ids).int()
    s["logits"] = torch.where(gone, math.nan, logits)
    return s


# ------------------------------------------------------------------------------------------------ a pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2605_26646_amd as umas
    case = s["case"]
    if case["kind"] == "top":
        ids, logits, lse = umas.umas_top_logits(s["H"], s["W"], case["k"], s["rowsel"])
        return {"ids": ids, "logits": logits, "lse": lse}
    if case["kind"] == "ce":
        stats, logp, dH, dW = umas.umas_cross_entropy_fwd_bwd(s["H"], s["W"], s["ids"], s["rowsel"], s["weight"], z_coef=case["z"], train_head=case["head"])
        out = {"loss": stats.view(torch.float32)[0], "logp": logp, "dH": dH}
    else:
        stats, kl, dH, dW = umas.umas_distill_fwd_bwd(s["H"], s["W"], s["ids"], s["logits"], s["teacher_lse"], s["rowsel"], s["weight"],
                                                      train_head=case["head"])
        out = {"loss": stats.view(torch.float32)[0], "kl": kl, "dH": dH}
    if case["head"]:
        out["dW"] = dW
    return out


def _selected(s):
    return s["H"] if s["rowsel"] is None else s["H"][s["rowsel"].long()]


def _of_rows(s, x):
    return x if s["rowsel"] is None else x[s["rowsel"].long()]


def _scatter(s, x, fill=0):
    if s["rowsel"] is None:
        return x
    out = torch.full((s["H"].shape[0], *x.shape[1:]), fill, dtype=x.dtype, device=x.device)
    out[s["rowsel"].long()] = x
    return out


def _run_plain(s):
    case = s["case"]
    h, W = _selected(s).float(), s["W"].float()
    z = h @ W.T
    m = z.amax(1, keepdim=True)
    lse = m[:, 0] + (z - m).exp_().sum(1).log_()
    if case["kind"] == "top":
        V = case["V"]
        bits = z.add_(0.0).view(torch.int32)                   # whole numbers in the order of the logits, then the lower token first
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * 2 ** 32
        key += torch.arange(V - 1, -1, -1, device="cuda")
        ids = V - 1 - (key.topk(case["k"], dim=1).values & 0xFFFFFFFF)
        return {"ids": _scatter(s, ids.int(), -1), "logits": _scatter(s, z.gather(1, ids)), "lse": _scatter(s, lse)}
    weight, ids, rows = _of_rows(s, s["weight"]), _of_rows(s, s["ids"]).long(), case["rows"]
    if case["kind"] == "ce":
        ids, t = ids[:, None], (ids >= 0).float()[:, None]
    else:
        logits = torch.where(ids >= 0, _of_rows(s, s["logits"]), -math.inf)
        top = logits.amax(1, keepdim=True).clamp_(min=-1e30)
        t = (logits - top).exp()
        if s["teacher_lse"] is None:
            t = t / t.sum(1, keepdim=True).clamp_(min=1e-30)
        else:
            t = t * (top - _of_rows(s, s["teacher_lse"])[:, None]).exp()
            t = torch.where(ids >= 0, t, 0.0)
    at = ids.clamp(min=0)
    zt = z.gather(1, at)
    mass = t.sum(1)
    g = weight * (mass > 0) / rows
    if case["kind"] == "ce":
        row = (zt[:, 0] - lse) * t[:, 0]
        loss = (g * (case["z"] * lse * lse - row)).sum()
        mass = mass + 2 * case["z"] * lse
    else:
        row = torch.where(t > 0, t * (t.clamp(min=1e-38).log() - zt + lse[:, None]), 0.0).sum(1)
        loss = (g * row).sum()
    dz = z.sub_(lse[:, None]).exp_().mul_((g * mass)[:, None])
    dz.scatter_add_(1, at, -g[:, None] * t)
    out = {"loss": loss, "logp" if case["kind"] == "ce" else "kl": _scatter(s, row), "dH": _scatter(s, (dz @ W).to(s["H"].dtype))}
    if case["head"]:
        out["dW"] = (dz.T @ h).to(s["W"].dtype)
    return out


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    rows, d, V = case["rows"], case["d"], case["V"]
    size = 2 if case["dtype"] == "bf16" else 4
    n = rows + rows // 4 + 1 if case["select"] else rows
    head, hidden = V * d * size, rows * d * size
    if case["kind"] == "top":
        return {"bytes": head + hidden + n * (8 * case["k"] + 4), "flops": 2.0 * rows * d * V}
    targets = 4 * n if case["kind"] == "ce" else 8 * n * case["k"]
    grads = n * d * size + (head if case["head"] else 0)
    return {"bytes": head + hidden + targets + 8 * n + grads, "flops": (6.0 if case["head"] else 4.0) * rows * d * V}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """The definition, differentiated by torch, in parts of the rows."""
    s = prepare(case, seed)
    n, V = s["H"].shape[0], case["V"]
    rows = torch.arange(n, device="cuda") if s["rowsel"] is None else s["rowsel"].long()
    W = s["W"].double().requires_grad_(case["kind"] != "top" and case["head"])
    step = max(1, int(3e8 / V))
    lse = torch.zeros(n, dtype=torch.float64, device="cuda")
    if case["kind"] == "top":
        logits = torch.zeros(n, case["k"], dtype=torch.float64, device="cuda")
        for part in rows.split(step):
            z = s["H"][part].double() @ W.T
            lse[part] = torch.logsumexp(z, 1)
            logits[part] = z.topk(case["k"], dim=1).values
        return {"ids": None, "logits": logits, "lse": lse}
    dH, row, loss = torch.zeros(s["H"].shape, dtype=torch.float64, device="cuda"), lse, 0.0
    for part in rows.split(step):
        h = s["H"][part].double().requires_grad_()
        logp_all = torch.log_softmax(h @ W.T, 1)
        w, ids = s["weight"][part].double(), s["ids"][part].long()
        if case["kind"] == "ce":
            has = ids >= 0
            lp = torch.where(has, logp_all.gather(1, ids.clamp(min=0)[:, None])[:, 0], 0.0)
            z0 = (h * W[0]).sum(1) - logp_all[:, 0]            # the logsumexp
            one = -lp + case["z"] * z0 ** 2 * has
            row[part] = lp.detach()
        else:
            teacher = torch.where(ids >= 0, s["logits"][part].double(), -math.inf)
            if s["teacher_lse"] is None:
                log_t = torch.log_softmax(teacher, 1)          # a row without places: no numbers, none of which counts
            else:
                log_t = teacher - s["teacher_lse"][part].double()[:, None]
            t = torch.where(ids >= 0, log_t.exp(), 0.0)
            one = (t * (torch.where(ids >= 0, log_t, 0.0) - logp_all.gather(1, ids.clamp(min=0)))).sum(1)
            row[part] = one.detach()
        total = (w * one).sum() / len(rows)
        total.backward()
        loss += float(total.detach())
        dH[part] = h.grad
    key = "logp" if case["kind"] == "ce" else "kl"
    out = {"loss": torch.tensor(loss, dtype=torch.float64), key: row, "dH": dH}
    if case["head"]:
        out["dW"] = W.grad
    return out
