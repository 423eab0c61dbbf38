"""One role's model taught by another's, then asked for tokens.

Two roles share a workflow: a planner, whose model is the larger one, and a solver.  The rollout's tokens are routed to the two models; for the solver's
tokens the planner's head leaves its largest logits (umas_top_logits).  The solver's projection and head are warmed up on the tokens the planner
would have said (umas_cross_entropy_fwd_bwd), then follow the planner's distribution (umas_distill_fwd_bwd), in micro-batches of whole trajectories
whose gradients add up.  At the end the solver answers one token at a time: its own largest logits, drawn from with their probabilities under the whole
vocabulary.  Everything is synthetic: contexts are random vectors, the models are a projection and a head.

    python examples/teach_role.py [--steps 60] [--rows-per-turn 48] [--vocabulary 4000] [--top 32]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_26646_amd as umas

PLANNER, SOLVER = 0, 1


def rollout(n_traj, rows_per_turn):
    """Every trajectory: the planner speaks, then the solver; each turn opens with eight tokens that are not the model's own."""
    n_turns = 2 * n_traj
    mask = torch.ones(n_turns, rows_per_turn, dtype=torch.uint8, device="cuda")
    mask[:, :8] = 0
    traj_turn_off = np.arange(n_traj + 1, dtype=np.int32) * 2
    streams = umas.umas_assign_token_rewards(
        n_roles=2, n_models=2, role_to_model=np.array([0, 1], np.int32), traj_turn_off=traj_turn_off,
        turn_role=np.tile(np.array([PLANNER, SOLVER], np.int32), n_traj),
        turn_tok_off=np.arange(n_turns + 1, dtype=np.int64) * rows_per_turn, tok_mask_global=mask.reshape(-1),
        traj_reward=np.zeros(n_traj, np.float32), place_mode=umas.PLACE_LAST)
    return streams, traj_turn_off


def projected(x, A, W):
    return (x @ A).bfloat16(), W.bfloat16()


def train(x, params, opt, parts, n_rows, teach):
    """One step over all parts: dW adds up in float32, dH rows of the parts go to the projection.  Returns the loss of the step."""
    A, W = params
    H, Wb = projected(x, A, W)
    dW = torch.empty(W.shape, dtype=torch.float32, device="cuda")
    A.grad, loss = torch.zeros_like(A), 0.0
    for i, rows in enumerate(parts):
        stats, _, dH, _ = teach(H, Wb, rows, accumulate_dW=i > 0, norm_rows=n_rows, dW=dW)
        A.grad += x.t() @ dH.float()                 # rows of other parts are zeros
        loss += float(umas.read_target_stats(stats)["loss"][0])
    W.grad = dW
    opt.step()
    return loss


def answer(x, params, k, gen):
    """The next token after one context, one of the k largest logits drawn in proportion to their probabilities, and its probability."""
    H, Wb = projected(x, *params)
    ids, logits, lse = umas.umas_top_logits(H, Wb, k)
    p = torch.exp(logits[0] - lse[0])                # under the whole vocabulary
    j = torch.multinomial(p, 1, generator=gen)[0]
    return int(ids[0, j]), float(p[j])


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--rows-per-turn", type=int, default=48)
    ap.add_argument("--vocabulary", type=int, default=4000)
    ap.add_argument("--top", type=int, default=32)
    args = ap.parse_args(argv)
    n_traj, V, k, context = 16, args.vocabulary, args.top, 96
    gen = torch.Generator(device="cuda").manual_seed(1)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)

    streams, traj_turn_off = rollout(n_traj, args.rows_per_turn)
    off, sel = streams.model_tok_off, streams.model_rowsel_off
    n = int(off[SOLVER + 1] - off[SOLVER])
    rows = streams.rowsel[int(sel[SOLVER]):int(sel[SOLVER + 1])].contiguous()
    mb, mb_off = umas.umas_ready_batch(streams, traj_turn_off, 2)
    cut = [int(c) for c in mb_off[SOLVER]]
    parts = [mb[a:b].contiguous() for a, b in zip(cut, cut[1:])]

    # what the planner's model says where the solver speaks
    x = randn(n, context)
    H_t, W_t = projected(x, randn(context, 256) / context ** 0.5, randn(V, 256) * 0.35)
    top_ids, top_logits, lse_t = umas.umas_top_logits(H_t, W_t, k, rows)

    params = [randn(context, 128) / context ** 0.5, 0.05 * randn(V, 128)]
    opt = torch.optim.Adam(params, lr=1e-2)
    said = top_ids[:, 0].contiguous()                # -1 on rows that are not the model's own
    by_tokens = lambda H, W, r, **kw: umas.umas_cross_entropy_fwd_bwd(H, W, said, r, z_coef=1e-4, **kw)
    by_teacher = lambda H, W, r, **kw: umas.umas_distill_fwd_bwd(H, W, top_ids, top_logits, lse_t, r, **kw)

    def divergence():
        H, Wb = projected(x, *params)
        stats, kl, _, _ = by_teacher(H, Wb, rows)
        ids, _, _ = umas.umas_top_logits(H, Wb, 1, rows)
        return float(umas.read_target_stats(stats)["loss"][0]), float((ids[rows.long(), 0] == said[rows.long()]).float().mean())

    first = divergence()
    warm = [train(x, params, opt, parts, len(rows), by_tokens) for _ in range(args.steps // 4)]
    then = [train(x, params, opt, parts, len(rows), by_teacher) for _ in range(args.steps - len(warm))]
    last = divergence()
    token, p = answer(x[int(rows[0]):int(rows[0]) + 1], params, k, gen)
    print(f"{len(rows)} rows of the solver, {len(parts)} micro-batches, vocabulary {V}, the planner's {k} largest logits")
    print(f"warm start: loss {warm[0]:.3f} -> {warm[-1]:.3f}" if warm else "no warm start")
    print(f"distillation: loss {then[0]:.3f} -> {then[-1]:.3f}")
    print(f"divergence from the planner {first[0]:.3f} -> {last[0]:.3f}, same first token {first[1]:.2f} -> {last[1]:.2f}")
    print(f"answers token {token} with probability {p:.3f} (the planner's first: {int(said[int(rows[0])])})")
    return dict(first=first, last=last, warm=warm, distill=then, answer=(token, p))


if __name__ == "__main__":
    main()
