"""A small data-parallel policy-training loop that keeps both of the library's
records: where each step's time went, and the step's own numbers.

Every rank has its own answers of ragged lengths (the commonest cause of ranks
waiting for each other).  Per step and rank the stages data, forward, backward
and optimizer are timed on the host; the numbers of the step (loss, KL, clipped
share, entropy, gradient norm, entries that are not finite) are taken on the
stream by the operators of stagefrontier_train.h and read once at the end, so
the record costs the loop no synchronisation.  The stage times of a window are
then gathered and accounted with ``sf_ingest`` and ``sf_frontier_summary``.

The ranks of this example take turns on one GPU and their gradients are added
in place of an all-reduce; the policy is one matrix over fixed features.

    python examples/policy_step.py [--ranks 4] [--steps 20] [--vocab 4099]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_06751_amd import stagefrontier as sf  # noqa: E402
from paper_2606_06751_amd import train  # noqa: E402

STAGES = ("data", "forward", "backward", "optimizer", "other")


def run(ranks=4, steps=20, vocab=4099, width=64, answers=8, longest=60, lr=20.0, max_norm=0.02, seed=0, device="cuda:0"):
    """Trains, and returns the record: per-step terms [T, 4], entropies, norms,
    non-finite counts, and the window's exposed time per stage with its top-2."""
    dev = torch.device(device)
    gen = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen).to(dev)

    weight, bias = normal(vocab, width) * 0.05, torch.zeros(vocab, device=dev)
    ref_weight = weight.clone()
    # per rank: features of each position, tokens taken, which are prompts, one
    # advantage per answer
    data = []
    for r in range(ranks):
        length = torch.randint(1, longest + 1, (answers,), generator=gen)
        start = torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(length, 0)])
        N = int(start[-1])
        data.append(dict(x=normal(N, width), t=torch.randint(0, vocab, (N,), generator=gen).to(dev),
                         mask=(torch.rand(N, generator=gen) < 0.8).to(dev), start=start.to(dev),
                         adv=normal(answers) + 0.5))
    tokens = sum(int(d["mask"].sum()) for d in data)
    for d in data:
        d["old"], _, _ = train.sf_token_logp(d["x"] @ weight.t(), d["t"], entropy=False)
        d["ref"], _, _ = train.sf_token_logp(d["x"] @ ref_weight.t(), d["t"], entropy=False)

    grads = train.GradSet([torch.zeros_like(weight), torch.zeros_like(bias)])
    terms = torch.zeros((steps, ranks, 4), device=dev)
    entropy = torch.zeros((steps, ranks), device=dev)
    total = torch.zeros((steps, 1), device=dev)
    wrong = torch.zeros((steps, 2), dtype=torch.int64, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    stages = torch.zeros((ranks, steps, 4), dtype=torch.int64)
    wall = torch.zeros((ranks, steps), dtype=torch.int64)
    for step in range(steps):
        begin = [0] * ranks
        for r, d in enumerate(data):
            begin[r] = t0 = time.perf_counter_ns()
            x, t = d["x"], torch.where(d["mask"], d["t"], -1)
            if r == 0:
                for g in grads.tensors:
                    g.zero_()
            t1 = time.perf_counter_ns()
            logits = torch.addmm(bias, x, weight.t())
            logp, lse, ent = train.sf_token_logp(logits, t)
            _, grad = train.sf_policy_loss(logp, d["old"], d["adv"], d["start"], ref_logp=d["ref"], mask=d["mask"],
                                           reduction=train.SF_SUM_TOKENS, scale=1.0 / tokens, kl_coef=0.02,
                                           out_terms=terms[step, r])
            entropy[step, r] = ent.sum() / tokens
            t2 = time.perf_counter_ns()
            train.sf_token_logp_grad(logits, t, lse, grad, out_grad=logits)
            grads.tensors[0].addmm_(logits.t(), x)
            grads.tensors[1].add_(logits.sum(0))
            t3 = time.perf_counter_ns()
            stages[r, step, 0], stages[r, step, 1], stages[r, step, 2] = t1 - t0, t2 - t1, t3 - t2
        t3 = time.perf_counter_ns()
        train.sf_grad_norm(grads, out_total=total[step], out_nonfinite=wrong[step])
        train.sf_grad_clip(grads, total[step], max_norm, status=status)
        weight.add_(grads.tensors[0], alpha=-lr)
        bias.add_(grads.tensors[1], alpha=-lr)
        t4 = time.perf_counter_ns()
        for r in range(ranks):
            stages[r, step, 3] = t4 - t3
            wall[r, step] = int(stages[r, step].sum()) + 1000
    d_ns, _ = sf.sf_ingest(stages.to(dev), wall.to(dev))
    _, _, exposed, _, top2 = sf.sf_frontier_summary(d_ns, window=steps)
    return dict(terms=terms.sum(1).cpu(), entropy=entropy.sum(1).cpu(), norm=total[:, 0].cpu(), wrong=wrong.cpu(),
                status=int(status), exposed=exposed[0].cpu(), top2=top2[0].cpu())


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--ranks", type=int, default=4)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--vocab", type=int, default=4099)
    a = ap.parse_args()
    rec = run(a.ranks, a.steps, a.vocab)
    print("step      loss    policy        kl  clipped  entropy      norm  not finite")
    for k in range(a.steps):
        loss, policy, kl, clipped = rec["terms"][k].tolist()
        print("%4d %9.5f %9.5f %9.6f %8.4f %8.4f %9.6f %11d" % (k, loss, policy, kl, clipped, rec["entropy"][k],
                                                                  rec["norm"][k], rec["wrong"][k].sum()))
    share = rec["exposed"].double() / rec["exposed"].sum()
    print("exposed time: " + ", ".join("%s %.1f%%" % (s, 100 * v) for s, v in zip(STAGES, share.tolist())))
    print("top-2: " + ", ".join("%s on rank %d" % (STAGES[s], r) for s, r in rec["top2"].tolist()))


if __name__ == "__main__":
    main()
