"""Performance cases of the operators that draw a policy step's random choices:
its answers, token by token or from drafts, and the dropout of its model.

Every case is one pass through one of them; its ``op`` says which:

- ``uniform``: ``sf_uniform``, uniform numbers by counter;
- ``sample``: ``sf_token_sample``, a token and its log-probability per row of
  logits, from given uniform numbers;
- ``verify``: ``sf_draft_verify``, drafted tokens accepted or replaced so that
  the target's distribution results, over ragged sequences;
- ``dropout``: ``sf_dropout``, forward with or without a residual, and the
  gradient, whose mask is made again.

Ranges: 1 to 2.5e7 uniform numbers; 1 to 16000 rows of 500 to 131072 logits (at
most 2.7e8 bytes); 1 to 512 sequences of 0 to 9 drafts over the same
vocabularies (at most 6.1e8 bytes in all), with the draft's logits or with
drafts that were looked up; 1 to 20000 rows of 1 to 8192 entries for dropout (at
most 1.35e8), whole rows or a rank's columns of them; bfloat16, float16 and
float32; up to half of the vocabulary masked with -inf.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
WORD = 0xFFFFFFFF


def listed():
    return [
        # the numbers of one verification: latency
        dict(name="uniform_step", op="uniform", n=321, first=0, site=7),
        # those of a whole rollout, drawn ahead
        dict(name="uniform_ahead", op="uniform", n=20480007, first=12345678901, site=1),
        # the next token of one answer: latency
        dict(name="sample_single", op="sample", N=1, V=50001, pad=63, dtype="bf16", temperature=0.7, masked=0.0, done=0.0),
        # a server's batch; a tenth of its answers have ended
        dict(name="sample_batch", op="sample", N=1000, V=131072, pad=0, dtype="bf16", temperature=1.0, masked=0.0, done=0.1),
        # many short rows: a small vocabulary (bytes, actions), some not allowed
        dict(name="sample_small_vocab", op="sample", N=16000, V=515, pad=5, dtype="f16", temperature=1.3, masked=0.3, done=0.0),
        # five drafts of one answer: latency
        dict(name="verify_single", op="verify", B=1, K=5, ragged=False, V=65536, pad=0, dtype="bf16", temperature=0.8,
             draft_temperature=0.8, masked=0.0, lookup=False, noise=0.5),
        # a server's batch
        dict(name="verify_batch", op="verify", B=256, K=4, ragged=False, V=131072, pad=0, dtype="bf16", temperature=1.0,
             draft_temperature=1.0, masked=0.0, lookup=False, noise=0.5),
        # drafts that stop where the draft model was unsure; a grammar masks half of an odd vocabulary in float32
        dict(name="verify_ragged", op="verify", B=61, K=8, ragged=True, V=32003, pad=0, dtype="f32", temperature=0.9,
             draft_temperature=1.1, masked=0.5, lookup=False, noise=0.8),
        # drafts looked up in the prompt: no distribution of their own
        dict(name="verify_lookup", op="verify", B=200, K=9, ragged=True, V=50001, pad=7, dtype="f16", temperature=0.7,
             draft_temperature=1.0, masked=0.0, lookup=True, noise=0.0),
        # one rank's columns of a few hidden states
        dict(name="dropout_shard", op="dropout", N=30, C=513, pad=11, first=1026, across=2052, p=0.1, dtype="bf16",
             out="bf16", residual=False, site=3),
        # the hidden states of a large micro-batch onto their residual
        dict(name="dropout_residual", op="dropout", N=16384, C=8192, pad=0, first=0, across=8192, p=0.1, dtype="bf16",
             out="bf16", residual=True, site=12),
        # a float32 residual's gradient back to bfloat16 hidden states
        dict(name="dropout_grad", op="dropout", N=4099, C=2048, pad=0, first=0, across=2048, p=0.25, dtype="f32",
             out="bf16", residual=False, site=5),
    ]


def _spread(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["uniform", "sample", "sample", "verify", "verify", "verify", "dropout", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    pad = rng.choice([0, 0, 1, 7, rng.randint(0, 64)])
    if op == "uniform":
        return dict(op=op, n=_spread(rng, 1, 20000000), first=rng.choice([0, rng.randint(0, 1 << 40)]),
                    site=rng.randint(0, WORD))
    if op == "dropout":
        while True:
            N, C = _spread(rng, 1, 20000), _spread(rng, 1, 8192)
            if N * C <= 130000000:
                break
        across = rng.choice([C, C, 2 * C, C + rng.randint(0, 999)])
        return dict(op=op, N=N, C=C, pad=pad, first=rng.choice([0, 0, rng.randint(0, across - C), rng.randint(0, 1 << 36)]),
                    across=across, p=rng.choice([0.1, 0.0, rng.uniform(0.0, 0.6)]), dtype=dtype,
                    out=rng.choice([dtype, dtype, "f32", "bf16"]), residual=rng.random() < 0.5, site=rng.randint(0, 100))
    masked = rng.choice([0.0, 0.0, rng.uniform(0.0, 0.5)])
    temperature = rng.choice([1.0, rng.uniform(0.4, 1.5)])
    if op == "sample":
        while True:
            N, V = _spread(rng, 1, 16000), _spread(rng, 500, 131072)
            if N * V * BYTES[dtype] <= 260000000:
                break
        return dict(op=op, N=N, V=V, pad=pad, dtype=dtype, temperature=temperature, masked=masked,
                    done=rng.choice([0.0, rng.uniform(0.0, 0.5)]))
    lookup = rng.random() < 0.3
    while True:
        B, K, V = _spread(rng, 1, 512), rng.randint(1, 9), _spread(rng, 500, 131072)
        if B * (K + 1 + (0 if lookup else K)) * V * BYTES[dtype] <= 600000000:
            break
    return dict(op=op, B=B, K=K, ragged=rng.random() < 0.5, V=V, pad=pad, dtype=dtype, temperature=temperature,
                draft_temperature=rng.choice([temperature, rng.uniform(0.5, 1.4)]), masked=masked, lookup=lookup,
                noise=rng.choice([0.5, rng.uniform(0.1, 1.2)]))


# -- inputs ------------------------------------------------------------------

def _generator(seed, device="cuda"):
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    return gen


def _float32(x):
    return float(np.float32(x))


def _key(gen):
    """The seed of a run and the number of a step, as its program holds them."""
    return torch.cat([torch.randint(-(1 << 62), 1 << 62, (1,), generator=gen, device="cuda"),
                      torch.randint(0, 1 << 20, (1,), generator=gen, device="cuda")])


def _logits(N, V, pad, dtype, masked, gen):
    """Rows between flat ones and ones that a few tokens share."""
    buf = torch.empty((N, V + pad), dtype=dtype, device="cuda")
    step = max(1, (1 << 27) // (V + pad))
    for i in range(0, N, step):
        part = torch.randn(buf[i:i + step].shape, generator=gen, device="cuda")
        part *= torch.rand((part.shape[0], 1), generator=gen, device="cuda") * 3.5 + 1.5
        if masked:
            part[torch.rand(part.shape, generator=gen, device="cuda") < masked] = -math.inf
        buf[i:i + step] = part
    return buf[:, :V]


def _drawn(logits, inv_t, gen):
    """One token of each row, drawn from its distribution."""
    out = torch.empty((logits.shape[0],), dtype=torch.int64, device="cuda")
    step = max(1, (1 << 26) // logits.shape[1])
    for i in range(0, logits.shape[0], step):
        e = -torch.log(torch.rand(logits[i:i + step].shape, generator=gen, device="cuda").clamp(min=1e-30))
        out[i:i + step] = (logits[i:i + step].float() * inv_t - torch.log(e)).argmax(1)
    return out


def _counts(case):
    """Drafts of each sequence: K, or spread evenly from none to K."""
    B, K = case["B"], case["K"]
    if not case["ragged"]:
        return np.full((B,), K, dtype=np.int64)
    return (np.arange(B) + 1) * (K + 1) // (B + 1)


def prepare(case, seed):
    gen = _generator(seed)
    op = case["op"]
    state = dict(case=case)
    if op == "uniform":
        state["key"] = _key(gen)
    elif op == "sample":
        N = case["N"]
        state["logits"] = _logits(N, case["V"], case["pad"], DTYPES[case["dtype"]], case["masked"], gen)
        state["uniform"] = torch.rand((N,), generator=gen, device="cuda")
        # answers that have ended take no part
        state["uniform"][torch.randperm(N, generator=gen, device="cuda")[:int(case["done"] * N)]] = -1.0
        state["inv_t"] = _float32(1.0 / case["temperature"])
    elif op == "verify":
        counts = np.random.default_rng(seed).permutation(_counts(case))
        B, D, V, dtype = case["B"], int(counts.sum()), case["V"], DTYPES[case["dtype"]]
        start = torch.zeros((B + 1,), dtype=torch.int64)
        start[1:] = torch.cumsum(torch.from_numpy(counts), 0)
        state["inv_t"], state["draft_inv_t"] = _float32(1.0 / case["temperature"]), _float32(1.0 / case["draft_temperature"])
        state["target"] = target = _logits(D + B, V, case["pad"], dtype, case["masked"], gen)
        # the target's row that each draft was made for
        row = torch.arange(D) + torch.repeat_interleave(torch.arange(B), torch.from_numpy(counts), output_size=D)
        row = row.cuda()
        if case["lookup"]:
            state["draft"] = None
            guess = _drawn(target[row], state["inv_t"], gen) if D else torch.zeros((0,), dtype=torch.int64, device="cuda")
            wild = torch.randint(0, V, (D,), generator=gen, device="cuda")
            state["token"] = torch.where(torch.rand((D,), generator=gen, device="cuda") < 0.7, guess, wild)
        else:
            buf = torch.empty((D, V + case["pad"]), dtype=dtype, device="cuda")
            state["draft"] = buf[:, :V]
            step = max(1, (1 << 27) // V)
            for i in range(0, D, step):
                part = target[row[i:i + step]].float()
                part += torch.randn(part.shape, generator=gen, device="cuda") * case["noise"]
                state["draft"][i:i + step] = part
            state["token"] = _drawn(state["draft"], state["draft_inv_t"], gen)
        state["start"] = start.cuda()
        state["uniform"] = torch.rand((D + B,), generator=gen, device="cuda")
    else:
        N, C, W = case["N"], case["C"], case["C"] + case["pad"]
        state["key"] = _key(gen)
        state["x"] = torch.randn((N, W), generator=gen, device="cuda").to(DTYPES[case["dtype"]])[:, :C]
        state["residual"] = None
        if case["residual"]:
            state["residual"] = torch.randn((N, W), generator=gen, device="cuda").to(DTYPES[case["out"]])[:, :C]
    return state


# -- one pass ----------------------------------------------------------------

def _own(state):
    from paper_2606_06751_amd import draw as d

    case = state["case"]
    op = case["op"]
    if op == "uniform":
        return d.sf_uniform(case["n"], state["key"], site=case["site"], first=case["first"])
    if op == "sample":
        return d.sf_token_sample(state["logits"], state["uniform"], inv_temperature=state["inv_t"])
    if op == "verify":
        return d.sf_draft_verify(state["target"], state["draft"], state["token"], state["start"], state["uniform"],
                                 inv_temperature=state["inv_t"], draft_inv_temperature=state["draft_inv_t"])
    return d.sf_dropout(state["x"], case["p"], state["key"], site=case["site"], first=case["first"],
                        index_stride=case["across"], residual=state["residual"], out_dtype=DTYPES[case["out"]])


def _plain_words(key, block, kind, site):
    """The four words of each counter block (Philox4x32-10), as int64 tensors."""
    k0, k1 = key[0] & WORD, (key[0] >> 32) & WORD
    c0, c1 = block & WORD, (block >> 32) | (kind << 31)
    c2 = torch.full_like(block, site)
    c3 = torch.zeros_like(block) + (key[1] & WORD)
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & WORD) ^ c1 ^ k0, b & WORD, ((a >> 32) & WORD) ^ c3 ^ k1, a & WORD
        k0, k1 = (k0 + 0x9E3779B9) & WORD, (k1 + 0xBB67AE85) & WORD
    return c0, c1, c2, c3


def _plain_uniform(state):
    case = state["case"]
    lo, hi = case["first"] // 4, (case["first"] + case["n"] - 1) // 4
    block = torch.arange(lo, hi + 1, device="cuda")
    words = torch.stack(_plain_words(state["key"], block, 1, case["site"]), 1).reshape(-1)
    at = case["first"] - 4 * lo
    return (words[at:at + case["n"]] >> 8).float() * 2.0 ** -24


def _plain_sample(state):
    u = state["uniform"].double()
    z = state["logits"].double() * state["inv_t"]
    top = z.max(1).values
    e = torch.exp(z - top[:, None])
    c = torch.cumsum(e, 1)
    total = c[:, -1]
    token = (c <= (u * total)[:, None]).sum(1).clamp(max=z.shape[1] - 1)
    logp = (z.gather(1, token[:, None])[:, 0] - top - torch.log(total)).float()
    took = (u >= 0) & (u < 1)
    return torch.where(took, token, -1), torch.where(took, logp, torch.zeros_like(logp))


def _log_softmax(x, inv_t):
    z = x.double() * inv_t
    z -= z.max(1, keepdim=True).values
    return z - torch.log(torch.exp(z).sum(1, keepdim=True))


def _plain_verify(state):
    start, token, u = state["start"], state["token"], state["uniform"].double()
    B, D = start.shape[0] - 1, token.shape[0]
    V = state["target"].shape[1]
    count = start[1:] - start[:-1]
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), count, output_size=D)
    row = torch.arange(D, device="cuda") + seq
    logp = _log_softmax(state["target"], state["inv_t"])
    lp = logp[row, token]
    if state["draft"] is None:
        logq = None
        accept = u[row] < torch.exp(lp)
    else:
        logq = _log_softmax(state["draft"], state["draft_inv_t"])
        accept = u[row] * torch.exp(logq[torch.arange(D, device="cuda"), token]) < torch.exp(lp)
    place = torch.arange(D, device="cuda") - start[seq]
    accepted = count.clone().scatter_reduce_(0, seq, torch.where(accept, count[seq], place), "amin")
    # the row that each sequence draws its last token from
    last = start[:-1] + torch.arange(B, device="cuda") + accepted
    p = torch.exp(logp[last])
    refused = torch.nonzero(accepted < count)[:, 0]
    if refused.numel():
        at = (start[:-1] + accepted)[refused]
        if logq is None:
            p[refused, token[at]] = 0.0
        else:
            p[refused] = (p[refused] - torch.exp(logq[at])).clamp(min=0.0)
    c = torch.cumsum(p, 1)
    drawn = (c <= (u[start[1:] + torch.arange(B, device="cuda")] * c[:, -1])[:, None]).sum(1).clamp(max=V - 1)
    out = torch.full((D + B,), -1, dtype=torch.int64, device="cuda")
    out_logp = torch.zeros((D + B,), device="cuda")
    keep = place < accepted[seq]
    out[row] = torch.where(keep, token, -1)
    out_logp[row] = torch.where(keep, lp, torch.zeros_like(lp)).float()
    out[last] = drawn
    out_logp[last] = logp[last, drawn].float()
    return accepted, out, out_logp


def _plain_dropout(state):
    case = state["case"]
    N, C = case["N"], case["C"]
    threshold = math.floor(_float32(case["p"]) * 65536.0 + 0.5)
    index = case["first"] + torch.arange(N, device="cuda")[:, None] * case["across"] + torch.arange(C, device="cuda")
    lo, hi = case["first"] // 8, (case["first"] + (N - 1) * case["across"] + C - 1) // 8
    # by blocks where the rows follow each other, else by entries
    dense = case["across"] <= 2 * C
    words = _plain_words(state["key"], torch.arange(lo, hi + 1, device="cuda") if dense else index >> 3, 0, case["site"])
    if dense:
        halves = torch.stack([w >> s & 0xFFFF for w in words for s in (0, 16)], 1).to(torch.int32).reshape(-1)
        bits = halves[index - 8 * lo]
    else:
        bits = torch.zeros_like(index)
        for i, w in enumerate(words):
            for j in (0, 1):
                bits = torch.where((index & 7) == 2 * i + j, w >> 16 * j & 0xFFFF, bits)
    scale = 65536.0 / (65536 - threshold) if threshold < 65536 else 0.0
    y = torch.where(bits >= threshold, state["x"].float() * scale, 0.0)
    if state["residual"] is not None:
        y = y + state["residual"].float()
    return y.to(DTYPES[case["out"]])


PLAIN = {"uniform": _plain_uniform, "sample": _plain_sample, "verify": _plain_verify, "dropout": _plain_dropout}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


# -- what a pass cannot do without -------------------------------------------

def work(case):
    op = case["op"]
    if op == "uniform":
        return {"bytes": 4 * case["n"] + 16, "flops": 2 * case["n"]}
    if op == "sample":
        rows = case["N"] - int(case["done"] * case["N"])  # the others are not read
        return {"bytes": rows * case["V"] * BYTES[case["dtype"]] + 16 * case["N"], "flops": 4 * rows * case["V"]}
    if op == "verify":
        # every row once
        B, D = case["B"], int(_counts(case).sum())
        rows = D + B + (0 if case["lookup"] else D)
        return {"bytes": rows * case["V"] * BYTES[case["dtype"]] + 24 * D + 32 * B, "flops": 4 * rows * case["V"]}
    n = case["N"] * case["C"]
    each = BYTES[case["dtype"]] + BYTES[case["out"]] * (2 if case["residual"] else 1)
    return {"bytes": n * each + 16, "flops": 2 * n}


# -- the definition in 64 bits -----------------------------------------------

def _exact_words(key, block, kind, site):
    """[n, 4] words by numpy's unsigned arithmetic."""
    mask, half = np.uint64(WORD), np.uint64(32)
    k = [np.uint64(key[0] & WORD), np.uint64((key[0] >> 32) & WORD)]
    n = len(block)
    block = block.astype(np.uint64)
    c = [block & mask, (block >> half) + np.uint64(kind << 31), np.full(n, site, np.uint64),
         np.full(n, key[1] & WORD, np.uint64)]
    for _ in range(10):
        first, second = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(second >> half) ^ c[1] ^ k[0], second & mask, (first >> half) ^ c[3] ^ k[1], first & mask]
        k = [(k[0] + np.uint64(0x9E3779B9)) & mask, (k[1] + np.uint64(0xBB67AE85)) & mask]
    return np.stack(c, 1)


def _exact_pick(weights, u):
    """The lowest place whose weights up to it pass u of their sum."""
    sums = torch.cumsum(weights, 0)
    at = int(torch.searchsorted(sums, sums[-1:] * u, right=True))
    return min(at, int(torch.nonzero(weights)[-1]))


def _exact_sample(state):
    token = torch.full(state["uniform"].shape, -1, dtype=torch.int64)
    logp = torch.zeros(state["uniform"].shape, dtype=torch.float64)
    for i, u in enumerate(state["uniform"].tolist()):
        if 0.0 <= u < 1.0:
            p = torch.softmax(state["logits"][i].double() * state["inv_t"], 0)
            token[i] = _exact_pick(p, u)
            logp[i] = math.log(p[token[i]])
    return token.cuda(), logp.cuda()


def _exact_verify(state):
    start, draft, u = state["start"].tolist(), state["token"].tolist(), state["uniform"].tolist()
    B, D = len(start) - 1, len(draft)
    accepted = torch.zeros((B,), dtype=torch.int64)
    token = torch.full((D + B,), -1, dtype=torch.int64)
    logp = torch.zeros((D + B,), dtype=torch.float64)
    for b in range(B):
        for i in range(start[b], start[b + 1] + 1):
            p = torch.softmax(state["target"][i + b].double() * state["inv_t"], 0)
            weights = p
            if i < start[b + 1]:
                t = draft[i]
                if state["draft"] is None:
                    q = torch.zeros_like(p)
                    q[t] = 1.0
                else:
                    q = torch.softmax(state["draft"][i].double() * state["draft_inv_t"], 0)
                if u[i + b] * float(q[t]) < float(p[t]):
                    accepted[b] += 1
                    token[i + b], logp[i + b] = t, math.log(float(p[t]))
                    continue
                weights = torch.clamp(p - q, min=0.0)
            t = _exact_pick(weights, u[start[b + 1] + b])
            token[i + b], logp[i + b] = t, math.log(float(p[t]))
            break
    return accepted.cuda(), token.cuda(), logp.cuda()


def exact(case, seed):
    op = case["op"]
    if op == "dropout" and case["N"] * case["across"] > 60000000:
        return None  # some minutes of the host's time
    state = prepare(case, seed)
    if op == "sample":
        return _exact_sample(state)
    if op == "verify":
        return _exact_verify(state)
    key = state["key"].tolist()
    if op == "uniform":
        block = np.arange(case["first"] // 4, (case["first"] + case["n"] - 1) // 4 + 1, dtype=np.int64)
        words = _exact_words(key, block, 1, case["site"]).reshape(-1)
        at = case["first"] % 4
        return torch.from_numpy((words[at:at + case["n"]] >> np.uint64(8)).astype(np.float64) / 2.0 ** 24).cuda()
    N, C, first, across = case["N"], case["C"], case["first"], case["across"]
    block = np.arange(first // 8, (first + (N - 1) * across + C - 1) // 8 + 1, dtype=np.int64)
    halves = _exact_words(key, block, 0, case["site"]).astype("<u4").view("<u2").reshape(-1)
    threshold = int(_float32(case["p"]) * 65536.0 + 0.5)
    keep = np.stack([halves[first % 8 + r * across:first % 8 + r * across + C] >= threshold for r in range(N)])
    y = state["x"].double() * torch.from_numpy(keep).cuda()
    if threshold < 65536:
        y = y * (65536.0 / (65536 - threshold))
    return y if state["residual"] is None else y + state["residual"].double()
