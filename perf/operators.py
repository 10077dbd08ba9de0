"""The two auxiliary losses of a routed-expert language model's training step, as cases that can be timed.

`balance_fwd`, `balance_bwd`: the load-balance loss of a router with the per-expert counts, per sequence of a packed batch, and its
gradients with respect to the router's weights and the layer's input.  `distill_fwd`, `distill_bwd`: distillation from a teacher's top
logits through the vocabulary projection, and its gradients with respect to the hidden states and the projection's weights.

Where `own` is false, `run` computes them in plain torch operations; where it is true, through the framework's entry points.  Sizes are
those of the library's workloads (`synth.WORKLOADS`) and of its tests, or lie between them.
"""
from __future__ import annotations

import math

import torch

own = False

MOST_BALANCE = 4.0 * 16384 * 7168 * 256       # multiply-adds of the widest router's two gradients, times two
MOST_DISTILL = 6.0 * 4096 * 7168 * 131072     # of the projection's forward and its two gradients


def _balance(name, op, T, d, E, k, score="softmax", bias="none", seqs=1, tail=0, dlogits=False):
    c = {"op": op, "T": T, "d": d, "E": E, "k": k, "score": score, "bias": bias, "seqs": seqs, "tail": tail, "dlogits": dlogits}
    return {"name": name, **c} if name else c


def _distill(name, op, N, H, V, K, tau=1.0, full=False):
    c = {"op": op, "N": N, "H": H, "V": V, "K": K, "tau": tau, "full": full}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the smallest layer of the test suite: the calls themselves are all there is
        _balance("balance_fwd_tiny", "balance_fwd", 256, 256, 8, 2),
        # a packed batch of 13 sequences of a mid-size layer with padding behind the last one
        _balance("balance_fwd_packed", "balance_fwd", 4096, 2048, 64, 6, seqs=13, tail=77),
        # one batch of a trillion-scale layer, balanced as a whole
        _balance("balance_fwd_large", "balance_fwd", 16384, 7168, 256, 8, "sigmoid", "post"),
        # widths and counts that fit no tile, a bias before the score, gradients of the logits asked for as well
        _balance("balance_bwd_odd", "balance_bwd", 1537, 1000, 20, 3, "sigmoid", "pre", seqs=5, tail=9, dlogits=True),
        # training step of a mid-size layer
        _balance("balance_bwd_mid", "balance_bwd", 4096, 2048, 64, 6, seqs=2),
        # training step of a trillion-scale layer, balanced per sequence
        _balance("balance_bwd_large", "balance_bwd", 16384, 7168, 256, 8, "sigmoid", "post", seqs=4),
        # the last, short chunk of a document over a small vocabulary
        _distill("distill_fwd_few", "distill_fwd", 64, 2048, 32000, 20),
        # evaluation or training of a small student
        _distill("distill_fwd_mid", "distill_fwd", 2048, 2048, 32000, 64, tau=2.0),
        # full hidden size and vocabulary
        _distill("distill_fwd_large", "distill_fwd", 8192, 7168, 131072, 64, full=True),
        # gradients of a small micro-batch: the weights and their gradients are most of the traffic
        _distill("distill_bwd_few", "distill_bwd", 256, 2048, 32000, 32, tau=2.0),
        # a token count that fits no tile, a vocabulary whose last block of columns is short, an odd number of entries
        _distill("distill_bwd_odd", "distill_bwd", 1537, 2048, 50304, 99, full=True),
        # gradients at full hidden size and vocabulary
        _distill("distill_bwd_large", "distill_bwd", 4096, 7168, 131072, 64, tau=1.5),
    ]


def _log(rng, lo, hi, step=1):
    """Log-uniform in [lo, hi], a multiple of `step`."""
    return max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))) / step) * step)


def draw(rng):
    """One more case of the same ranges: tokens from 1 on, any number of experts, widths in multiples of 8, vocabularies of 8."""
    while True:
        op = rng.choice(["balance_fwd", "balance_bwd", "distill_fwd", "distill_bwd"])
        step = rng.choice([8, 64])
        if op.startswith("balance"):
            T, d, E = _log(rng, 1, 16384), _log(rng, 256, 7168, step), _log(rng, 8, 384)
            score = rng.choice(["softmax", "sigmoid"])
            bias = rng.choice(["none", "pre", "post"] if score == "sigmoid" else ["none", "pre"])
            if 4.0 * T * d * E <= MOST_BALANCE:
                tail = rng.choice([0, rng.randint(0, T // 8)])
                return _balance(None, op, T, d, E, rng.randint(1, min(8, E)), score, bias, rng.choice([1, _log(rng, 1, 32)]), tail,
                                rng.random() < 0.25)
        else:
            N, H, V = _log(rng, 1, 8192), _log(rng, 512, 7168, step), _log(rng, 4096, 131072, step)
            if (2.0 if op == "distill_fwd" else 6.0) * N * H * V <= MOST_DISTILL:
                return _distill(None, op, N, H, V, rng.randint(1, 128), rng.choice([1.0, 1.5, 2.0, 4.0]), rng.random() < 0.5)


def _generator(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1_000_003 + stream)
    return g


def _normal(shape, std, g, dtype=torch.bfloat16):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 27) // shape[1])
    for r in range(0, shape[0], step):
        part = out[r:r + step]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * std)
    return out


def _cuts(case, seed):
    """Sequence offsets of a packed batch: random cuts (an empty sequence may be among them), the last `tail` tokens are padding."""
    g = torch.Generator()
    g.manual_seed(seed * 31 + 7)
    end = case["T"] - case["tail"]
    inner = torch.randint(0, end + 1, (case["seqs"] - 1,), generator=g).sort().values
    return torch.cat([torch.zeros(1, dtype=torch.int64), inner, torch.full((1,), end)])


def _prepare_balance(case, seed):
    T, d, E, k = case["T"], case["d"], case["E"], case["k"]
    g = _generator(seed, 1)
    x = _normal((T, d), 1.0, g)
    W_r = _normal((d, E), 0.02, g, torch.float32)
    bias = torch.randn(E, generator=g, device="cuda") * 0.01 if case["bias"] != "none" else None
    logits = x.float() @ W_r
    key = logits if case["score"] == "softmax" else torch.sigmoid(logits)
    picks = torch.topk(key if bias is None else key + bias, k, dim=1).indices.to(torch.int32).contiguous()
    offsets = _cuts(case, seed).to(torch.int32).cuda()
    seqs = case["seqs"]
    # (from the offsets alone: counts are what the forward returns)
    owner = torch.searchsorted(offsets[1:], torch.arange(T, device="cuda", dtype=torch.int32), right=True)
    inside = (owner < seqs)[:, None].expand(T, k)
    counts = torch.bincount((owner.clamp(max=seqs - 1)[:, None] * E + picks)[inside], minlength=seqs * E).view(seqs, E).to(torch.int32)
    return {"case": case, "x": x, "W_r": W_r, "bias": bias, "logits": logits, "picks": picks, "offsets": offsets, "counts": counts,
            # upstream weight of a mean over the sequences, with the usual small coefficient
            "dloss": torch.full((seqs,), 0.01 / seqs, device="cuda") * (0.5 + torch.rand(seqs, generator=g, device="cuda"))}


def _prepare_distill(case, seed):
    N, H, V, K = case["N"], case["H"], case["V"], case["K"]
    g = _generator(seed, 2)
    X = _normal((N, H), 1.0, g)
    W = _normal((H, V), 0.02, g)
    # a teacher's list: frequent (low) tokens are likelier, logits fall with the rank, a few lists are short and a few tokens masked
    place = (torch.arange(K, device="cuda") + torch.rand((N, K), generator=g, device="cuda")) / K
    ids = (place.pow(1.5) * V).to(torch.int32).clamp(max=V - 1)
    t = 12.0 - 2.0 * torch.log1p(torch.arange(K, device="cuda", dtype=torch.float32)) + torch.randn((N, K), generator=g, device="cuda")
    t, rank = t.sort(dim=1, descending=True)
    ids = ids.gather(1, rank)
    length = torch.where(torch.rand(N, generator=g, device="cuda") < 0.1, torch.randint(0, K + 1, (N,), generator=g, device="cuda"), K)
    ids = torch.where(torch.arange(K, device="cuda")[None, :] < length[:, None], ids, -1).contiguous()
    st = {"case": case, "X": X, "W": W, "ids": ids, "t": t.contiguous(), "teacher_lse": None}
    if case["full"]:
        # the teacher's log-sum-exp over its whole vocabulary: its list holds most of the probability, not all
        s = torch.where(ids >= 0, t / case["tau"], -math.inf)
        st["teacher_lse"] = torch.logaddexp(torch.logsumexp(s, 1), torch.full((N,), 1.0, device="cuda"))
    if case["op"] == "distill_bwd":
        # what the forward leaves: the student's logits at the teacher's tokens and its log-sum-exp
        lse, student = torch.empty(N, device="cuda"), torch.empty((N, K), device="cuda")
        Wf = W.float()
        step = max(1, (1 << 28) // V)
        for r in range(0, N, step):
            y = X[r:r + step].float() @ Wf
            lse[r:r + step] = torch.logsumexp(y / case["tau"], 1)
            i = ids[r:r + step]
            student[r:r + step] = torch.where(i >= 0, y.gather(1, i.clamp(min=0).long()), 0.0)
        st["lse"], st["student"] = lse, student
        # upstream weight of a mean over the tokens
        st["dloss"] = torch.full((N,), 1.0 / N, device="cuda") * (0.5 + torch.rand(N, generator=g, device="cuda"))
    return st


def prepare(case, seed):
    return _prepare_balance(case, seed) if case["op"].startswith("balance") else _prepare_distill(case, seed)


# ------------------------------------------------------------------------------------------------ plain forms
def _scores(st):
    z = st["logits"]
    if st["case"]["bias"] == "pre":
        z = z + st["bias"]
    if st["case"]["score"] == "softmax":
        e = torch.exp(z - z.max(1, keepdim=True).values)
        return e / e.sum(1, keepdim=True), None
    s = 1.0 / (1.0 + torch.exp(-z))
    return s / s.sum(1, keepdim=True), s


def _members(st):
    """[S, T] 0/1 matrix of the tokens of each sequence, and the sequences' lengths."""
    off, T = st["offsets"].long(), st["case"]["T"]
    t = torch.arange(T, device=off.device)[None, :]
    return ((t >= off[:-1, None]) & (t < off[1:, None])).float(), (off[1:] - off[:-1]).float()


def _plain_balance_fwd(st):
    c = st["case"]
    p, _ = _scores(st)
    member, length = _members(st)
    picked = (st["picks"].long()[:, :, None] == torch.arange(c["E"], device=p.device)).float().sum(1)
    counts = member @ picked
    prob = (member @ p) / length.clamp(min=1)[:, None]
    loss = (counts * prob).sum(1) * (c["E"] / c["k"]) / length.clamp(min=1)
    return {"counts": counts.to(torch.int32), "prob": prob, "loss": loss}


def _plain_balance_bwd(st):
    c = st["case"]
    p, s = _scores(st)
    member, length = _members(st)
    weight = st["dloss"] * (c["E"] / c["k"]) / length.clamp(min=1) ** 2
    coef = member.T @ (weight[:, None] * st["counts"].float())
    dz = p * (coef - (p * coef).sum(1, keepdim=True))
    if s is not None:
        dz = dz * (1.0 - s)
    out = {"dW_r": st["x"].float().T @ dz, "dX": (dz @ st["W_r"].T).to(torch.bfloat16)}
    if c["bias"] == "pre":
        out["dbias"] = dz.sum(0)
    if c["dlogits"]:
        out["dlogits"] = dz
    return out


def _teacher(st):
    valid = st["ids"] >= 0
    t = torch.where(valid, st["t"] / st["case"]["tau"], -math.inf)
    if st["teacher_lse"] is not None:
        q = torch.exp(t - st["teacher_lse"][:, None])
        return valid, q, torch.where(valid, t - st["teacher_lse"][:, None], 0.0)
    m = t.max(1, keepdim=True).values
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(t - m)
    total = e.sum(1, keepdim=True)
    total = torch.where(total == 0.0, 1.0, total)
    return valid, e / total, torch.where(valid, t - m - torch.log(total), 0.0)


def _plain_distill_fwd(st):
    tau = st["case"]["tau"]
    y = st["X"].float() @ st["W"].float()
    m = y.max(1, keepdim=True).values
    lse = m[:, 0] / tau + torch.log(torch.exp((y - m) / tau).sum(1))
    valid, q, logq = _teacher(st)
    student = torch.where(valid, y.gather(1, st["ids"].clamp(min=0).long()), 0.0)
    loss = (q * (logq - student / tau + lse[:, None])).sum(1)
    return {"loss": loss, "lse": lse, "student": student}


def _plain_distill_bwd(st):
    tau = st["case"]["tau"]
    X, W = st["X"].float(), st["W"].float()
    valid, q, _ = _teacher(st)
    dY = torch.exp((X @ W) / tau - st["lse"][:, None]) * q.sum(1, keepdim=True)
    dY.scatter_add_(1, st["ids"].clamp(min=0).long(), -q)
    dY *= (st["dloss"] / tau)[:, None]
    return {"dX": (dY @ W.T).to(torch.bfloat16), "dW": (X.T @ dY).to(torch.bfloat16)}


# ------------------------------------------------------------------------------------------------ the framework's calls
_kept = {}     # what a program keeps from step to step: a context per layer shape, a workspace per call shape


def _context(c):
    from paper_2607_01844_b200 import binding, synth
    key = tuple(c[n] for n in ("T", "d", "E", "k", "score", "bias"))
    if key not in _kept:
        score = synth.SCORE_SOFTMAX if c["score"] == "softmax" else synth.SCORE_SIGMOID
        mode = {"none": synth.BIAS_NONE, "pre": synth.BIAS_PRE_LOGIT, "post": synth.BIAS_POST_SCORE}[c["bias"]]
        _kept[key] = binding.Context(c["T"], c["d"], c["E"], c["k"], 64, score, mode)
    return _kept[key]


def _workspace(key, size):
    if key not in _kept:
        _kept[key] = torch.empty(max(256, size()), dtype=torch.uint8, device="cuda")
    return _kept[key]


def _own_balance(st):
    from paper_2607_01844_b200 import binding
    c = st["case"]
    ctx, seqs, backward = _context(c), c["seqs"], c["op"] == "balance_bwd"
    ws = _workspace((c["op"], id(ctx), seqs), lambda: binding.mop_moe_balance_workspace_bytes(ctx, seqs, backward))
    f32 = dict(dtype=torch.float32, device="cuda")
    if not backward:
        counts = torch.empty((seqs, c["E"]), dtype=torch.int32, device="cuda")
        prob, loss = torch.empty((seqs, c["E"]), **f32), torch.empty((seqs,), **f32)
        binding.mop_moe_balance_loss_fwd(ctx, st["logits"], st["bias"], st["picks"], st["offsets"], counts, prob, loss, ws)
        return {"counts": counts, "prob": prob, "loss": loss}
    out = {"dW_r": torch.empty((c["d"], c["E"]), **f32), "dX": torch.empty((c["T"], c["d"]), dtype=torch.bfloat16, device="cuda")}
    if c["bias"] == "pre":
        out["dbias"] = torch.empty((c["E"],), **f32)
    if c["dlogits"]:
        out["dlogits"] = torch.empty((c["T"], c["E"]), **f32)
    binding.mop_moe_balance_loss_bwd(ctx, st["logits"], st["bias"], st["offsets"], st["counts"], st["dloss"], st["x"], st["W_r"],
                                     out.get("dlogits"), out["dW_r"], out.get("dbias"), out["dX"], False, ws)
    return out


def _own_distill(st):
    from paper_2607_01844_b200 import binding
    c = st["case"]
    N, H, V, K = c["N"], c["H"], c["V"], c["K"]
    f32 = dict(dtype=torch.float32, device="cuda")
    if c["op"] == "distill_fwd":
        ws = _workspace(("distill_fwd", N, H, V, K), lambda: binding.mop_vocab_distill_workspace_bytes(N, H, V, K))
        loss, lse, student = torch.empty((N,), **f32), torch.empty((N,), **f32), torch.empty((N, K), **f32)
        binding.mop_vocab_distill_fwd(0, st["X"], st["W"], st["ids"], st["t"], c["tau"], loss, student, lse, st["teacher_lse"], ws)
        return {"loss": loss, "lse": lse, "student": student}
    ws = _workspace(("distill_bwd", N, H, V, K), lambda: binding.mop_vocab_distill_bwd_workspace_bytes(N, H, V, K))
    dX = torch.empty((N, H), dtype=torch.bfloat16, device="cuda")
    dW = torch.empty((H, V), dtype=torch.bfloat16, device="cuda")
    binding.mop_vocab_distill_bwd(0, st["X"], st["W"], st["ids"], st["t"], c["tau"], st["student"], st["lse"], st["dloss"], dX, dW,
                                  st["teacher_lse"], ws)
    return {"dX": dX, "dW": dW}


def run(state):
    op = state["case"]["op"]
    if own:
        return _own_balance(state) if op.startswith("balance") else _own_distill(state)
    return {"balance_fwd": _plain_balance_fwd, "balance_bwd": _plain_balance_bwd,
            "distill_fwd": _plain_distill_fwd, "distill_bwd": _plain_distill_bwd}[op](state)


# ------------------------------------------------------------------------------------------------ definition in 64 bits
def _exact_balance(c, st):
    """Sequence by sequence, as the loss is defined."""
    E, k, off = c["E"], c["k"], st["offsets"].tolist()
    z = st["logits"].double() + (st["bias"].double() if c["bias"] == "pre" else 0.0)
    f64 = dict(dtype=torch.float64, device="cuda")
    counts, prob, loss = torch.zeros((c["seqs"], E), dtype=torch.int64, device="cuda"), torch.zeros((c["seqs"], E), **f64), torch.zeros(c["seqs"], **f64)
    dz = torch.zeros_like(z)
    for s in range(c["seqs"]):
        rows = slice(off[s], off[s + 1])
        n = off[s + 1] - off[s]
        if n == 0:
            continue
        score = torch.softmax(z[rows], 1) if c["score"] == "softmax" else torch.sigmoid(z[rows])
        p = score / score.sum(1, keepdim=True)
        counts[s] = torch.bincount(st["picks"][rows].reshape(-1).long(), minlength=E)
        prob[s] = p.mean(0)
        loss[s] = E / (k * n) * torch.dot(counts[s].double(), prob[s])
        dp = (st["dloss"][s].double() * E / (k * n * n) * counts[s].double()).expand(n, E)
        ds = (dp - (dp * p).sum(1, keepdim=True)) / score.sum(1, keepdim=True)
        dz[rows] = ds * score if c["score"] == "softmax" else ds * score * (1.0 - score)
    if c["op"] == "balance_fwd":
        return {"counts": counts, "prob": prob, "loss": loss}
    out = {"dW_r": st["x"].double().T @ dz, "dX": dz @ st["W_r"].double().T}
    if c["bias"] == "pre":
        out["dbias"] = dz.sum(0)
    if c["dlogits"]:
        out["dlogits"] = dz
    return out


def _exact_distill(c, st):
    """A block of tokens at a time, teacher and student as distributions over the whole vocabulary."""
    N, V, tau = c["N"], c["V"], c["tau"]
    W = st["W"].double()
    loss, lse, student, dX, dW = [], [], [], [], 0.0
    step = max(1, (1 << 27) // V)
    for r in range(0, N, step):
        rows = slice(r, r + step)
        X, ids = st["X"][rows].double(), st["ids"][rows].long()
        y = X @ W
        lse.append(torch.logsumexp(y / tau, 1))
        logp = (y / tau).sub_(lse[-1][:, None])
        t = torch.where(ids >= 0, st["t"][rows].double() / tau, -math.inf)
        norm = torch.logsumexp(t, 1) if st["teacher_lse"] is None else st["teacher_lse"][rows].double()
        q = torch.where(ids >= 0, torch.exp(t - norm[:, None]), 0.0)
        at = ids.clamp(min=0)
        student.append(torch.where(ids >= 0, y.gather(1, at), 0.0))
        loss.append((torch.special.xlogy(q, q) - q * logp.gather(1, at)).sum(1))
        if c["op"] == "distill_bwd":
            dY = logp.exp_().mul_(q.sum(1, keepdim=True)).scatter_add_(1, at, -q).mul_(st["dloss"][rows].double()[:, None] / tau)
            dX.append(dY @ W.T)
            dW = dW + X.T @ dY
    if c["op"] == "distill_fwd":
        return {"loss": torch.cat(loss), "lse": torch.cat(lse), "student": torch.cat(student)}
    return {"dX": torch.cat(dX), "dW": dW}


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_balance(case, st) if case["op"].startswith("balance") else _exact_distill(case, st)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"].startswith("balance"):
        T, d, E, k, S = (c[n] for n in ("T", "d", "E", "k", "seqs"))
        if c["op"] == "balance_fwd":
            return {"bytes": 4.0 * T * E + 4.0 * T * k + 8.0 * S * E, "flops": 6.0 * T * E}
        return {"bytes": 4.0 * T * E * (2 if c["dlogits"] else 1) + 4.0 * T * d + 8.0 * d * E + 4.0 * S * E, "flops": 4.0 * T * d * E}
    N, H, V, K = (c[n] for n in ("N", "H", "V", "K"))
    if c["op"] == "distill_fwd":
        return {"bytes": 2.0 * N * H + 2.0 * H * V + 12.0 * N * K + 8.0 * N, "flops": 2.0 * N * H * V}
    return {"bytes": 4.0 * N * H + 4.0 * H * V + 12.0 * N * K + 8.0 * N, "flops": 6.0 * N * H * V}
