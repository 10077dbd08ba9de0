"""Distillation from a teacher's top logits through the vocabulary projection: the CUDA path against the fp64 oracle.

Tolerances.  A logit is summed on the tensor cores in segments of 256 of H: at most 17 additions that truncate (a step of 2^-23 of the
sum of magnitudes each) and one rounding per segment: 20 x 2^-23 of A = sum |x| |w| in all.  lse takes over the largest error of its
logits (over tau), an exponential of an argument of at most 2^7 (its rounding 2^-18 x ln 2 at the far end, where the terms are 2^-100;
2^-21 where they count) and a logarithm: 4e-6 + 2^-22 |lse|.  dX and dW: dY is rounded to bf16 (2^-8 of each term), the product once
more (2^-8 of the result); their random parts are at most 2^-8 / sqrt 3 each, so the norm of the difference stays below 4e-3."""
import numpy as np
import pytest
import torch

import oracle
from paper_2607_01844_b200 import binding, synth

pytestmark = pytest.mark.gpu

SUM_TOL = 20 * 2.0 ** -23


def inputs(N, H, V, K, seed=0, std=None, device="cuda", spread=1.0):
    g = torch.Generator(device=device).manual_seed(seed + 3)
    X = torch.randn((N, H), generator=g, device=device).to(torch.bfloat16)
    W = (torch.randn((H, V), generator=g, device=device) * (std or 2.0 / H ** 0.5)).to(torch.bfloat16)
    ids = (torch.rand((N, K), generator=g, device=device) * V * spread).to(torch.int32).clamp_(max=V - 1)
    t = torch.randn((N, K), generator=g, device=device) * 3
    dloss = torch.randn((N,), generator=g, device=device) + 0.5
    return X, W, ids, t, dloss


def forward(X, W, ids, t, tau, tlse=None, ws=None, stream=None):
    N, K = ids.shape
    loss, lse = torch.full((N,), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda")
    student = torch.full((N, K), 7.0, device="cuda")
    ws = binding.mop_vocab_distill_fwd(0, X, W, ids, t, tau, loss, student, lse, tlse, ws, stream)
    return loss, student, lse, ws


def backward(X, W, ids, t, tau, student, lse, dloss, tlse=None, ws=None, stream=None):
    dX = torch.full(X.shape, 3.0, device="cuda", dtype=torch.bfloat16)
    dW = torch.full(W.shape, 3.0, device="cuda", dtype=torch.bfloat16)
    ws = binding.mop_vocab_distill_bwd(0, X, W, ids, t, tau, student, lse, dloss, dX, dW, tlse, ws, stream)
    return dX, dW, ws


def f64(t):
    return t.double().cpu().numpy()


def host(X, W, ids, t, tlse):
    return synth.bits(X), synth.bits(W), ids.cpu().numpy(), f64(t), None if tlse is None else f64(tlse)


def check_forward(X, W, ids, t, tau, tlse, loss, student, lse):
    xb, wb, i, tt, tl = host(X, W, ids, t, tlse)
    want_loss, want_student, want_lse = oracle.vocab_distill(xb, wb, i, tt, tau, tl)
    A = np.abs(oracle.bf16_bits_to_f64(xb)) @ np.abs(oracle.bf16_bits_to_f64(wb))
    far = SUM_TOL * A.max(1)
    lse_tol = far / tau + 4e-6 + 2.0 ** -22 * np.abs(want_lse)
    assert (np.abs(f64(student) - want_student) <= far[:, None]).all()
    assert (np.abs(f64(lse) - want_lse) <= lse_tol).all()
    _, q, logq = oracle._teacher(i, tt, tau, wb.shape[1], tl)
    size = np.where(q > 0, q * (np.abs(np.where(q > 0, logq, 0)) + np.abs(want_student) / tau + np.abs(want_lse)[:, None]), 0).sum(1)
    # q itself is an exponential of an argument of at most 2^5 here: 2e-6 relative
    assert (np.abs(f64(loss) - want_loss) <= q.sum(1) * (lse_tol + far / tau) + 3e-6 * size).all()


def check_backward(X, W, ids, t, tau, tlse, dloss, dX, dW):
    xb, wb, i, tt, tl = host(X, W, ids, t, tlse)
    dY = oracle.vocab_distill_dlogits(xb, wb, i, tt, tau, f64(dloss), tl)
    x, w = oracle.bf16_bits_to_f64(xb), oracle.bf16_bits_to_f64(wb)
    for got, want, terms in ((f64(dX), dY @ w.T, np.abs(dY) @ np.abs(w).T), (f64(dW), x.T @ dY, np.abs(x).T @ np.abs(dY))):
        # (2^-7 of the terms: their rounding, and a softmax whose logits are off by the forward's bound)
        assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -7 * terms + 1e-30).all()
        norm = np.linalg.norm(want)
        assert np.linalg.norm(got - want) <= 4e-3 * norm


SHAPES = [
    # N, H, V, K, tau, teacher's own log-sum-exp, spread of the entries over the vocabulary
    (1, 8, 8, 1, 1.0, False, 1.0),
    (1, 64, 64, 3, 2.0, True, 1.0),
    (300, 128, 1024, 17, 1.0, False, 1.0),
    (129, 200, 328, 32, 1.5, False, 1.0),                # neither width a multiple of 64
    (257, 328, 8192 + 200, 64, 2.0, True, 1.0),
    (513, 256, 16384 + 72, 33, 4.0, False, 0.3),         # dX in several ranges of its columns
    (64, 1032, 4160, 100, 1.0, True, 1.0),               # five segments of K, the last of one block that is nearly empty
    (37, 72, 1000, 256, 0.5, False, 0.1),                # the longest lists, all within 100 columns: places named many times
    (1100, 136, 520, 128, 1.0, False, 1.0),
    # tiles of every width on single CTAs (one row per lane quarter and more), and both widths of a pair
    (3, 64, 9472, 20, 1.0, False, 1.0),                  # 64 columns
    (65, 128, 18944 - 8, 20, 1.0, True, 1.0),            # 128
    (64, 264, 28416 - 64, 31, 2.0, False, 1.0),          # 192
    (128, 128, 37888, 70, 1.0, False, 1.0),              # 256
    (90, 72, 57000, 9, 1.0, False, 0.01),                # 192, two rounds
    (129, 128, 9472 - 128, 40, 1.0, False, 1.0),         # a pair's 128
    (33, 2048, 264, 12, 1.0, False, 1.0),                # few columns, a long sum
]


@pytest.mark.parametrize("N,H,V,K,tau,full,spread", SHAPES, ids=lambda v: str(v))
def test_distillation_matches_the_oracle(N, H, V, K, tau, full, spread):
    X, W, ids, t, dloss = inputs(N, H, V, K, seed=N + V, spread=spread)
    ids[0, 0], ids[-1, -1] = 0, V - 1
    tlse = torch.logsumexp(t / tau, 1) + 0.4 if full else None
    loss, student, lse, ws = forward(X, W, ids, t, tau, tlse)
    binding.mop_vocab_poll(0, ws)
    check_forward(X, W, ids, t, tau, tlse, loss, student, lse)
    again = forward(X, W, ids, t, tau, tlse)
    assert all(torch.equal(a, b) for a, b in zip((loss, student, lse), again[:3]))        # reproducible bit for bit
    dX, dW, ws = backward(X, W, ids, t, tau, student, lse, dloss, tlse)
    binding.mop_vocab_poll(0, ws)
    check_backward(X, W, ids, t, tau, tlse, dloss, dX, dW)
    dX2, dW2, _ = backward(X, W, ids, t, tau, student, lse, dloss, tlse)
    assert torch.equal(dX, dX2) and torch.equal(dW, dW2)


@pytest.mark.parametrize("full", [False, True], ids=["renormalised", "whole"])
def test_short_lists_empty_lists_and_entries_without_probability(full):
    N, H, V, K = 140, 64, 700 // 8 * 8, 20
    X, W, ids, t, dloss = inputs(N, H, V, K, seed=5)
    tlse = torch.logsumexp(t, 1) + 0.2 if full else None
    ids[10:20, 5:] = -1                                  # short lists; their logits hold anything
    t[10:20, 5:] = float("nan")
    ids[20:30] = V                                       # behind the last column: no entries at all
    t[20:30] = float("inf")
    ids[30:40] = torch.iinfo(torch.int32).min
    ids[40:50] = 17                                      # one place, K times
    ids[50:60, 1:] = ids[50:60, :1]
    t[60:70, ::2] = -float("inf")                        # entries with probability 0
    t[70:75] = -float("inf")                             # nothing but those
    t[75:80, 3:] = torch.finfo(torch.float32).min
    loss, student, lse, _ = forward(X, W, ids, t, 1.0, tlse)
    clean = torch.where((ids >= 0) & (ids < V), t, 0.0)
    check_forward(X, W, ids, clean, 1.0, tlse, loss, student, lse)
    for rows in (slice(20, 40), slice(70, 75)):
        assert float(loss[rows].abs().max()) == 0.0
    dX, dW, _ = backward(X, W, ids, t, 1.0, student, lse, dloss, tlse)
    check_backward(X, W, ids, clean, 1.0, tlse, dloss, dX, dW)
    assert float(dX[20:40].abs().max()) == 0.0 and float(dX[70:75].abs().max()) == 0.0


def test_logits_far_from_zero():
    """A softmax that sits on one column, logits of some hundreds: nothing overflows, the rest of the row is 0."""
    N, H, V, K = 70, 64, 600, 8
    X, W, ids, t, dloss = inputs(N, H, V, K, seed=6, std=8.0)
    for tau in (1.0, 0.25, 30.0):
        loss, student, lse, _ = forward(X, W, ids, t, tau)
        xb, wb, i, tt, _ = host(X, W, ids, t, None)
        want_loss, want_student, want_lse = oracle.vocab_distill(xb, wb, i, tt, tau)
        # logits of up to 300: 20 x 2^-23 of sum |x| |w| (about 330), over tau
        assert np.abs(f64(lse) - want_lse).max() <= (SUM_TOL * 700 + 2.0 ** -22 * np.abs(want_lse).max()) / min(tau, 1.0)
        assert np.abs(f64(loss) - want_loss).max() <= 2 * (SUM_TOL * 700 / tau + 2.0 ** -21 * np.abs(want_loss).max())
        dX, dW, _ = backward(X, W, ids, t, tau, student, lse, dloss)
        check_backward(X, W, ids, t, tau, None, dloss, dX, dW)


@pytest.mark.parametrize("column", [40, 599])
@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=["nan", "inf"])
def test_a_logit_that_is_not_finite_shows_in_the_loss(column, value):
    N, H, V, K = 70, 128, 600, 4
    X, W, ids, t, _ = inputs(N, H, V, K, seed=7)
    ids[ids == column] = 0
    W[5, column] = value
    loss, _, lse, _ = forward(X, W, ids, t, 1.0)
    lost = ~(X[:, 5].double() * value < float("inf"))
    assert int(lost.sum()) > N // 4 and not torch.isfinite(loss[lost]).any() and not torch.isfinite(lse[lost]).any()
    assert torch.isfinite(loss[~lost]).all()


@pytest.mark.parametrize("N,H", [(100, 256), (200, 256), (33000, 72)], ids=["few-tokens", "one-block", "three-blocks"])
def test_nothing_is_taken_from_what_the_workspace_held(N, H):
    """The same bits whether the workspaces hold NaN, small counts or another call's sums, calls back to back."""
    V, K = 2 * 8192 + 72, 40
    calls = []
    for seed in (1, 2):
        X, W, ids, t, dloss = inputs(N, H, V, K, seed=seed)
        _, student, lse, _ = forward(X, W, ids, t, 2.0)
        calls.append((X, W, ids, t, dloss, student, lse))
    wf = torch.empty(binding.mop_vocab_distill_workspace_bytes(N, H, V, K), dtype=torch.uint8, device="cuda")
    wb = torch.empty(binding.mop_vocab_distill_bwd_workspace_bytes(N, H, V, K), dtype=torch.uint8, device="cuda")
    first = []
    for fill in (0xFF, 1, 2, None):
        for ws in (wf, wb):
            if fill == 0xFF:
                ws.fill_(fill)
            elif fill:
                ws.view(torch.int32).fill_(fill)
        out = []
        for X, W, ids, t, dloss, student, lse in calls:
            a = forward(X, W, ids, t, 2.0, None, wf)[:3]
            out.append((*a, *backward(X, W, ids, t, 2.0, student, lse, dloss, None, wb)[:2]))
        binding.mop_vocab_poll(0, wf)
        binding.mop_vocab_poll(0, wb)
        first = first or out
        for a, b in zip(first, out):
            assert all(torch.isfinite(y.float()).all() and torch.equal(x, y) for x, y in zip(a, b))


def test_on_another_stream_and_in_a_replayed_graph():
    N, H, V, K, tau = 150, 192, 8192 + 64, 24, 1.5
    X, W, ids, t, dloss = inputs(N, H, V, K, seed=11)
    want = forward(X, W, ids, t, tau)[:3]
    want_b = backward(X, W, ids, t, tau, want[1], want[2], dloss)[:2]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = forward(X, W, ids, t, tau, stream=side)
    got_b = backward(X, W, ids, t, tau, want[1], want[2], dloss, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want + want_b, got[:3] + got_b[:2]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, student, lse, _ = forward(X, W, ids, t, tau)
        dX, dW, _ = backward(X, W, ids, t, tau, student, lse, dloss)
    for old, new in zip((X, W, ids, t, dloss), inputs(N, H, V, K, seed=12)):
        old.copy_(new)
    graph.replay()
    check_forward(X, W, ids, t, tau, None, loss, student, lse)
    check_backward(X, W, ids, t, tau, None, dloss, dX, dW)


def test_nothing_is_written_outside_the_outputs_and_the_workspaces():
    N, H, V, K = 131, 72, 8192 + 328, 21
    X, W, ids, t, dloss = inputs(N, H, V, K, seed=13)
    margin, fences = 4096, []

    def fenced(shape, dtype=torch.uint8):
        n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        whole = torch.full((n + 2 * margin,), 0xA5, dtype=torch.uint8, device="cuda")
        fences.append((whole, n))
        return whole[margin:margin + n].view(dtype).view(shape)
    loss, student, lse = fenced((N,), torch.float32), fenced((N, K), torch.float32), fenced((N,), torch.float32)
    dX, dW = fenced((N, H), torch.bfloat16), fenced((H, V), torch.bfloat16)
    size = lambda n: -(-n // 256) * 256
    wf = fenced((size(binding.mop_vocab_distill_workspace_bytes(N, H, V, K)),))
    wb = fenced((size(binding.mop_vocab_distill_bwd_workspace_bytes(N, H, V, K)),))
    binding.mop_vocab_distill_fwd(0, X, W, ids, t, 1.0, loss, student, lse, None, wf)
    binding.mop_vocab_distill_bwd(0, X, W, ids, t, 1.0, student, lse, dloss, dX, dW, None, wb)
    check_forward(X, W, ids, t, 1.0, None, loss, student, lse)
    check_backward(X, W, ids, t, 1.0, None, dloss, dX, dW)
    for whole, n in fences:
        assert bool((whole[:margin] == 0xA5).all()) and bool((whole[margin + n:] == 0xA5).all())


@pytest.mark.parametrize("N,H,V", [(33000, 72, 16384 + 72),       # three blocks of columns, the last one shorter and of no whole chunk
                                   (33001, 328, 8192 + 8),        # two
                                   (700, 2048, 4096),             # one block, dX in several ranges
                                   (2304, 2040, 4096)],           # one block, dX in one range: stored at once
                         ids=lambda v: str(v))
def test_blocks_of_columns_against_fp64_on_the_device(N, H, V):
    K, tau = 50, 1.5
    X, W, ids, t, dloss = inputs(N, H, V, K, seed=N)
    loss, student, lse, _ = forward(X, W, ids, t, tau)
    dX, dW, _ = backward(X, W, ids, t, tau, student, lse, dloss)
    Y = X.double() @ W.double()
    ref = torch.logsumexp(Y / tau, 1)
    far = SUM_TOL * float((X.double().abs().max() * W.double().abs().sum(0).max()).item())
    assert float((lse.double() - ref).abs().max()) <= far / tau + 4e-6 + 2.0 ** -22 * float(ref.abs().max())
    q = torch.softmax(t.double() / tau, 1)
    want_loss = (q * (q.log() - Y.gather(1, ids.long()) / tau + ref[:, None])).sum(1)
    assert float((loss.double() - want_loss).abs().max()) <= 2 * far / tau + 4e-6 + 3e-6 * float(ref.abs().max())
    dY = torch.softmax(Y / tau, 1).scatter_add_(1, ids.long(), -q) * (dloss.double() / tau)[:, None]
    for got, want, terms in ((dX, dY @ W.double().T, dY.abs() @ W.double().abs().T), (dW, X.double().T @ dY, X.double().abs().T @ dY.abs())):
        err = (got.double() - want).abs()
        assert bool((err <= 2.0 ** -8 * want.abs() + 2.0 ** -7 * terms).all()) and float(err.norm() / want.norm()) <= 4e-3


def test_full_size_sampled_rows_and_invariant():
    """N = 8192, H = 7168, V = 131072: sampled tokens against the oracle, and the vocabulary sum of dW, which vanishes because every row
    of dY sums to zero (a renormalised teacher)."""
    N, H, V, K = 8192, 7168, 131072, 64
    X, W, ids, t, dloss = inputs(N, H, V, K, seed=15, std=0.02)
    loss, student, lse, ws = forward(X, W, ids, t, 2.0)
    binding.mop_vocab_poll(0, ws)
    r = torch.as_tensor(np.sort(np.random.default_rng(6).choice(N, 5, replace=False)), device="cuda")
    check_forward(X[r], W, ids[r], t[r], 2.0, None, loss[r], student[r], lse[r])
    dX, dW, ws = backward(X, W, ids, t, 2.0, student, lse, dloss)
    binding.mop_vocab_poll(0, ws)
    dY = oracle.vocab_distill_dlogits(synth.bits(X[r]), synth.bits(W), ids[r].cpu().numpy(), f64(t[r]), 2.0, f64(dloss[r]))
    want = dY @ oracle.bf16_bits_to_f64(synth.bits(W)).T
    assert np.linalg.norm(f64(dX[r]) - want) <= 4e-3 * np.linalg.norm(want)
    for h in range(0, H, 1024):                          # the roundings of V terms, each 2^-8 of one at most
        part = dW[h:h + 1024].double()
        assert float((part.sum(1).abs() / part.abs().sum(1)).max()) < 2.0 ** -8


@pytest.mark.parametrize("N,H,V", [(5, 7168, 409600), (33000, 64, 131072)], ids=["weights", "logits"])
def test_weights_and_logits_beyond_31_bits(N, H, V):
    """H V, or N V, > 2^31, against fp64 on the device in slabs of the vocabulary; entries at the far end."""
    K, tau = 8, 1.0
    X, W, ids, t, dloss = inputs(N, H, V, K, seed=N, std=2.0 / H ** 0.5)
    ids[:, -1] = V - 1 - torch.arange(N, device="cuda", dtype=torch.int32) % 100
    loss, student, lse, _ = forward(X, W, ids, t, tau)
    dX, dW, ws = backward(X, W, ids, t, tau, student, lse, dloss)
    binding.mop_vocab_poll(0, ws)
    x, step = X.double(), 1 << 13
    ref = torch.full((N,), -float("inf"), device="cuda", dtype=torch.float64)
    picked = torch.zeros((N, K), device="cuda", dtype=torch.float64)
    for v in range(0, V, step):
        Y = x @ W[:, v:v + step].double()
        ref = torch.logaddexp(ref, torch.logsumexp(Y, 1))
        here = (ids >= v) & (ids < v + step)
        picked = torch.where(here, Y.gather(1, (ids - v).clamp(0, Y.shape[1] - 1).long()), picked)
    far = SUM_TOL * 12 * H ** 0.5 * float(x.abs().max())          # sum |x| |w|: w has 2 / sqrt(H)
    assert float((student.double() - picked).abs().max()) <= far
    assert float((lse.double() - ref).abs().max()) <= far + 4e-6 + 2.0 ** -22 * float(ref.abs().max())
    q = torch.softmax(t.double(), 1)
    want_dX, err, norm = torch.zeros_like(x), 0.0, 0.0
    for v in range(0, V, step):
        w = W[:, v:v + step].double()
        dY = (x @ w - ref[:, None]).exp()
        here = (ids >= v) & (ids < v + step)
        dY.scatter_add_(1, torch.where(here, ids - v, 0).long(), torch.where(here, -q, 0.0))
        dY *= dloss.double()[:, None]
        want_dX += dY @ w.T
        want = x.T @ dY
        err, norm = err + float((dW[:, v:v + step].double() - want).square().sum()), norm + float(want.square().sum())
    assert (err / norm) ** 0.5 <= 4e-3
    assert float((dX.double() - want_dX).norm() / want_dX.norm()) <= 4e-3


def test_refusals():
    N, H, V, K = 64, 64, 128, 5
    X, W, ids, t, dloss = inputs(N, H, V, K, seed=16)
    loss, student, lse, ws = forward(X, W, ids, t, 1.0)
    dX, dW = torch.empty_like(X), torch.empty_like(W)

    def code(fn, *args):
        with pytest.raises(binding.MopError) as e:
            fn(*args)
        return e.value.code
    fwd, bwd = binding.mop_vocab_distill_fwd, binding.mop_vocab_distill_bwd
    for tau in (0.0, -1.0, float("nan"), float("inf")):
        assert code(fwd, 0, X, W, ids, t, tau, loss, student, lse, None, ws) == 1
    assert code(fwd, 0, X[:, :60].contiguous(), W[:60].contiguous(), ids, t, 1.0, loss, student, lse, None, ws) == 3
    assert code(fwd, 0, X, W[:, :100].contiguous(), ids, t, 1.0, loss, student, lse, None, ws) == 3
    long = torch.zeros((N, 257), dtype=torch.int32, device="cuda")
    assert code(fwd, 0, X, W, long, long.float(), 1.0, loss, long.float(), lse, None, ws) == 2
    assert code(fwd, 0, X, W, ids, t, 1.0, loss, student, lse, None, ws[128:]) == 3
    assert code(fwd, 0, X, W, ids, t, 1.0, loss, student, None, None, ws) == 1
    assert code(fwd, -1, X, W, ids, t, 1.0, loss, student, lse, None, ws) == 1
    wb = torch.empty(binding.mop_vocab_distill_bwd_workspace_bytes(N, H, V, K), dtype=torch.uint8, device="cuda")
    assert code(bwd, 0, X, W, ids, t, 1.0, None, lse, dloss, dX, dW, None, wb) == 1
    assert code(bwd, 0, X, W, ids, t, 1.0, student, lse, dloss, dX.view(-1)[1:64 * 64 - 63].view(63, 64), dW, None, wb) == 3
    assert binding.mop_vocab_distill_workspace_bytes(64, 64, 100, 5) == 0
    assert binding.mop_vocab_distill_bwd_workspace_bytes(64, 64, 128, 0) == 0


def test_no_tokens():
    X, W, ids, t, dloss = inputs(0, 64, 128, 3, seed=17)
    loss, student, lse, _ = forward(X, W, ids, t, 1.0)
    dX, dW, _ = backward(X, W, ids, t, 1.0, student, lse, dloss)
    assert float(dW.abs().max()) == 0.0


@pytest.mark.parametrize("N,H,V,K,tau", [(1, 64, 1000, 5, 1.0), (2, 200, 2888, 126, 1.0), (10, 1936, 4104, 126, 1.0), (33, 72, 8200, 64, 0.5), (64, 512, 8192, 31, 1.0),
                                         (65, 136, 8200, 126, 1.0), (100, 1000, 5000, 64, 4.0), (128, 256, 16384, 9, 1.0),
                                         (64, 8, (1 << 22) + 520, 4, 1.0), (128, 8, (1 << 21) + 520, 4, 1.0)])     # two blocks of columns
def test_few_tokens_keep_the_logit_gradients_to_sixteen_bits(N, H, V, K, tau):
    """Up to 128 tokens dY has two bf16 pieces: 2^-16 of each term is left out.  Sums: the tensor core drops up to 2^-23 of a partial sum in
    each step of 16, at most 512 steps in a range here (2^-14 of the terms); gradients are rounded once (2^-8).  dY itself is off by what
    its exponent is: the logits, twice (the sum behind lse, and formed again), 4e-6 + 2^-20 |lse| for lse and its scaling, 6e-6 for the
    exponential and the products around it, of p and of q."""
    X, W, ids, t, dloss = inputs(N, H, V, K, seed=N + K, std=2.0 / H ** 0.5)
    loss, student, lse, _ = forward(X, W, ids, t, tau)
    dX, dW, ws = backward(X, W, ids, t, tau, student, lse, dloss)
    binding.mop_vocab_poll(0, ws)
    x, w = X.double(), W.double()
    Y = x @ w
    ref = torch.logsumexp(Y / tau, 1)
    far = SUM_TOL * float((x.abs() @ w.abs()).max())
    valid = (ids >= 0) & (ids < V)
    at = torch.where(valid, ids, 0).long()
    s = torch.where(valid, t.double() / tau, -float("inf"))
    q = torch.where(valid, torch.softmax(s, 1), 0.0).nan_to_num(0.0)
    off = 2 * far / tau + 1e-5 + 2.0 ** -20 * ref.abs()[:, None]
    p = torch.exp(Y / tau - ref[:, None]) * q.sum(1, keepdim=True)
    size = p.scatter_add(1, at, q) * (dloss.double().abs()[:, None] / tau) * off
    dY = p.scatter_add(1, at, -q) * (dloss.double()[:, None] / tau)
    del Y, p
    for got, want, terms, base in ((dX, dY @ w.T, dY.abs() @ w.abs().T, size @ w.abs().T), (dW, x.T @ dY, x.abs().T @ dY.abs(), x.abs().T @ size)):
        assert bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -16 + 2.0 ** -14) * terms + base + 1e-30).all())
