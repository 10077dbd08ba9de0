"""Load-balance loss of the router: the CUDA path against the fp64 oracle.

Tolerances.  A score p is an exponential of an argument of at most 32 in size (its rounding, 2^-20 of log2 units, is 6.6e-7 of the
value; the exponential itself 2.4e-7), a sum and a division: 1.5e-6 relative at most.  A mean adds at most 7 + 16 + 148 + 8 terms in a
row, each half a step of 2^-24 off: 1.1e-5 more.  dz = w p (c - m) with the counts taken relative to their mean: 5e-6 of w p (|c| + m|c|).
dW_r adds T such terms in fp32 (pieces of dz of 24 bits): 1e-5 of sum |x| |dz|.  dX: operands of 11 bits (2 x 2^-11 of sum |dz| |W_r|) and
one rounding to bf16 (2^-8 of the result)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2607_01844_b200 import binding, synth

pytestmark = pytest.mark.gpu

SOFTMAX, SIGMOID = synth.SCORE_SOFTMAX, synth.SCORE_SIGMOID
NONE, POST, PRE = synth.BIAS_NONE, synth.BIAS_POST_SCORE, synth.BIAS_PRE_LOGIT
P_RTOL = 1.3e-5


class Case:
    """Inputs on the device (padding rows hold NaN everywhere), a context and a workspace that starts as NaN."""

    def __init__(self, T, d, E, k, score, mode, off, seed=0, std=1.5, path=binding.GEMM_AUTO):
        g = torch.Generator(device="cuda").manual_seed(seed + 17)
        self.T, self.d, self.E, self.k, self.score, self.mode, self.off = T, d, E, k, score, mode, off
        self.logits = torch.randn((T, E), generator=g, device="cuda") * std
        self.bias = torch.randn(E, generator=g, device="cuda") * 0.2 if mode != NONE else None
        self.idx = torch.rand((T, E), generator=g, device="cuda").topk(k, 1).indices.to(torch.int32).contiguous() if T else \
            torch.empty((0, k), dtype=torch.int32, device="cuda")
        self.x = torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16)
        self.W_r = torch.randn((d, E), generator=g, device="cuda") * 0.05
        self.S = len(off) - 1 if off is not None else 1
        self.dloss = torch.randn(self.S, generator=g, device="cuda") + 0.3
        self.offs = None if off is None else torch.tensor(off, dtype=torch.int32, device="cuda")
        self.bounds = [0, T] if off is None else off
        self.pad = torch.ones(T, dtype=torch.bool)
        self.pad[self.bounds[0]:self.bounds[-1]] = False
        self.pad = self.pad.cuda()
        self.logits[self.pad] = float("nan")
        self.x[self.pad] = float("nan")
        self.idx[self.pad] = 1 << 30
        self.ctx = binding.Context(T, d, E, k, 64, score, mode, gemm_path=path)

    def workspace(self, backward):
        n = max(256, binding.mop_moe_balance_workspace_bytes(self.ctx, self.S, backward))
        return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")

    def forward(self, stream=None, ws=None):
        counts = torch.full((self.S, self.E), -7, dtype=torch.int32, device="cuda")
        prob, loss = torch.full((self.S, self.E), 7.0, device="cuda"), torch.full((self.S,), 7.0, device="cuda")
        binding.mop_moe_balance_loss_fwd(self.ctx, self.logits, self.bias, self.idx, self.offs, counts, prob, loss,
                                         self.workspace(False) if ws is None else ws, stream)
        return counts, prob, loss

    def outputs(self, fill=3.0):
        f32 = dict(device="cuda", dtype=torch.float32)
        return {"dlogits": torch.full((self.T, self.E), fill, **f32), "dW_r": torch.full((self.d, self.E), fill, **f32),
                "dbias": torch.full((self.E,), fill, **f32), "dX": torch.full((self.T, self.d), fill, device="cuda", dtype=torch.bfloat16)}

    def backward(self, counts, out, accumulate=False, stream=None, ws=None):
        binding.mop_moe_balance_loss_bwd(self.ctx, self.logits, self.bias, self.offs, counts, self.dloss, self.x, self.W_r,
                                         out.get("dlogits"), out.get("dW_r"), out.get("dbias"), out.get("dX"), accumulate,
                                         self.workspace(True) if ws is None else ws, stream)
        return out

    def np(self, t):
        return None if t is None else t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()

    def reference(self):
        fwd = oracle.balance_loss(self.np(self.logits), self.np(self.bias), self.k, self.score, self.mode, self.np(self.idx), self.bounds)
        dz = oracle.balance_loss_bwd(self.np(self.logits), self.np(self.bias), self.k, self.score, self.mode, fwd[0], self.bounds,
                                     self.np(self.dloss))
        return fwd, dz

    def dz_scale(self, counts):
        """w p (|c| + sum p |c|) with c relative to the mean count, per logit: what 5e-6 is relative to."""
        out = np.zeros((self.T, self.E))
        for s in range(self.S):
            a, b = self.bounds[s], self.bounds[s + 1]
            if a == b:
                continue
            _, p, _ = oracle._balance_scores(self.np(self.logits[a:b]), self.np(self.bias), self.score, self.mode)
            c = np.abs(counts[s] - np.rint(self.k * (b - a) / self.E))[None, :]
            out[a:b] = abs(float(self.dloss[s])) * self.E / (self.k * (b - a) ** 2) * p * (c + (p * c).sum(1, keepdims=True))
        return out


def check_forward(c, got):
    counts, prob, loss = (c.np(t) for t in got)
    (want_counts, want_prob, want_loss), _ = c.reference()
    assert np.array_equal(counts, want_counts)
    assert np.allclose(prob, want_prob, rtol=P_RTOL, atol=1e-30), np.abs(prob / np.maximum(want_prob, 1e-30) - 1).max()
    assert np.allclose(loss, want_loss, rtol=2 * P_RTOL, atol=0)
    return want_counts


def check_backward(c, out, base=0.0, accumulate=False):
    (counts, _, _), dz = c.reference()
    scale = c.dz_scale(counts)
    pad = c.pad.cpu().numpy()
    x, W = np.where(pad[:, None], 0.0, c.np(c.x)), c.np(c.W_r)
    base = base if accumulate else 0.0
    if "dlogits" in out:
        assert (np.abs(c.np(out["dlogits"]) - dz) <= 5e-6 * scale + 1e-6 * np.abs(dz)).all()
    if "dbias" in out:
        want = dz.sum(0) if c.mode == PRE else np.zeros(c.E)
        got = c.np(out["dbias"])
        assert (np.abs(got - base - want) <= 1e-5 * (scale + np.abs(dz)).sum(0) + 2.0 ** -24 * abs(base)).all()
    if "dW_r" in out:
        got, want = c.np(out["dW_r"]), x.T @ dz
        assert (np.abs(got - base - want) <= 1e-5 * (np.abs(x).T @ (scale + np.abs(dz))) + 2.0 ** -24 * abs(base)).all()
    if "dX" in out:
        got, want = c.np(out["dX"]), base + dz @ W.T
        # (half a step of a subnormal result, and of a dz whose row is far below the smallest normal of 11 bits)
        assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -10 * np.abs(dz) + 5e-6 * scale) @ np.abs(W).T + 1e-38).all()
        if accumulate:
            assert (got[pad] == base).all()
        else:
            assert (got[pad] == 0.0).all()


LAYERS = [
    # T, d, E, k, score, mode, offsets
    (1, 8, 1, 1, SOFTMAX, NONE, None),
    (1, 64, 8, 2, SIGMOID, NONE, [0, 1]),
    (37, 72, 5, 3, SOFTMAX, PRE, [0, 1, 1, 30, 37]),                      # an odd number of experts, an empty sequence
    (256, 256, 8, 2, SOFTMAX, NONE, None),                               # the smallest layer of the workloads
    (300, 200, 20, 3, SIGMOID, PRE, [11, 60, 60, 61, 290]),               # padding on both sides
    (513, 128, 33, 4, SIGMOID, POST, [0, 0, 513, 513]),                   # empty first and last sequences
    (2500, 64, 64, 6, SOFTMAX, NONE, list(range(0, 2501))),               # a sequence for every token
    (2367, 136, 130, 8, SOFTMAX, PRE, [0, 16, 32, 33, 2000, 2300]),       # two vectors a lane, cuts at and beside block borders
    (2368, 64, 256, 8, SIGMOID, POST, [0, 1184, 2368]),
    (700, 64, 384, 8, SIGMOID, NONE, [5, 695]),
    (90, 64, 1000, 32, SOFTMAX, NONE, [0, 40, 90]),
    (64, 64, 1024, 32, SIGMOID, PRE, None),
    (50, 64, 7, 7, SOFTMAX, NONE, [20, 20, 20]),                          # no token belongs to a sequence
    (2000, 64, 3, 2, SIGMOID, NONE, [0, 1000, 1990]),                     # fewer vectors than CTAs that finish a sequence
    (1500, 64, 1001, 4, SOFTMAX, NONE, [0, 0, 700, 1500]),                # an odd number of experts for each of them
    (1300, 64, 600, 4, SOFTMAX, PRE, [13 * i for i in range(100)]),       # many sequences and many experts
]


@pytest.mark.parametrize("T,d,E,k,score,mode,off", LAYERS, ids=lambda v: str(v) if isinstance(v, int) else "")
def test_balance_loss_and_gradients_match_the_oracle(T, d, E, k, score, mode, off):
    c = Case(T, d, E, k, score, mode, off, seed=T + E)
    got = c.forward()
    counts = check_forward(c, got)
    assert counts.sum() == k * (c.bounds[-1] - c.bounds[0])
    again = c.forward()
    assert all(torch.equal(a, b) for a, b in zip(got, again))             # reproducible bit for bit
    for accumulate in (False, True):
        out = c.backward(got[0], c.outputs(0.5), accumulate)
        check_backward(c, out, 0.5, accumulate)
        again = c.backward(got[0], c.outputs(0.5), accumulate)
        assert all(torch.equal(out[n], again[n]) for n in out)
    binding.mop_poll(c.ctx)


@pytest.mark.parametrize("T,d,E,k,score,mode,off", [(37, 72, 5, 3, SOFTMAX, PRE, [0, 1, 1, 30, 37]), (300, 200, 130, 3, SIGMOID, PRE, [11, 60, 60, 61, 290])],
                         ids=lambda v: str(v) if isinstance(v, int) else "")
def test_the_products_on_the_cuda_cores(T, d, E, k, score, mode, off):
    c = Case(T, d, E, k, score, mode, off, seed=T, path=binding.GEMM_SCALAR)
    got = c.forward()
    check_forward(c, got)
    for accumulate in (False, True):
        check_backward(c, c.backward(got[0], c.outputs(0.5), accumulate), 0.5, accumulate)
    out = {"dW_r": c.outputs()["dW_r"]}                                   # (dz in the workspace)
    check_backward(c, c.backward(got[0], out))


@pytest.mark.parametrize("T,d,E,off", [(4100, 328, 72, [70, 4000]),       # ranges of tokens; both edge blocks hold padding; E in one narrow tile
                                       (64 * 40, 512, 300, [64, 64 * 39]),  # edges on block borders; a wide and a narrow tile
                                       (1000, 2064, 256, [130, 150]),      # all tokens inside one block
                                       (5000, 264, 200, [0, 4999])],       # one token of padding
                         ids=lambda v: str(v) if isinstance(v, int) else "")
def test_ranges_of_tokens_that_fit_no_block(T, d, E, off):
    c = Case(T, d, E, 4, SOFTMAX, NONE, off, seed=d)
    got = c.forward()
    check_forward(c, got)
    check_backward(c, c.backward(got[0], c.outputs()))
    check_backward(c, c.backward(got[0], c.outputs(0.5), True), 0.5, True)
    binding.mop_poll(c.ctx)


@pytest.mark.parametrize("which", [("dlogits",), ("dW_r",), ("dX",), ("dbias",), ("dW_r", "dX")], ids="-".join)
def test_each_gradient_alone(which):
    c = Case(150, 72, 20, 3, SIGMOID, PRE, [3, 70, 149], seed=4)
    counts = c.forward()[0]
    every = c.backward(counts, c.outputs())
    out = c.backward(counts, {n: t for n, t in c.outputs().items() if n in which})
    assert all(torch.equal(out[n], every[n]) for n in which)


@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_masked_experts_masked_tokens_and_dropped_picks(score):
    """-inf and the lowest fp32 logit take an expert out, a row of nothing but -inf adds nothing, picks outside the experts do not count."""
    c = Case(200, 64, 24, 4, score, NONE, [0, 100, 200], seed=9)
    c.logits[:, 3] = -float("inf")
    c.logits[:, 7] = torch.finfo(torch.float32).min
    c.logits[50:60] = -float("inf")
    c.idx[10:20] = -1
    c.idx[20:30] = 24
    c.idx[30, :] = 5                                                      # the same expert four times
    got = c.forward()
    check_forward(c, got)
    assert float(got[1][:, 3].abs().max()) == 0.0 and float(got[1][:, 7].abs().max()) == 0.0
    out = c.backward(got[0], c.outputs())
    check_backward(c, out)
    assert float(out["dlogits"][50:60].abs().max()) == 0.0


def test_large_and_tiny_upstream_weights_keep_their_gradients():
    """Row scales of the dX product: weights 10^30 apart in one batch."""
    c = Case(96, 64, 16, 2, SOFTMAX, NONE, [0, 32, 64, 96], seed=12)
    counts = c.forward()[0]
    c.dloss.copy_(torch.tensor([1e-18, 1.0, 1e12]))
    check_backward(c, c.backward(counts, c.outputs()))
    c.dloss.zero_()
    out = c.backward(counts, c.outputs())
    assert all(float(t.abs().max()) == 0.0 for t in out.values())


def test_a_nan_logit_shows_in_its_sequence_only():
    c = Case(128, 64, 12, 2, SIGMOID, NONE, [0, 64, 128], seed=13)
    clean = c.forward()
    c.logits[70, 4] = float("nan")
    got = c.forward()
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1][0], clean[1][0]) and torch.isnan(got[2][1]) and not torch.isnan(got[2][0])
    out = c.backward(got[0], c.outputs())
    assert not torch.isnan(out["dX"][:70].float()).any() and torch.isnan(out["dX"][70].float()).all() and torch.isnan(out["dW_r"]).any()


def test_nearly_balanced_load_keeps_its_digits():
    """Counts within one of each other: the differences that the gradient is made of are a thousandth of the counts."""
    T, E, k = 2048, 16, 8
    c = Case(T, 64, E, k, SOFTMAX, NONE, None, seed=14)
    c.idx = ((torch.arange(T, device="cuda")[:, None] * k + torch.arange(k, device="cuda")[None, :]) % E).to(torch.int32).contiguous()
    c.idx[0, 0] = 9
    got = c.forward()
    check_forward(c, got)
    check_backward(c, c.backward(got[0], c.outputs()))


def test_on_another_stream_and_in_a_replayed_graph():
    c = Case(400, 72, 40, 4, SIGMOID, PRE, [0, 130, 400], seed=21)
    want = c.forward()
    want_b = c.backward(want[0], c.outputs())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.forward(stream=side)
    got_b = c.backward(want[0], c.outputs(), stream=side)
    side.synchronize()
    ws, wb, static = c.workspace(False), c.workspace(True), c.outputs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        counts, prob, loss = c.forward(ws=ws)
        c.backward(counts, static, ws=wb)
    fresh = Case(400, 72, 40, 4, SIGMOID, PRE, [0, 130, 400], seed=22)
    for t, f in ((c.logits, fresh.logits), (c.idx, fresh.idx), (c.x, fresh.x)):
        t.copy_(f)
    graph.replay()
    check_forward(c, (counts, prob, loss))
    check_backward(c, static)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert all(torch.equal(want_b[n], got_b[n]) for n in want_b)


def test_nothing_is_written_outside_the_outputs_and_the_workspace():
    c = Case(301, 200, 21, 3, SOFTMAX, PRE, [0, 100, 290], seed=23)
    margin = 4096

    def fenced(n):
        whole = torch.full((n + 2 * margin,), 0xA5, dtype=torch.uint8, device="cuda")
        return whole, whole[margin:margin + n]
    fences = []

    def out(shape, dtype):
        whole, part = fenced(int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size())
        fences.append((whole, part.numel()))
        return part.view(dtype).view(shape)
    ws = [fenced(binding.mop_moe_balance_workspace_bytes(c.ctx, c.S, b)) for b in (False, True)]
    fences += [(w, p.numel()) for w, p in ws]
    counts, prob, loss = out((c.S, c.E), torch.int32), out((c.S, c.E), torch.float32), out((c.S,), torch.float32)
    binding.mop_moe_balance_loss_fwd(c.ctx, c.logits, c.bias, c.idx, c.offs, counts, prob, loss, ws[0][1])
    grads = {"dlogits": out((c.T, c.E), torch.float32), "dW_r": out((c.d, c.E), torch.float32), "dbias": out((c.E,), torch.float32),
             "dX": out((c.T, c.d), torch.bfloat16)}
    c.backward(counts, grads, ws=ws[1][1])
    check_forward(c, (counts, prob, loss))
    check_backward(c, grads)
    for whole, n in fences:
        assert bool((whole[:margin] == 0xA5).all()) and bool((whole[margin + n:] == 0xA5).all())


def test_refusals():
    c = Case(64, 64, 8, 2, SIGMOID, PRE, [0, 64], seed=31)
    counts, prob, loss = c.forward()
    out, ws = c.outputs(), c.workspace(True)

    def code(fn, *args):
        with pytest.raises(binding.MopError) as e:
            fn(*args)
        return e.value.code
    fwd, bwd = binding.mop_moe_balance_loss_fwd, binding.mop_moe_balance_loss_bwd
    assert code(fwd, c.ctx, c.logits, None, c.idx, c.offs, counts, prob, loss, ws) == 1                 # the context has a bias
    assert code(fwd, c.ctx, c.logits, c.bias, c.idx, c.offs, counts, None, loss, ws) == 1
    assert code(fwd, c.ctx, c.logits, c.bias, c.idx, c.offs, counts, prob, loss, ws[16:]) == 3          # workspace off its 256 bytes
    assert code(fwd, c.ctx, c.logits, c.bias, c.idx, None, counts, prob, loss.expand(2).contiguous(), ws) == 1  # two sequences, no offsets
    args = (c.ctx, c.logits, c.bias, c.offs, counts, c.dloss)
    assert code(bwd, *args, c.x, c.W_r, None, None, None, None, False, ws) == 1                         # nothing asked for
    assert code(bwd, *args, None, c.W_r, None, out["dW_r"], None, None, False, ws) == 1                 # dW_r without x
    assert code(bwd, *args, c.x, None, None, None, None, out["dX"], False, ws) == 1                     # dX without W_r
    assert code(bwd, *args, c.x, c.W_r, None, None, None, out["dX"], 2, ws) == 1
    assert code(bwd, *args, c.x, c.W_r, None, None, out["dbias"][1:], None, False, ws) == 3
    assert binding.mop_moe_balance_workspace_bytes(c.ctx, 0) == 0


def test_no_tokens():
    c = Case(0, 64, 8, 2, SIGMOID, PRE, [0, 0, 0], seed=32)
    counts, prob, loss = c.forward()
    assert int(counts.abs().sum()) == 0 and float(prob.abs().sum()) == 0.0 and float(loss.abs().sum()) == 0.0
    out = c.backward(counts, c.outputs())
    assert float(out["dW_r"].abs().sum()) == 0.0 and float(out["dbias"].abs().sum()) == 0.0
    out = c.backward(counts, c.outputs(), accumulate=True)
    assert bool((out["dW_r"] == 3.0).all()) and bool((out["dbias"] == 3.0).all())


@pytest.mark.parametrize("score,mode", [(SOFTMAX, NONE), (SIGMOID, PRE)], ids=["softmax", "sigmoid-pre"])
def test_a_training_step_of_the_layer_with_the_balance_loss(score, mode):
    """route -> forward -> backward -> router backward -> balance backward, added to the same dW_r and dX: the balance loss's share
    of both against automatic differentiation of the long form."""
    w = synth.small("c1_tiny", T=300, d=256, E=16, k=4, f=128, score_fn=score, bias_mode=mode, bias_std=0.1, backward=True)
    inp = synth.make_inputs(w, "cuda")
    ctx, buf = binding.context_for(w), binding.LayerBuffers(w)
    logits = torch.empty((w.T, w.E), device="cuda")
    binding.forward(ctx, inp, buf)
    binding.mop_moe_route(ctx, inp["x"], inp["W_r"], inp["bias"], buf.idx, buf.gate, logits)
    binding.backward(ctx, inp, buf)
    dW_r, dbias = torch.empty((w.d, w.E), device="cuda"), torch.empty((w.E,), device="cuda")
    off = torch.tensor([0, 120, 300], dtype=torch.int32, device="cuda")
    binding.mop_moe_route_bwd(ctx, logits, inp["bias"], buf.idx, buf.gate, buf.dgate, buf.Xp, buf.offsets, buf.perm_row, inp["W_r"], dW_r,
                              dbias, buf.dX)
    before = [t.double().clone() for t in (dW_r, dbias, buf.dX)]
    counts = torch.empty((2, w.E), dtype=torch.int32, device="cuda")
    prob, loss = torch.empty((2, w.E), device="cuda"), torch.empty((2,), device="cuda")
    ws = torch.empty(max(binding.mop_moe_balance_workspace_bytes(ctx, 2, b) for b in (False, True)), dtype=torch.uint8, device="cuda")
    binding.mop_moe_balance_loss_fwd(ctx, logits, inp["bias"], buf.idx, off, counts, prob, loss, ws)
    assert torch.equal(counts.sum(0, dtype=torch.int32), buf.counts)
    dloss = torch.tensor([40.0, 60.0], device="cuda")
    binding.mop_moe_balance_loss_bwd(ctx, logits, inp["bias"], off, counts, dloss, inp["x"], inp["W_r"], None, dW_r, dbias, buf.dX, True, ws)
    binding.mop_poll(ctx)
    x, W = inp["x"].double().requires_grad_(), inp["W_r"].double().requires_grad_()
    b = (inp["bias"].double() if inp["bias"] is not None else torch.zeros(w.E, device="cuda", dtype=torch.float64)).requires_grad_()
    z = x @ W + (b if mode == PRE else 0.0)
    s = torch.softmax(z, 1) if score == SOFTMAX else torch.sigmoid(z)
    p = s / s.sum(1, keepdim=True)
    total = 0.0
    for i, (lo, hi) in enumerate(((0, 120), (120, 300))):
        want = w.E / (w.k * (hi - lo)) * (counts[i].double() * p[lo:hi].mean(0)).sum()
        assert abs(want.item() - loss[i].item()) < 2e-5 * want.item()
        total = total + dloss[i].double() * want
    total.backward()
    for got, was, grad, step in ((dW_r, before[0], W.grad, 2.0 ** -24), (buf.dX, before[2], x.grad, 2.0 ** -8)):
        assert float(grad.abs().max()) > 0
        # one rounding of the sum to the output's type; the share itself is within 2^-9 (operands of 11 bits) or far better
        assert ((got.double() - was - grad).abs() <= step * (was + grad).abs() + (2.0 ** -9 if step > 1e-6 else 1e-4) * grad.abs().max()).all()
    if mode == PRE:
        assert torch.allclose(dbias.double() - before[1], b.grad, rtol=1e-4, atol=1e-6 * float(before[1].abs().max()))


def test_logits_beyond_31_bits():
    """T E > 2^31: counts and means of everything, gradients of the last rows and dW_r of everything, against fp64 on the device."""
    T, E, d = (1 << 21) + 4100, 1024, 64
    ctx = binding.Context(T, d, E, 1, 64, SIGMOID, NONE)
    g = torch.Generator(device="cuda").manual_seed(40)
    logits = torch.empty((T, E), device="cuda").normal_(generator=g)
    idx = torch.randint(0, E, (T, 1), generator=g, device="cuda", dtype=torch.int32)
    x = torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16)
    W_r = torch.randn((d, E), generator=g, device="cuda") * 0.05
    offs = torch.tensor([0, T - 3000, T], dtype=torch.int32, device="cuda")
    counts = torch.empty((2, E), dtype=torch.int32, device="cuda")
    prob, loss = torch.empty((2, E), device="cuda"), torch.empty((2,), device="cuda")
    ws = torch.empty(max(binding.mop_moe_balance_workspace_bytes(ctx, 2, b) for b in (False, True)), dtype=torch.uint8, device="cuda")
    binding.mop_moe_balance_loss_fwd(ctx, logits, None, idx, offs, counts, prob, loss, ws)
    dloss = torch.tensor([3000.0, 1.0], device="cuda")
    dW, dX = torch.empty((d, E), device="cuda"), torch.empty((T, d), device="cuda", dtype=torch.bfloat16)
    binding.mop_moe_balance_loss_bwd(ctx, logits, None, offs, counts, dloss, x, W_r, None, dW, None, dX, False, ws)
    binding.mop_poll(ctx)
    total, want_dW, terms = torch.zeros(E, device="cuda", dtype=torch.float64), torch.zeros((d, E), device="cuda", dtype=torch.float64), 0.0
    for s, (a, b) in enumerate(((0, T - 3000), (T - 3000, T))):
        assert torch.equal(counts[s], torch.bincount(idx[a:b, 0].long(), minlength=E).to(torch.int32))
        c = dloss[s].double() * E / float(b - a) ** 2 * counts[s].double()
        total.zero_()
        for r in range(a, b, 1 << 17):
            z = torch.sigmoid(logits[r:min(b, r + (1 << 17))].double())
            p = z / z.sum(1, keepdim=True)
            total += p.sum(0)
            dz = p * (1 - z) * (c - (p * c).sum(1, keepdim=True))
            xs = x[r:min(b, r + (1 << 17))].double()
            want_dW += xs.T @ dz
            terms = terms + xs.abs().T @ (dz.abs() + p * (c - c.mean()).abs())
        # (7100 tokens a block, 444 for a warp of its sixteen, 296 blocks over four slices: 444 + 16 + 74 + 4 half steps at most)
        assert float((prob[s].double() * (b - a) / total - 1).abs().max()) <= 538 * 2.0 ** -24 + 1.5e-6
        want = (dz @ W_r.double().T)[-3000:]
        got = dX[b - want.shape[0]:b].double()
        assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -9 * (dz[-3000:].abs() @ W_r.double().abs().T)).all())
    assert bool(((dW.double() - want_dW).abs() <= 1e-5 * terms).all())
