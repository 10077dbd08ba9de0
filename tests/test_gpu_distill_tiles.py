"""Distillation: every tile width over more than one round of the SMs, and what one bf16 piece of the logit gradients costs, against fp64 on
the device.

Bounds.  A logit is summed on the tensor cores in segments of 512 of H, 32 steps of 16: each step drops up to 2^-23 of the sum so far, and
adding a segment in fp32 is off by 2^-24 of it: (33 + ceil(H / 512) / 2) 2^-23 of A = sum |x| |w| at most, with as many steps as H has where
that is less.  The backward forms the logits again in one sum of ceil(H / 16) steps.  lse takes over the largest error of its logits (over
the temperature), 4e-6 for the exponentials and their sum, 2^-22 of itself for the logarithm and the product that scales it.
dY = dloss / tau (Q p - q) is off by what its two terms are: both logit errors, those of lse, 2^-22 of the logits and lse for the scaled
arguments, 6e-6 for the exponentials of p and q and the products around them; then by its rounding, 2^-8 of it with one bf16 piece and 2^-16 with two.  dX and dW add such terms, dropping 2^-23 of
the sum per step of 16 of their K, and are rounded once (2^-8)."""
import pytest
import torch

from test_gpu_distill import backward, forward, inputs

from paper_2607_01844_b200 import binding

pytestmark = pytest.mark.gpu

# N, H, V, K: columns of the forward's tile, rounds of the SMs (of the 74 pairs above 128 tokens)
TILES = {
    (3, 64, 9472, 20): (128, 1),
    (65, 128, 18936, 20): (128, 1),
    (64, 264, 28352, 31): (192, 1),
    (60, 72, 37896, 9): (192, 2),             # rows of half a tile
    (90, 72, 50304, 40): (192, 2),
    (100, 136, 44608, 126): (192, 2),         # many entries: some rows have more than eight in a tile
    (90, 64, 84000, 9): (192, 3),
    (64, 72, 75776, 20): (256, 2),
    (90, 72, 57000, 9): (256, 2),
    (200, 72, 28000, 33): (128, 3),           # pairs
    (257, 72, 19144, 9): (256, 3),
    (40, 4104, 1000, 12): (128, 1),           # nine segments of H
    (140, 4104, 1000, 12): (128, 1),
}


def steps(n):
    return -(-n // 16)


def logit_bounds(H):
    """Of the forward and of the logits formed again, relative to sum |x| |w|."""
    return (min(32, steps(H)) + 1 + -(-H // 512) / 2) * 2.0 ** -23, (steps(H) + 1) * 2.0 ** -23


class Reference:
    def __init__(self, X, W, ids, t, tau, dloss):
        N, V, H = X.shape[0], W.shape[1], X.shape[1]
        self.x, self.w = X.double(), W.double()
        valid = (ids >= 0) & (ids < V)
        at = torch.where(valid, ids, 0).long()
        Y, A = self.x @ self.w, (self.x.abs() @ self.w.abs()).amax(1, keepdim=True)
        self.lse = torch.logsumexp(Y / tau, 1)
        q = torch.where(valid, torch.softmax(torch.where(valid, t.double() / tau, -float("inf")), 1), 0.0).nan_to_num(0.0)
        picked = torch.where(valid, Y.gather(1, at), 0.0)
        logq = torch.where(q > 0, q.log(), 0.0)
        self.student, self.loss = picked, (q * (logq - picked / tau + self.lse[:, None])).sum(1)
        fwd, again = logit_bounds(H)
        self.student_tol = fwd * A
        self.lse_tol = (fwd * A / tau)[:, 0] + 4e-6 + 2.0 ** -22 * self.lse.abs()
        size = q * (logq.abs() + picked.abs() / tau + self.lse.abs()[:, None])
        self.loss_tol = q.sum(1) * (self.lse_tol + (fwd * A / tau)[:, 0]) + 3e-6 * size.sum(1)
        p = torch.exp(Y / tau - self.lse[:, None]) * q.sum(1, keepdim=True)
        g = dloss.double()[:, None] / tau
        far = self.lse.abs() + Y.abs().amax(1) / tau
        off = self.lse_tol[:, None] + again * A / tau + 6e-6 + 2.0 ** -22 * far[:, None]
        self.size = p.scatter_add(1, at, q) * g.abs() * off         # what dY is off by before its rounding
        self.dY = p.scatter_add(1, at, -q) * g
        self.piece = 2.0 ** -16 if N <= 128 else 2.0 ** -8

    def check_forward(self, loss, student, lse):
        assert bool(((student.double() - self.student).abs() <= self.student_tol).all())
        assert bool(((lse.double() - self.lse).abs() <= self.lse_tol).all())
        assert bool(((loss.double() - self.loss).abs() <= self.loss_tol).all())

    def check_backward(self, dX, dW):
        dY, x, w = self.dY, self.x, self.w
        for got, want, terms, base, k in ((dX, dY @ w.T, dY.abs() @ w.abs().T, self.size @ w.abs().T, w.shape[1]),
                                          (dW, x.T @ dY, x.abs().T @ dY.abs(), x.abs().T @ self.size, 2 * x.shape[0])):
            bound = 2.0 ** -8 * want.abs() + (self.piece + steps(k) * 2.0 ** -23) * terms + (1 + 2.0 ** -7) * base + 1e-30
            assert bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("N,H,V,K", TILES, ids=lambda v: str(v))
def test_tiles_of_every_width_in_several_rounds(N, H, V, K):
    X, W, ids, t, dloss = inputs(N, H, V, K, seed=V, spread=0.02 if K > 100 else 1.0)
    ids[0, 0], ids[-1, -1] = 0, V - 1
    ref = Reference(X, W, ids, t, 1.5, dloss)
    loss, student, lse, ws = forward(X, W, ids, t, 1.5)
    binding.mop_vocab_poll(0, ws)
    ref.check_forward(loss, student, lse)
    dX, dW, ws = backward(X, W, ids, t, 1.5, student, lse, dloss)
    binding.mop_vocab_poll(0, ws)
    ref.check_backward(dX, dW)


@pytest.mark.parametrize("few", [False, True], ids=["every-token", "three-tokens"])
@pytest.mark.parametrize("K", [5, 64])
@pytest.mark.parametrize("N", [128, 129, 300, 2000])
def test_rows_of_dX_with_one_and_two_pieces_of_the_logit_gradients(N, K, few):
    """A row of dX is a sum over the vocabulary of its own token's dY, so its error has nothing to average out against, whatever the number of
    tokens: with one piece the roundings, 2^-8 of each dY at most, make up to 2^-8 sqrt(sum_v dY^2 |w_v|^2) where the columns w_v are
    uncorrelated, half as much again allowed for those that are; with two it is the rounding of dX itself.  Tokens whose upstream weight
    is zero have no gradient at all."""
    X, W, ids, t, dloss = inputs(N, 256, 4096, K, seed=N + K)
    if few:
        keep = torch.tensor([1, N // 2, N - 1], device="cuda")
        dloss = torch.zeros_like(dloss).index_copy_(0, keep, dloss[keep] + 2.0)
    ref = Reference(X, W, ids, t, 1.0, dloss)
    _, student, lse, _ = forward(X, W, ids, t, 1.0)
    dX, dW, _ = backward(X, W, ids, t, 1.0, student, lse, dloss)
    ref.check_backward(dX, dW)
    want = ref.dY @ ref.w.T
    err = (dX.double() - want).norm(dim=1)
    spread = (ref.dY.square() @ ref.w.square().sum(0)).sqrt()
    small = (ref.size @ ref.w.abs().T).norm(dim=1) + (steps(4096) * 2.0 ** -23 + 2.0 ** -16) * (ref.dY.abs() @ ref.w.abs().T).norm(dim=1)
    pieces = 1.5 * spread if N > 128 else 0.0
    assert bool((err <= 2.0 ** -8 * (want.norm(dim=1) + pieces) + 1.01 * small).all())
    if few:
        rest = torch.ones(N, dtype=torch.bool, device="cuda")
        rest[keep] = False
        assert float(dX[rest].abs().max()) == 0.0
    once = (want.to(torch.bfloat16).double() - want).norm(dim=1)
    print(f"N {N}, K {K}, few {few}: rows of dX {float((err / once)[once > 0].max()):.2f} times rounding once, "
          f"all {float(err.norm() / once.norm()):.2f}")
