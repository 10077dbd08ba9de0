"""Pins of the oracle's auxiliary losses: against automatic differentiation of the long form in fp64, differences, and hand-worked cases."""
import numpy as np
import pytest
import torch

import oracle
from paper_2607_01844_b200 import synth

MODES = [(synth.SCORE_SOFTMAX, synth.BIAS_NONE), (synth.SCORE_SOFTMAX, synth.BIAS_PRE_LOGIT), (synth.SCORE_SIGMOID, synth.BIAS_NONE),
         (synth.SCORE_SIGMOID, synth.BIAS_POST_SCORE), (synth.SCORE_SIGMOID, synth.BIAS_PRE_LOGIT)]


def long_form_balance(z, bias, k, score_fn, bias_mode, counts, off):
    """sum over the sequences' losses, as torch operations on z (and the bias) in fp64."""
    if bias_mode == synth.BIAS_PRE_LOGIT:
        z = z + bias
    p = torch.softmax(z, 1) if score_fn == synth.SCORE_SOFTMAX else torch.sigmoid(z) / torch.sigmoid(z).sum(1, keepdim=True)
    out = []
    for s in range(len(off) - 1):
        n = off[s + 1] - off[s]
        f = torch.as_tensor(counts[s], dtype=torch.float64) / max(1, k * n)
        out.append(z.shape[1] * (f * p[off[s]:off[s + 1]].sum(0) / max(1, n)).sum())
    return torch.stack(out)


@pytest.mark.parametrize("score_fn,bias_mode", MODES)
def test_balance_loss_and_gradient_against_autodiff(score_fn, bias_mode):
    T, E, k, off = 23, 7, 3, [2, 9, 9, 20]
    g = torch.Generator().manual_seed(3)
    z = torch.randn((T, E), generator=g, dtype=torch.float64, requires_grad=True)
    bias = (torch.randn(E, generator=g, dtype=torch.float64) * 0.3).requires_grad_(bias_mode == synth.BIAS_PRE_LOGIT)
    idx = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)]).numpy()
    dloss = np.array([0.7, -1.3, 2.0])
    counts, prob, loss = oracle.balance_loss(z.detach().numpy(), bias.detach().numpy(), k, score_fn, bias_mode, idx, off)
    assert counts.sum(1).tolist() == [k * 7, 0, k * 11] and np.allclose(prob.sum(1), [1, 0, 1])
    want = long_form_balance(z, bias, k, score_fn, bias_mode, counts, off)
    assert np.allclose(loss, want.detach().numpy(), rtol=1e-13)
    (want * torch.as_tensor(dloss)).sum().backward()
    dz = oracle.balance_loss_bwd(z.detach().numpy(), bias.detach().numpy(), k, score_fn, bias_mode, counts, off, dloss)
    assert np.allclose(dz, z.grad.numpy(), rtol=1e-10, atol=1e-15)
    if bias_mode == synth.BIAS_PRE_LOGIT:
        assert np.allclose(dz.sum(0), bias.grad.numpy(), rtol=1e-10, atol=1e-15)


def test_balance_loss_is_one_under_a_perfect_balance_and_its_gradient_zero():
    T, E, k = 12, 6, 2
    idx = np.array([[(2 * t) % E, (2 * t + 1) % E] for t in range(T)])
    z = np.zeros((T, E))
    counts, prob, loss = oracle.balance_loss(z, None, k, synth.SCORE_SOFTMAX, synth.BIAS_NONE, idx, [0, T])
    assert (counts == T * k // E).all() and np.allclose(prob, 1 / E) and np.allclose(loss, 1.0)
    # (1/6 is rounded: six of them add up to 1 within 6 half steps of 2^-53; times c = 1/12 and p = 1/6)
    assert np.abs(oracle.balance_loss_bwd(z, None, k, synth.SCORE_SOFTMAX, synth.BIAS_NONE, counts, [0, T], [1.0])).max() < 1e-16


def test_balance_gradient_against_differences():
    T, E, k, off, h = 9, 5, 2, [0, 4, 9], 1e-6
    rng = np.random.default_rng(1)
    z = rng.normal(size=(T, E))
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    for score_fn in (synth.SCORE_SOFTMAX, synth.SCORE_SIGMOID):
        counts, _, _ = oracle.balance_loss(z, None, k, score_fn, synth.BIAS_NONE, idx, off)
        dz = oracle.balance_loss_bwd(z, None, k, score_fn, synth.BIAS_NONE, counts, off, [1.0, 1.0])
        for t, e in ((0, 0), (3, 4), (4, 2), (8, 1)):
            up, down = z.copy(), z.copy()
            up[t, e] += h
            down[t, e] -= h
            num = (oracle.balance_loss(up, None, k, score_fn, synth.BIAS_NONE, idx, off)[2].sum() -
                   oracle.balance_loss(down, None, k, score_fn, synth.BIAS_NONE, idx, off)[2].sum()) / (2 * h)
            assert abs(num - dz[t, e]) < 1e-8


def test_masked_experts_and_tokens_add_nothing():
    z = np.zeros((3, 4))
    z[0, 1:] = -np.inf
    z[1] = -np.inf
    for score_fn in (synth.SCORE_SOFTMAX, synth.SCORE_SIGMOID):
        counts, prob, _ = oracle.balance_loss(z, None, 1, score_fn, synth.BIAS_NONE, np.array([[0], [-1], [9]]), [0, 3])
        assert counts.tolist() == [[1, 0, 0, 0]]
        assert np.allclose(prob, np.array([1.25, 0.25, 0.25, 0.25]) / 3)
        assert np.isfinite(oracle.balance_loss_bwd(z, None, 1, score_fn, synth.BIAS_NONE, counts, [0, 3], [1.0])).all()
