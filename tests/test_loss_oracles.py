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


def _distill_inputs(N=9, H=6, V=23, K=5, seed=4):
    rng = np.random.default_rng(seed)
    X, W = synth.bits(torch.from_numpy(rng.normal(size=(N, H))).to(torch.bfloat16)), synth.bits(torch.from_numpy(rng.normal(size=(H, V))).to(torch.bfloat16))
    ids = rng.integers(0, V, size=(N, K))
    t = rng.normal(size=(N, K)) * 3
    ids[1, 2:] = -1                                  # a short list
    ids[2] = V                                       # none at all
    ids[3, 1] = ids[3, 0]                            # a place that is named twice
    t[4, 0] = -np.inf
    return X, W, ids, t


@pytest.mark.parametrize("full", [False, True], ids=["renormalised", "whole"])
@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_distillation_against_autodiff_of_the_divergence(tau, full):
    X, W, ids, t = _distill_inputs()
    V = W.shape[1]
    dloss = np.linspace(-1, 2, X.shape[0])
    tlse = np.log(np.exp(np.where(np.isfinite(t), t, -50) / tau).sum(1) + 3.0) if full else None
    Y = torch.as_tensor(oracle.bf16_bits_to_f64(X) @ oracle.bf16_bits_to_f64(W)).requires_grad_()
    logp = torch.log_softmax(Y / tau, 1)
    want = []
    for n in range(X.shape[0]):
        keep = [k for k in range(ids.shape[1]) if 0 <= ids[n, k] < V]
        s = torch.as_tensor(t[n, keep] / tau)
        logq = s - (torch.as_tensor(tlse[n]) if full else torch.logsumexp(s, 0)) if keep else s
        q = torch.exp(logq)
        want.append(sum((q[i] * (logq[i] - logp[n, ids[n, k]]) for i, k in enumerate(keep) if q[i] > 0), torch.zeros((), dtype=torch.float64)))
    want = torch.stack(want)
    (want * torch.as_tensor(dloss)).sum().backward()
    loss, student, lse = oracle.vocab_distill(X, W, ids, t, tau, tlse)
    assert np.allclose(loss, want.detach().numpy(), rtol=1e-12, atol=1e-13) and loss[2] == 0.0 and (full or (loss >= -1e-13).all())
    assert np.allclose(lse, torch.logsumexp(Y / tau, 1).detach().numpy())
    assert np.allclose(student[0], Y[0].detach().numpy()[ids[0]]) and (student[1, 2:] == 0).all()
    dY = oracle.vocab_distill_dlogits(X, W, ids, t, tau, dloss, tlse)
    assert np.allclose(dY, Y.grad.numpy(), rtol=1e-10, atol=1e-14) and (dY[2] == 0).all()


def test_distillation_gradient_against_differences():
    _, _, ids, t = _distill_inputs()
    rng = np.random.default_rng(8)
    Y, h, tau = rng.normal(size=(9, 23)), 1e-6, 1.7
    eye = synth.bits(torch.eye(23).to(torch.bfloat16))

    def total(Y):                                     # (the projection is not what is differentiated: X = Y, W = 1)
        valid, q, logq = oracle._teacher(ids, t, tau, 23, None)
        logp = Y / tau - np.log(np.exp(Y / tau).sum(1, keepdims=True))
        return np.where(q > 0, q * (np.where(q > 0, logq, 0) - np.take_along_axis(logp, np.where(valid, ids, 0), 1)), 0).sum()
    Yb = synth.bits(torch.from_numpy(Y).to(torch.bfloat16))
    Y = oracle.bf16_bits_to_f64(Yb)
    dY = oracle.vocab_distill_dlogits(Yb, eye, ids, t, tau, np.ones(9))
    for n, v in ((0, int(ids[0, 0])), (3, int(ids[3, 0])), (5, 11), (2, 4)):
        up, down = Y.copy(), Y.copy()
        up[n, v] += h
        down[n, v] -= h
        assert abs((total(up) - total(down)) / (2 * h) - dY[n, v]) < 1e-8
