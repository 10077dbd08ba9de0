"""Load-balance loss of the router: rows of logits, padding and router weights at the ends of their ranges, against the fp64 oracle with
the bounds of test_gpu_balance.py."""
import numpy as np
import pytest
import torch

from paper_2607_01844_b200 import synth
from test_gpu_balance import Case, check_backward, check_forward

pytestmark = pytest.mark.gpu

SOFTMAX, SIGMOID = synth.SCORE_SOFTMAX, synth.SCORE_SIGMOID
NONE, POST, PRE = synth.BIAS_NONE, synth.BIAS_POST_SCORE, synth.BIAS_PRE_LOGIT


class FarCase(Case):
    """Rows whose probabilities leave fp32's normal range.  There p is off by 2^-126 at most (it may be flushed to zero), and so is each of
    the three products behind it in dz = w p (1 - s) (c - m), where |c - m| is at most twice the largest count C: 2^-126 (2 |w| C + 2 C + 2)
    in all, besides what is relative to the result."""

    def dz_scale(self, counts):
        C = np.abs(counts).max()
        w = max(abs(float(self.dloss[s])) * self.E / (self.k * max(1, self.bounds[s + 1] - self.bounds[s]) ** 2) for s in range(self.S))
        return super().dz_scale(counts) + 2.0 ** -126 * (2 * w * C + 2 * C + 2) / 5e-6


@pytest.mark.parametrize("T,E,k,mode,off", [(150, 5, 2, NONE, [0, 60, 150]), (301, 24, 4, PRE, [7, 100, 290]), (150, 64, 6, POST, None),
                                            (90, 130, 8, NONE, [0, 90]), (64, 1000, 4, PRE, None)], ids=lambda v: str(v) if isinstance(v, int) else "")
def test_sigmoid_scores_of_rows_far_below_zero(T, E, k, mode, off):
    """p is a quotient of sigmoids, and stays one where they are below every fp32 number: rows around -20 to -600, some with masked
    experts, beside ordinary ones in the same warp.  (Logits and biases are multiples of 2^-8: their sum has no rounding of its own, which
    at -600 would be 2^-15 of the score.)"""
    c = FarCase(T, 64, E, k, SIGMOID, mode, off, seed=E)
    for t in (c.logits, c.bias):
        if t is not None:
            t.mul_(256).round_().div_(256)
    at = torch.tensor([0.0, -20.0, -60.0, -86.0, -89.0, -95.0, -104.0, -150.0, -600.0], device="cuda")
    c.logits += at[torch.arange(T, device="cuda") % 9][:, None]
    c.logits[::2, 1] = -float("inf")
    c.logits[3::11, 2] = 4.0                              # one expert near, the others far
    c.logits[c.pad] = float("nan")
    got = c.forward()
    assert all(bool(torch.isfinite(t).all()) for t in got)
    check_forward(c, got)
    check_backward(c, c.backward(got[0], c.outputs()))


def test_sigmoid_scores_of_a_row_of_the_lowest_logits():
    """Equal logits get equal scores, also at fp32's lowest value, and nothing but -inf gets none."""
    c = Case(40, 64, 24, 3, SIGMOID, NONE, [0, 20, 40], seed=2)
    c.logits[:20] = torch.finfo(torch.float32).min
    c.logits[20:] = -float("inf")
    _, prob, loss = c.forward()
    assert float((prob[0] * 24 - 1).abs().max()) <= 1.3e-5 and abs(float(loss[0]) - 1) <= 2.6e-5
    assert float(prob[1].abs().max()) == 0.0 and float(loss[1]) == 0.0


PADDED = [(300, 200, 20, [11, 60, 60, 61, 290]), (700, 72, 40, [130, 140]), (513, 264, 130, [0, 512]), (600, 64, 8, [300, 300]),
          (2400, 1032, 64, [700, 1100, 1700])]       # whole tiles of padding among the others


@pytest.mark.parametrize("T,d,E,off", PADDED, ids=lambda v: str(v) if isinstance(v, int) else "")
def test_accumulating_leaves_rows_of_padding_to_the_bit(T, d, E, off):
    """dX of padding tokens may hold anything, NaN of any pattern among it."""
    c = Case(T, d, E, 3, SIGMOID, PRE, off, seed=T)
    counts = c.forward()[0]
    out = c.outputs(0.5)
    bits = torch.randint(-32768, 32768, (T, d), device="cuda", dtype=torch.int32).to(torch.int16)
    bits[:, ::5] = 0x7F81                                 # a signalling NaN
    bits[:, 1::5] = -1                                    # a negative one with every bit set
    raw = out["dX"].view(torch.int16)
    raw[c.pad] = bits[c.pad]
    c.backward(counts, out, True)
    assert torch.equal(raw[c.pad], bits[c.pad])
    raw[c.pad] = c.outputs(0.5)["dX"].view(torch.int16)[c.pad]
    check_backward(c, out, 0.5, True)


@pytest.mark.parametrize("T,d,E,off", PADDED, ids=lambda v: str(v) if isinstance(v, int) else "")
@pytest.mark.parametrize("value", [float("inf"), float("nan")], ids=["inf", "nan"])
def test_router_weights_that_are_not_finite_leave_padding_alone(T, d, E, off, value):
    c = Case(T, d, E, 3, SIGMOID, PRE, off, seed=T)
    c.W_r[5, 1] = value
    counts = c.forward()[0]
    out = c.backward(counts, c.outputs())
    assert float(out["dX"][c.pad].abs().max()) == 0.0
    kept = c.outputs(0.5)
    c.backward(counts, kept, True)
    assert bool((kept["dX"][c.pad] == 0.5).all())
    inside = out["dX"][~c.pad].float()
    assert not torch.isfinite(inside[:, 5]).any() or inside.numel() == 0


@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")], ids=["inf", "minus-inf", "nan"])
def test_a_router_weight_that_is_not_finite_shows_in_its_column_of_dX_only(value):
    """A column of dX is one row of W_r; the rows that share its scale keep their digits."""
    c = Case(200, 136, 24, 4, SOFTMAX, NONE, [0, 90, 200], seed=8)
    counts = c.forward()[0]
    c.W_r[37, 3] = 0.0
    want = c.backward(counts, c.outputs())["dX"]
    c.W_r[37, 3] = value
    got = c.backward(counts, c.outputs())["dX"]
    other = torch.arange(136, device="cuda") != 37
    assert torch.equal(got[:, other], want[:, other]) and not torch.isfinite(got[:, 37]).any()
