"""The vocabulary projection's calls where the workspace, the stream or the batch is out of the ordinary."""
import pytest
import torch

from paper_2607_01844_b200 import binding

pytestmark = pytest.mark.gpu


def test_a_poll_after_a_call_without_tokens_finds_nothing():
    """Whatever the workspace held: a caller's fresh memory, or the word of an earlier call whose wait ran out."""
    H, V, K = 64, 128, 3
    bf = dict(device="cuda", dtype=torch.bfloat16)
    f32 = dict(device="cuda", dtype=torch.float32)
    X, W, none = torch.empty((0, H), **bf), torch.randn((H, V), device="cuda").to(torch.bfloat16), torch.empty((0,), **f32)
    ids, t = torch.empty((0, K), device="cuda", dtype=torch.int32), torch.empty((0, K), **f32)
    targets = torch.empty((0,), device="cuda", dtype=torch.int32)
    dX, dW = torch.empty((0, H), **bf), torch.full((H, V), 3.0, **bf)
    dW32 = torch.full((H, V), 3.0, **f32)
    ws = torch.empty((4096,), device="cuda", dtype=torch.uint8)
    for call in (lambda: binding.mop_vocab_distill_fwd(0, X, W, ids, t, 1.0, none, t, none, None, ws),
                 lambda: binding.mop_vocab_distill_bwd(0, X, W, ids, t, 1.0, t, none, none, dX, dW, None, ws),
                 lambda: binding.mop_vocab_loss_fwd(0, X, W, targets, none, none, ws),
                 lambda: binding.mop_vocab_loss_bwd(0, X, W, targets, none, none, dX, dW32, ws)):
        ws.fill_(0xFF)
        call()
        binding.mop_vocab_poll(0, ws)
    assert float(dW.abs().max()) == 0.0 and float(dW32.abs().max()) == 0.0
