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


def vocab_calls(stream):
    """The four calls with a workspace of their own, on `stream`; each returns it."""
    N, H, V, K = 300, 64, 1024, 5
    g = torch.Generator(device="cuda").manual_seed(1)
    X = torch.randn((N, H), generator=g, device="cuda").to(torch.bfloat16)
    W = torch.randn((H, V), generator=g, device="cuda").to(torch.bfloat16)
    ids = torch.randint(0, V, (N, K), generator=g, device="cuda", dtype=torch.int32)
    t, f = torch.randn((N, K), generator=g, device="cuda"), torch.zeros((N,), device="cuda")
    loss, lse, student = torch.zeros_like(f), torch.zeros_like(f), torch.zeros_like(t)
    targets, dX, dW, dW32 = ids[:, 0].contiguous(), torch.empty_like(X), torch.empty_like(W), torch.empty((H, V), device="cuda")
    yield lambda: binding.mop_vocab_distill_fwd(0, X, W, ids, t, 1.0, loss, student, lse, None, None, stream)
    yield lambda: binding.mop_vocab_distill_bwd(0, X, W, ids, t, 1.0, student, lse, f, dX, dW, None, None, stream)
    yield lambda: binding.mop_vocab_loss_fwd(0, X, W, targets, loss, lse, None, stream)
    yield lambda: binding.mop_vocab_loss_bwd(0, X, W, targets, lse, f, dX, dW32, None, stream)


@pytest.mark.parametrize("raw", [False, True], ids=["stream", "handle"])
def test_a_default_workspace_belongs_to_the_stream_of_the_call(raw):
    """Dropped while the call is in flight, it is not handed to an allocation of the current stream, but to the call's next one."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for call in vocab_calls(side.cuda_stream if raw else side):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        workspace = call()
        at, size = workspace.data_ptr(), workspace.numel()
        del workspace
        here = [torch.empty((size,), dtype=torch.uint8, device="cuda") for _ in range(4)]
        assert at not in [t.data_ptr() for t in here]
        with torch.cuda.stream(side):
            assert torch.empty((size,), dtype=torch.uint8, device="cuda").data_ptr() == at
    side.synchronize()


def test_calls_that_overlap_on_two_streams():
    """Two sequences of the losses' calls at once, each with a context, workspaces and outputs of its own: the same bits as one after the
    other.  Replayed graphs that share their workspaces, one behind the other on a stream, give them too."""
    from test_gpu_balance import SIGMOID, Case
    from test_gpu_balance import PRE

    def job(i):
        c = Case(1500 + 64 * i, 264, 40, 4, SIGMOID, PRE, [5, 700, 1400], seed=i)
        g = torch.Generator(device="cuda").manual_seed(i)
        N, H, V, K = (100, 300)[i], 264, 8192 + 520, 20
        X = torch.randn((N, H), generator=g, device="cuda").to(torch.bfloat16)
        W = (torch.randn((H, V), generator=g, device="cuda") * 0.1).to(torch.bfloat16)
        ids = torch.randint(0, V, (N, K), generator=g, device="cuda", dtype=torch.int32)
        t, dloss = torch.randn((N, K), generator=g, device="cuda"), torch.randn((N,), generator=g, device="cuda")
        wf, wb = c.workspace(False), c.workspace(True)
        df = torch.empty(binding.mop_vocab_distill_workspace_bytes(N, H, V, K), dtype=torch.uint8, device="cuda")
        db = torch.empty(binding.mop_vocab_distill_bwd_workspace_bytes(N, H, V, K), dtype=torch.uint8, device="cuda")

        def run():
            fwd = c.forward(ws=wf)
            out = c.backward(fwd[0], c.outputs(0.5), True, ws=wb)
            loss, lse, student = torch.empty((N,), device="cuda"), torch.empty((N,), device="cuda"), torch.empty((N, K), device="cuda")
            dX, dW = torch.empty_like(X), torch.empty_like(W)
            binding.mop_vocab_distill_fwd(0, X, W, ids, t, 1.0, loss, student, lse, None, df)
            binding.mop_vocab_distill_bwd(0, X, W, ids, t, 1.0, student, lse, dloss, dX, dW, None, db)
            return [*fwd, *out.values(), loss, lse, student, dX, dW]
        return run
    jobs = [job(0), job(1)]
    want = [run() for run in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(10):
        got = []
        for run, stream in zip(jobs, streams):
            with torch.cuda.stream(stream):
                got.append(run())
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x.nan_to_num(), y.nan_to_num()) for x, y in zip(a, b))
    graphs = []
    for run in (jobs[0], jobs[0]):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, run()))
    for graph, out in graphs * 3:
        graph.replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        assert all(torch.equal(x.nan_to_num(), y.nan_to_num()) for x, y in zip(want[0], out))
