"""The residual gated block's operators as programs call them: in graphs beside other calls, on streams of their
own, in place, and at the ends of what they accept. Tolerances are those of test_gpu_blocks.py unless one is given."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_blocks import block_inputs, blocks, norm_inputs, normal, rng, run_block, run_norm  # noqa: E402


# ----------------------------------------------------------------------------- graphs
def replayed(call, larger):
    """What a graph of call() gives on three replays, with calls that outgrow the handle's workspace between capture
    and replay, and the memory that they left behind written over."""
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call()
    for rows in (1, 2, 3):
        larger(rows)
        torch.cuda.synchronize()
        filled = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(8)]
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        del filled
        yield [o.clone() for o in outs]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_block_graph_outlives_larger_calls(dtype):
    t = block_inputs(70, 128, 256, dtype, 6)
    big = [block_inputs(n, 128, 256, dtype, n) for n in (700, 3000, 5000)]
    op = blocks.GatedBlock(128, 256, dtype=dtype)
    want = run_block(op, *t)
    for got in replayed(lambda: run_block(op, *t), lambda n: run_block(op, *big[n - 1])):
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_norm_graph_outlives_larger_calls():
    t, d = norm_inputs(60, 1000, "f32", 7, 20)
    big = [norm_inputs(n, 1000, "f32", n, 20) for n in (2000, 9000, 30000)]
    op = blocks.ResidualNorm(1000, dtype="f32", norm="layer", group=20)
    want = run_norm(op, t, d)
    for got in replayed(lambda: list(run_norm(op, t, d).values()), lambda n: run_norm(op, *big[n - 1])):
        assert all(torch.equal(a, b) for a, b in zip(got, want.values()))


def test_int8_graph_outlives_larger_calls():
    g = rng(8)
    codes, scales = blocks.quantize_weight(normal(g, 96, 500).float().cuda())
    x = normal(g, 6000, 500).float().cuda()
    op = blocks.Int8Linear(codes, scales, dtype="f32")
    want = op(x[:80])
    for got in replayed(lambda: [op(x[:80])], lambda n: op(x[:2000 * n])):
        assert torch.equal(got[0], want)
