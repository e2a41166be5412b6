"""The residual gated block's operators as programs call them: in graphs beside other calls, on streams of their
own, in place, and at the ends of what they accept. Tolerances are those of test_gpu_blocks.py unless one is given."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2407_09486_amd import binding  # noqa: E402
from test_gpu_blocks import (act64, adam64, adam_inputs, block64, block_inputs, blocks, close, norm_inputs, normal, rng,  # noqa: E402
                             run_block, run_norm)


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


# ----------------------------------------------------------------------------- streams
def stream_of(t):
    """The stream whose memory pool holds a tensor."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not of torch's allocator")


def on_both(call):
    """call(stream)'s tensors on torch's current stream and on one given; the latter have to belong to it."""
    want = call(None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.empty(1 << 26, device="cuda")
    for _ in range(20):
        busy.normal_()                         # the current stream is behind
    got = call(side)
    side.synchronize()
    assert all(stream_of(t) == side.cuda_stream for t in got)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()


def test_block_results_belong_to_the_stream_given():
    t = block_inputs(700, 256, 384, "bf16", 4)
    op = blocks.GatedBlock(256, 384)

    def call(stream):
        y, kept = op.forward(*t[:4], save=True, stream=stream)
        return [y, kept, *op.backward(*t[:4], t[4], kept, stream=stream), op.saved(300, stream=stream)]

    def without_the_rest(stream):
        y, kept, *grads = call(stream)[:-1]
        return [y, *grads]

    on_both(without_the_rest)
    side = torch.cuda.Stream()
    assert all(stream_of(a) == side.cuda_stream for a in call(side)[1::5])
    torch.cuda.synchronize()


def test_norm_results_belong_to_the_stream_given():
    t, d = norm_inputs(300, 1000, "f32", 7, 20)
    op = blocks.ResidualNorm(1000, dtype="f32", norm="layer", group=20)
    w = [t[k] for k in ("post", "pre", "post_bias", "pre_bias")]

    def call(stream):
        res, out, stats = op.forward(t["residual"], t["branch"], *w, gate=t["gate"], stream=stream)
        g = op.backward(t["residual"], t["branch"], *w, *d, stats, gate=t["gate"], stream=stream)
        return [res, out, stats, *g.values()]

    on_both(call)


def test_int8_and_adamw_results_belong_to_the_stream_given():
    g = rng(8)
    codes, scales = blocks.quantize_weight(normal(g, 96, 500).float().cuda())
    op = blocks.Int8Linear(codes, scales, dtype="f32")
    for rows in (1, 20, 300):
        x = normal(g, rows, 500).float().cuda()
        on_both(lambda stream: [op(x, stream=stream)])
    p = [normal(g, n).float().cuda() for n in (5000, 300)]
    adam = blocks.AdamW(p, [a * 0.1 for a in p], bits=8)
    adam.step()
    on_both(lambda stream: [a for part in adam.states(stream=stream) for a in part])


def test_what_a_handle_drops_waits_for_the_stream_given():
    """Gradients that set_grads replaces are not reused before the steps queued on the stream are done."""
    g = rng(9)
    side = torch.cuda.Stream()
    p = [normal(g, 1 << 20).float().cuda()]
    old = normal(g, 1 << 20).float().cuda()
    at, op = old.data_ptr(), blocks.AdamW(p, [old])
    fresh = torch.zeros(1 << 20, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy = torch.empty(1 << 28, device="cuda")
        for _ in range(100):
            busy.normal_()
    op.step(stream=side)
    op.set_grads([fresh], stream=side)
    del old
    again = torch.empty(1 << 20, device="cuda")
    assert again.data_ptr() != at
    torch.cuda.synchronize()


# ----------------------------------------------------------------------------- refusals
@pytest.mark.parametrize("name", ["post", "pre", "post_bias", "pre_bias"])
@pytest.mark.parametrize("bad", ["type", "short", "host", "apart"])
def test_norm_vectors_are_checked_in_both_directions(name, bad):
    t, d = norm_inputs(6, 64, "bf16", 3)
    op = blocks.ResidualNorm(64, norm="layer")
    order = ("post", "pre", "post_bias", "pre_bias")
    stats = op.forward(t["residual"], t["branch"], *(t[k] for k in order))[2]
    torch.cuda.synchronize()
    v = t[name]
    t[name] = {"type": v.bfloat16(), "short": v[:63], "host": v.cpu(), "apart": v.repeat_interleave(2)[::2]}[bad]
    with pytest.raises(ValueError, match=name):
        op.forward(t["residual"], t["branch"], *(t[k] for k in order))
    with pytest.raises(ValueError, match=name):
        op.backward(t["residual"], t["branch"], *(t[k] for k in order), *d, stats)


# ----------------------------------------------------------------------------- in place
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("model", [5, 200, 513, 519, 1030, 2051, 3079, 4095, 6001, 12290])
def test_norms_in_place(model, dtype, post):
    """res over residual, at widths whose last piece begins a wave: the row's last values are two threads' to read."""
    rows = 400
    t, _ = norm_inputs(rows, model, dtype, model, biases=False, post=post)
    op = blocks.ResidualNorm(model, dtype=dtype, keep=0.75)
    want = op.forward(t["residual"], t["branch"], t["post"], t["pre"])
    res, out, stats = t["residual"].clone(), torch.empty_like(t["residual"]), torch.empty(rows, 4, device="cuda")
    status = binding.lib().enova_resnorm_forward(
        op.handle, res.data_ptr(), t["branch"].data_ptr(), rows, t["post"].data_ptr() if post else None, None,
        t["pre"].data_ptr(), None, None, res.data_ptr(), out.data_ptr(), stats.data_ptr(),
        torch.cuda.current_stream().cuda_stream)
    assert status == binding.ENOVA_OK
    assert all(torch.equal(a, b) for a, b in zip((res, out, stats), want))


# ----------------------------------------------------------------------------- long calls
def windows_of(rows, run):
    """Row ranges at both ends and around the places where one launch's rows end."""
    return [slice(max(at - 40, 0), min(at + 40, rows)) for at in (0, run, rows // 2, rows)]


def test_int8_product_of_more_rows_than_a_launch_has_threads_for():
    rows = (1 << 24) + 5                       # blocks of 256 threads, one a row
    g = rng(8)
    codes, scales = blocks.quantize_weight(normal(g, 8, 16).float().cuda())
    op = blocks.Int8Linear(codes, scales)
    x = torch.randn(rows, 16, dtype=torch.bfloat16, device="cuda")
    y = op(x)
    for s in windows_of(rows, 1 << 23):
        assert torch.equal(y[s], op(x[s]))


def test_norms_of_more_rows_than_a_launch_has_threads_for():
    rows = (1 << 28) + 5                       # teams of 16 threads
    op = blocks.ResidualNorm(2, group=3)
    post, pre = (torch.tensor([0.5, 2.0], device="cuda") for _ in range(2))
    residual, branch = (torch.randn(rows, 2, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gate = torch.randn(-(-rows // 3), 2, device="cuda")
    got = op.forward(residual, branch, post, pre, gate=gate)
    for s in windows_of(rows, 1 << 27):
        first = s.start // 3 * 3
        part = op.forward(residual[first:s.stop], branch[first:s.stop], post, pre, gate=gate[first // 3:-(-s.stop // 3)])
        assert all(torch.equal(a[first:s.stop], b) for a, b in zip(got, part))


def test_gradients_of_no_rows_are_zeros_in_all_of_a_large_weight():
    model, hidden = 1 << 16, (1 << 16) + 1
    op = blocks.GatedBlock(model, hidden)
    dw = torch.full((model, hidden), 1.0, dtype=torch.bfloat16, device="cuda")
    w = dw.data_ptr()                          # of no rows nothing is read
    status = binding.lib().enova_gated_backward(op.handle, None, model, 0, w, w, w, None, None, model, None, model, None,
                                                None, w, torch.cuda.current_stream().cuda_stream)
    assert status == binding.ENOVA_OK and not dw.any()


# ----------------------------------------------------------------------------- AdamW
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-50, 1e-42, 1.2e-38, 1e-8])
def test_adamw_of_gradients_that_are_zero(eps, bits):
    """However small eps is, an element without a gradient only decays, and the others step by lr."""
    g = rng(4)
    p = normal(g, 1000).float().cuda()
    d = normal(g, 1000).float().cuda()
    d[::3] = 0.0
    want = p.double() * (1 - 1e-2 * 0.01) - torch.sign(d.double()) * 1e-2 * (d.abs() / (d.abs() + eps)).nan_to_num()
    op = blocks.AdamW([p], [d], bits=bits, eps=eps, lr=1e-2)
    op.step()
    assert (p.double() - want).abs().max() <= 4 * 2.0 ** -24 * 4      # p of up to 4


# ----------------------------------------------------------------------------- activations
@pytest.mark.parametrize("rows", [60, 3001])
@pytest.mark.parametrize("act,ends", [("gelu", 11.0), ("silu", 70.0)])
def test_block_f32_activations_are_those_of_fp32(act, ends, rows):
    """act(g) and act'(g) by themselves, through weights of 0 and 1, far into the tail.

    GELU: erfc of a product rounded once and of a rounded constant is off by 2 (g^2 / 2) 1.3 units of 2^-24, the
    function and the products by a few more. SiLU: an exponential, a sum, a quotient and a product. The derivatives
    are sums of such terms up to 1.1 in size."""
    g = torch.linspace(-ends, ends, rows, device="cuda")
    x = torch.stack([g, torch.ones_like(g)], 1)
    wg, wu, wd = (torch.tensor(w, device="cuda") for w in ([[1.0, 0.0]], [[0.0, 1.0]], [[1.0], [0.0]]))
    dy = torch.zeros_like(x)
    dy[:, 0] = 1.0
    y, dx, *_ = run_block(blocks.GatedBlock(2, 1, dtype="f32", act=act), x, wg, wu, wd, dy)
    v = g.double().requires_grad_(True)
    a = 0.5 * v * torch.special.erfc(-v / 2 ** 0.5) if act == "gelu" else v * torch.sigmoid(v)
    da, = torch.autograd.grad(a.sum(), v)
    a, v = a.detach(), v.detach()
    tol = (8 + (2 * v * v if act == "gelu" else 0)) * 2.0 ** -24 * a.abs()
    assert ((y[:, 0].double() - a).abs() <= tol).all()
    assert ((dx[:, 1].double() - a).abs() <= tol).all()
    assert (dx[:, 0].double() - da).abs().max() <= 1e-6


@pytest.mark.parametrize("saved", [True, False])
@pytest.mark.parametrize("rows", [20, 300])
def test_block_relu_derivative_of_a_small_g_beside_large_ones(rows, saved):
    """A hidden unit whose g is 2^-50 of its neighbours' is as much on as they are (its own value is kept to 2^-39 of
    the largest: nothing)."""
    t = block_inputs(rows, 8, 16, "bf16", rows)
    t[0].abs_()
    t[1].abs_().add_(0.1)
    t[1][3] *= 2.0 ** -50
    t[1][12] *= -(2.0 ** -50)
    got = run_block(blocks.GatedBlock(8, 16, act="relu"), *t, saved=saved)
    want = block64(*t, "relu")
    for unit in range(16):
        close(got[2][unit], want[2][unit], 2e-2, f"dwg[{unit}]")
        if unit != 3:
            close(got[3][unit], want[3][unit], 2e-2, f"dwu[{unit}]")
    assert float(got[3][3].abs().max()) <= 2.0 ** -38 * float(want[3].abs().max())
    assert not got[2][12].any() and not got[3][12].any()


def test_adamw_states_into_one_list_given():
    g = rng(4)
    p = [normal(g, n).float().cuda() for n in (1000, 7)]
    op = blocks.AdamW(p, [a * 0.1 for a in p], bits=8)
    op.step()
    want = op.states()
    for which in (0, 1):
        mine = [torch.full_like(a, 9.0) for a in p]
        got = op.states(**{"mv"[which]: mine})
        assert all(a is b for a, b in zip(got[which], mine))
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


@pytest.mark.parametrize("rows", [20, 90])
@pytest.mark.parametrize("act", ["gelu", "relu"])
def test_block_f32_rows_of_all_sizes_with_other_activations(act, rows):
    """As for SiLU in test_gpu_blocks_edges.py: within four times the worst row of the formula in fp32."""
    t = block_inputs(rows, 72, 136, "f32", 21)
    size = 10.0 ** torch.linspace(-8, 8, rows, device="cuda")[:, None]
    t[0] *= size
    t[4] /= size
    t[4][:, 5] *= 1e-6
    t[3][:, 9] *= 1e-6
    got = run_block(blocks.GatedBlock(72, 136, dtype="f32", act=act), *t)
    v = [a.cpu().requires_grad_(True) for a in t[:4]]
    y = (act64(v[0] @ v[1].T, act) * (v[0] @ v[2].T)) @ v[3].T
    plain = [y.detach(), *torch.autograd.grad(y, v, t[4].cpu())]

    def worst(a, b):
        return float(((a.double().cpu() - b).norm(dim=1) / b.norm(dim=1)).max())

    for name, a, f, b in zip(("y", "dx", "dwg", "dwu", "dwd"), got, plain, block64(*t, act)):
        assert worst(a, b) <= 4 * worst(f, b), (name, worst(a, b), worst(f, b))


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("grad", ["bf16", "f32"])
def test_adamw_bf16_parameters_with_8_bit_states(grad, shift):
    """A step from the states' own values: p is the rounding of the formula's, m and sqrt(v) within a code and its dither."""
    p, g = adam_inputs("bf16", grad, 6, shift)
    op = blocks.AdamW(p, g, bits=8, lr=1e-2)
    m, v = ([a.clone() for a in s] for s in op.states())
    for n in range(1, 5):
        before = [a.double() for a in p]
        op.step(grad_scale=2.0)
        got_m, got_v = op.states()
        for i in range(len(p)):
            q, wm, wv = adam64(before[i], 2.0 * g[i].double(), m[i].double(), v[i].double(), n, 1e-2)
            off = 3e-7 * q.abs() + 1e-7        # three roundings in fp32, and ten of an update of up to 0.1
            assert ((p[i] >= (q - off).bfloat16()) & (p[i] <= (q + off).bfloat16())).all()
            for part in range(0, p[i].numel(), 256):
                s = slice(part, part + 256)
                assert (got_m[i][s] - wm[s]).abs().max() <= wm[s].abs().max() * (2 / 127) + 1e-12
                assert (got_v[i][s].double().sqrt() - wv[s].sqrt()).abs().max() <= wv[s].sqrt().max() * (2 / 255) + 1e-12
        m, v = ([a.clone() for a in s] for s in (got_m, got_v))
