"""A training step that a caller captured, replayed after the trainer has taken larger steps."""
import numpy as np
import pytest

from harness import log
from oracle import elbo
from paper_2407_09486_amd import workloads as wl
from test_gpu_train import _cfg, _dev, _init, _trainer

pytestmark = pytest.mark.gpu


def test_captured_step_outlives_larger_ones():
    """Bit for bit the steps of a trainer that captured nothing."""
    import torch
    cfg = _cfg(8, 32, 48, 8, "relu")
    p0 = _init(cfg)
    ga, eb = _trainer(cfg, p0), _trainer(cfg, p0)
    eb.set_graph(False)
    b = wl.training_batch(cfg, 5000, seed=5)
    V, lab, eps = (_dev(a) for a in (b.V, b.labels, b.eps))
    small = V[:200], lab[:200], eps[:200]
    larger = [(V[:n], lab[:n], eps[:n]) for n in (600, 2500, 5000)]
    log("a caller's capture of a training step, then larger steps")
    ga.step(*small)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, capture_error_mode="thread_local"):
        ga.step(*small)
    for batch in larger:
        ga.step(*batch)
        torch.cuda.synchronize()
        filled = [torch.full((1 << 18,), float("nan"), device="cuda") for _ in range(16)]
        g.replay()
        torch.cuda.synchronize()
        del filled
    eb.step(*small)
    for batch in larger:
        eb.step(*batch)
        eb.step(*small)
    pa, pb = ga.params(), eb.params()
    for name in elbo.PARAMS:
        assert np.array_equal(pa[name], pb[name]), name
    ga.close()
    eb.close()
