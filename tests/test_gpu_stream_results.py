"""What the detector's and the configuration scan's methods return belongs to the stream that they are given."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from harness import detector, upload  # noqa: E402
from paper_2407_09486_amd import binding, workloads as wl  # noqa: E402
from test_gpu_blocks_use import on_both  # noqa: E402


def test_detector_results():
    cfg = wl.CONFIGS["c1"]
    work = wl.generate(cfg)
    det = detector(cfg, wl.make_weights(cfg), "auto")
    x, so = upload(work)
    woff = det.window_offsets(work.stream_offsets)
    n, wo = int(woff[-1]), torch.from_numpy(woff).cuda()
    on_both(lambda stream: list(det.score(x, so, wo, n, threshold=1.0, flags=True, stream=stream)))
    on_both(lambda stream: list(det.score_ext(x, so, wo, n, stream=stream)))
    scores = det.score(x, so, wo, n)[0]
    on_both(lambda stream: [det.threshold(scores, so, wo, flags=True, stream=stream)[2]])
    det.close()


def test_configuration_results():
    x = torch.from_numpy(np.ascontiguousarray(wl.config_series(2, 700, seed=3).x, np.float32)).cuda()
    offsets = np.array([0, 700, 1400], np.int64)
    scan = binding.ConfigScanner(x.shape[1], 64, 1, col_finished=0, col_running=1, col_exec_time=4, col_mem_util=5)
    so, woff = torch.from_numpy(offsets).cuda(), scan.window_offsets(offsets)
    wo, n = torch.from_numpy(woff).cuda(), int(woff[-1])
    on_both(lambda stream: list(scan.scan(x, so, wo, n, stream=stream)))
    on_both(lambda stream: list(scan.recommend(x, so, stream=stream)))
    scan.close()
