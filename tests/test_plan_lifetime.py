"""A plan's device table and the streams that read it: dropped while a step is still queued on another
stream, its memory is not handed out before that step has run."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from gpu_helpers import f64, lib
from oracle import stage_oracle as S
from paper_2604_11947_amd import resbm as R


class Table:
    """Stands for the device table: notes the streams that are recorded."""
    is_cuda = True

    def __init__(self):
        self.recorded = []

    def record_stream(self, stream):
        self.recorded.append(stream)

    def data_ptr(self):
        return 0


@pytest.fixture
def on(monkeypatch):
    """A plan made while stream 10 is current, and a library whose calls succeed."""
    now = SimpleNamespace(raw=10)
    monkeypatch.setattr(R, "_raw_stream", lambda device: now.raw)
    monkeypatch.setattr(R, "_torch_stream", lambda stream, device: ("stream", int(getattr(stream, "cuda_stream", stream))))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: SimpleNamespace(cuda_stream=now.raw))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(R, "_marshal", None)
    monkeypatch.setattr(R, "_one_gpu", lambda *a: None)
    L = R.Library.__new__(R.Library)
    L.cdll = SimpleNamespace(resbm_adamw_update=lambda *a: R.OK, resbm_grad_norm=lambda *a: R.OK)
    host = R.AdamWTensor()
    return now, L, R.AdamWPlan(host, Table(), [], torch.device("cuda", 0))


def test_streams_of_steps_are_recorded(on):
    now, L, P = on
    out = SimpleNamespace(dtype=torch.float32, dim=lambda: 1, numel=lambda: 2, is_contiguous=lambda: True, device=P.device,
                          data_ptr=lambda: 0)
    norm = lambda **k: L.grad_norm(P, 1.0, out, ws=out, **k)
    L.adamw_update(P, 1e-3, 1), norm(), L.adamw_update(P, 1e-3, 1, stream=10)
    assert P.table.recorded == []                       # the stream that the table belongs to
    L.adamw_update(P, 1e-3, 1, stream=20)
    norm(stream=SimpleNamespace(cuda_stream=30))
    assert P.table.recorded == [("stream", 20), ("stream", 30)]
    now.raw = 40                                        # another stream is current
    L.adamw_update(P, 1e-3, 1), norm()
    assert [s.cuda_stream for s in P.table.recorded[2:]] == [40]


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["object", "handle", "current"])
def test_a_dropped_plan_with_a_step_still_queued(how):
    """The plan goes while the side stream is busy before the step; what the caller's stream then allocates and
    fills does not reach the step."""
    L = lib()
    n = 5000
    g = torch.Generator(device="cuda").manual_seed(1)
    t = {k: [torch.randn(n, generator=g, device="cuda").abs() for _ in range(30)] for k in ("p", "g", "m", "v")}
    out, ref_out = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    before = [[f64(x) for x in t[k]] for k in ("p", "g", "m", "v")]
    L.grad_norm(L.grad_plan(t["g"]), 1.0, ref_out)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    size = 0
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)

    def step():
        nonlocal size
        P, Q = L.adamw_plan(t["p"], t["g"], t["m"], t["v"]), L.grad_plan(t["g"])
        size = P.table.untyped_storage().nbytes()
        ws = L.grad_norm_workspace(Q)
        if how == "current":
            with torch.cuda.stream(side):
                L.grad_norm(Q, 1.0, out, ws=ws)
                L.adamw_update(P, 1e-2, 1)
        else:
            s = side if how == "object" else side.cuda_stream
            L.grad_norm(Q, 1.0, out, ws=ws, stream=s)
            L.adamw_update(P, 1e-2, 1, stream=s)
        return ws

    ws = step()
    keep = [torch.empty(size, dtype=torch.uint8, device="cuda").fill_(0) for _ in range(100)]
    torch.cuda.synchronize()
    assert torch.equal(out, ref_out) and len(keep) == 100 and ws.numel()
    for i, (p, gr, m, v) in enumerate(zip(*before)):
        rp, _, _ = S.adamw(p, gr, m, v, 1e-2, 1, 0.9, 0.95, 1e-8, 0.0)
        # 3 u |p| and 26 u of an update of lr m / c1 / (sqrt(v / c2) + eps) each
        upd = np.abs(rp - p)
        assert np.all(np.abs(f64(t["p"][i]) - rp) <= 2.0 ** -24 * (3 * np.abs(p) + 26 * upd))
