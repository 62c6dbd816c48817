"""Tensors of a GPU that is not the current one: the library is called with theirs as the current device, since
a launch on a device's default stream goes to that one; the native marshalling hands such calls back."""
from types import SimpleNamespace

import pytest
import torch

from paper_2604_11947_amd import resbm as R


class Current:
    """Stands for torch's current device."""

    def __init__(self):
        self.index = 0

    def device(self, dev):
        outer = self

        class Guard:
            def __enter__(self):
                self.before, outer.index = outer.index, dev.index

            def __exit__(self, *a):
                outer.index = self.before
        return Guard()


@pytest.fixture
def cur(monkeypatch):
    c = Current()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: c.index)
    monkeypatch.setattr(torch.cuda, "device", c.device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: SimpleNamespace(cuda_stream=0))
    monkeypatch.setattr(R, "_marshal", None)
    return c


class Tensor:
    """Stands for a (rows, cols) tensor on a GPU."""

    def __init__(self, dtype, *shape, dev=1):
        self.dtype, self.shape, self.device, self.is_cuda = dtype, shape, torch.device("cuda", dev), True

    dim = lambda self: len(self.shape)
    stride = lambda self, i: (self.shape[-1], 1)[i]
    data_ptr = lambda self: 256
    is_contiguous = lambda self: True

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n


@pytest.mark.parametrize("dev", [0, 1, 3])
def test_calls_run_on_the_tensors_device(cur, dev):
    seen = []
    L = R.Library.__new__(R.Library)
    L.io_dtype = torch.bfloat16

    class Cdll:
        def __getattr__(self, name):
            return lambda *a: seen.append((name, cur.index)) or R.OK
    L.cdll = Cdll()
    T, n, r = 4, 64, 8
    act, f = (lambda *s: Tensor(torch.bfloat16, *s, dev=dev)), (lambda *s: Tensor(torch.float32, *s, dev=dev))
    ws = Tensor(torch.uint8, 1 << 20, dev=dev)
    L.skip_norm_fwd(act(T, n), f(n), act(T, n))
    L.skip_norm_q8_fwd(act(T, n), f(n), Tensor(torch.float8_e4m3fn, T, n, dev=dev), f(T, 2))
    L.skip_norm_bwd(act(T, n), f(n), f(T), act(T, n), act(T, n), f(n), ws=ws)
    plan = SimpleNamespace(q8=False, used_on=lambda s: None, host_ptr=0, table_ptr=0, table=ws, device=torch.device("cuda", dev))
    L.adamw_update(plan, 1e-3, 1)
    L.grad_norm(plan, 1.0, f(2), ws=ws)
    L.encode_fwd(act(T, n), act(T, n), f(n, r), act(T, r), f(T, r), ws=ws)
    L.decode_fwd(act(T, r), f(r, n), act(T, n), ws=ws)
    L.decode_bwd(act(T, r), f(r, n), act(T, n), None, act(T, r), f(r, n), ws=ws)
    L.encode_bwd(act(T, n), f(n, r), f(T, r), act(T, r), act(T, n), f(n, r), ws=ws)
    L.muon_update(f(n, r), f(n, r), None, 0.1, ws=ws)
    L.decode_qkv_fwd(act(T, r), f(r, n), f(n), act(n, 64), act(T, 64), ws=ws)
    assert len(seen) == 11 and all(d == dev for _, d in seen), seen
    assert cur.index == 0


def test_an_error_leaves_the_current_device(cur):
    L = R.Library.__new__(R.Library)
    L.cdll = SimpleNamespace(op=lambda *a: R.E_NULL)
    L.strerror = lambda st: "null"
    with pytest.raises(R.ResbmError):
        L._run("op", Tensor(torch.float32, 1, dev=2), None)
    assert cur.index == 0
