"""Without a workspace argument, every op allocates its own on the stream that it runs on: freed with the call's
return, it is then not handed out on the caller's stream while the op is still queued."""
import contextlib
from types import SimpleNamespace

import pytest
import torch

from gpu_helpers import lib
from paper_2604_11947_amd import resbm as R
from test_current_device import Tensor

T, N, M, RK = 4, 64, 64, 8


def ops(L, act, f, f64, **k):
    """name -> call, of every op that can allocate a workspace."""
    plan = SimpleNamespace(q8=False, used_on=lambda s: None, host_ptr=0, table_ptr=0, table=f(1), device=torch.device("cuda", 0))
    return {
        "encode_fwd": lambda: L.encode_fwd(act(T, N), act(T, N), f(N, RK), act(T, RK), f(T, RK), **k),
        "decode_bwd": lambda: L.decode_bwd(act(T, RK), f(RK, N), act(T, N), None, act(T, RK), f(RK, N), **k),
        "encode_bwd": lambda: L.encode_bwd(act(T, N), f(N, RK), f(T, RK), act(T, RK), act(T, N), f(N, RK), **k),
        "encode2_fwd": lambda: L.encode2_fwd(act(T, N), act(T, N), act(N, M), act(M, RK), act(T, RK), act(T, M), **k),
        "decode2_fwd": lambda: L.decode2_fwd(act(T, RK), act(RK, M), act(M, N), act(T, N), act(T, M), **k),
        "decode2_bwd": lambda: L.decode2_bwd(act(T, RK), act(T, M), act(T, N), None, act(RK, M), act(M, N), act(T, RK),
                                             f(RK, M), f(M, N), **k),
        "encode2_bwd": lambda: L.encode2_bwd(act(T, N), act(T, M), act(T, RK), act(N, M), act(M, RK), act(T, N), f(N, M),
                                             f(M, RK), **k),
        "ffn_encode_fwd": lambda: L.ffn_encode_fwd(act(T, 128), act(128, N), act(T, N), f(N, RK), act(T, N), act(T, RK), f(T, RK), **k),
        "decode_qkv_fwd": lambda: L.decode_qkv_fwd(act(T, RK), f(RK, N), f(N), act(N, 64), act(T, 64), **k),
        "newton_schulz": lambda: L.newton_schulz(f(N, RK), f(N, RK), **k),
        "muon_update": lambda: L.muon_update(f(N, RK), f(N, RK), None, 0.1, **k),
        "spectrum": lambda: L.spectrum(f(N, RK), f64(RK), f64(1), **k),
        "skip_norm_bwd": lambda: L.skip_norm_bwd(act(T, N), f(N), f(T), act(T, N), act(T, N), f(N), **k),
        "grad_norm": lambda: L.grad_norm(plan, 1.0, f(2), **k),
    }


NAMES = list(ops(None, None, lambda *s: None, None))


@pytest.mark.parametrize("name", NAMES)
def test_the_stream_of_the_allocation(name, monkeypatch):
    at, now = [], [None]

    @contextlib.contextmanager
    def allocating_on(stream, device):
        now[0] = stream
        yield
        now[0] = None

    def empty(*a, **k):
        at.append(now[0])
        return torch.zeros(4096, dtype=torch.uint8)

    class Cdll:
        def __getattr__(self, fn):
            return lambda *a: 256 if fn.endswith("_bytes") else R.OK
    L = R.Library.__new__(R.Library)
    L.cdll, L.io_dtype = Cdll(), torch.bfloat16
    monkeypatch.setattr(R, "_marshal", None)
    monkeypatch.setattr(R, "_allocating_on", allocating_on)
    monkeypatch.setattr(R, "_one_gpu", lambda *a: None)
    monkeypatch.setattr(R.torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    tensor = lambda dt: lambda *s: Tensor(dt, *s, dev=0)
    ops(L, tensor(torch.bfloat16), tensor(torch.float32), tensor(torch.float64), stream=77)[name]()
    assert at == [77]


@pytest.mark.gpu
def test_a_workspace_behind_a_busy_stream():
    """The boundary's backward ops queued on a busy side stream, by object and by handle, while the caller's
    stream allocates and fills memory of the workspace's size."""
    L = lib()
    t, n, r = 1000, 512, 32
    g = torch.Generator(device="cuda").manual_seed(3)
    rn = lambda *s, dt=torch.bfloat16: torch.randn(*s, generator=g, device="cuda").to(dt)
    f32 = torch.float32
    z, gz, gb, b, a = rn(t, n), rn(t, n), rn(t, r), rn(t, r), rn(t, r, dt=f32)
    W_e, W_d = rn(n, r, dt=f32), rn(r, n, dt=f32)

    def run(stream=None):
        o = [torch.zeros(t, r, dtype=torch.bfloat16, device="cuda"), torch.zeros(r, n, device="cuda"),
             torch.zeros(t, n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, r, device="cuda")]
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(side):
                torch.cuda._sleep(2_000_000)
        L.decode_bwd(b, W_d, gz, None, o[0], o[1], stream=stream)
        L.encode_bwd(z, W_e, a, gb, o[2], o[3], stream=stream)
        keep = [torch.empty(size, dtype=torch.uint8, device="cuda").fill_(0xFF) for _ in range(100)]
        torch.cuda.synchronize()
        del keep
        return o

    side, size = torch.cuda.Stream(), L.workspace(t, n, r, "cuda").numel() + 256
    ref = run()
    for stream in (side, side.cuda_stream):
        for x, y in zip(run(stream), ref):
            assert torch.equal(x, y)
