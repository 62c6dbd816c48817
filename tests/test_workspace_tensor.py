"""A workspace is as many bytes as it has elements, one after the other: an expanded tensor, which has fewer, and
a strided one are refused, through the native marshalling and without it."""
import pytest
import torch

from gpu_helpers import lib
from paper_2604_11947_amd import resbm as R


def test_room():
    assert R._room(None) == (None, 0)
    buf = torch.zeros(4096, dtype=torch.uint8)
    assert R._room(buf[256:])[1] == 3840
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(4096), buf[::2], buf.view(64, 64).t()):
        with pytest.raises(ValueError, match="ws: expected a contiguous"):
            R._room(bad)


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_ops_refuse_an_expanded_workspace(native, monkeypatch):
    L = lib()
    if not native:
        monkeypatch.setattr(R, "_marshal", None)
    T, n, r = 300, 512, 8
    bad = torch.zeros(1, dtype=torch.uint8, device="cuda").expand(1 << 26)
    x, g, rs = torch.ones(T, n, dtype=torch.bfloat16, device="cuda"), torch.ones(n, device="cuda"), torch.ones(T, device="cuda")
    b, W = torch.ones(T, r, dtype=torch.bfloat16, device="cuda"), torch.ones(r, n, device="cuda")
    gx, dg, out = torch.empty_like(x), torch.zeros(n, device="cuda"), torch.zeros(2, device="cuda")
    P = L.grad_plan([torch.ones(100_000, device="cuda")])
    for call in (lambda: L.skip_norm_bwd(x, g, rs, x, gx, dg, ws=bad), lambda: L.grad_norm(P, 1.0, out, ws=bad),
                 lambda: L.decode_fwd(b, W, gx, ws=bad), lambda: L.decode_bwd(b, W, x, None, b.clone(), W.clone(), ws=bad)):
        with pytest.raises(ValueError, match="ws: expected a contiguous"):
            call()
    torch.cuda.synchronize()
    assert not bool(dg.any()) and not bool(out.any())
