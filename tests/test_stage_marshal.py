"""The native marshalling of the residual norm's, AdamW's and the gradient norm's calls: the same
results as the Python path, which takes over for anything but the plain case."""
import pytest
import torch

from gpu_helpers import lib
from paper_2604_11947_amd import resbm as R


def test_hands_host_tensors_back():
    x, g = torch.zeros(4, 64, dtype=torch.bfloat16), torch.ones(64)
    assert R._marshal.skip_norm_fwd(0, 0, x, g, None, None, None, None, 1e-5, x) is None
    assert R._marshal.skip_norm_q8_fwd(0, 0, x, g, None, None, None, None, 1e-5, x, g) is None
    assert R._marshal.skip_norm_bwd(0, 0, x, g, g, x, x, g, None, False, g) is None
    assert R._marshal.adamw_update(0, 0, x, 0.1, 1, (0.9, 0.95), 1e-8, None, None) is None
    assert R._marshal.grad_norm(0, 0, x, 1.0, g, g) is None


@pytest.mark.gpu
def test_same_calls_as_the_python_path(monkeypatch):
    L = lib()
    T, n, r = 37, 192, 12
    g = torch.Generator(device="cuda").manual_seed(0)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, res, gy = (rn(T, n + 8).bfloat16()[:, :n] for _ in range(3))
    b, gamma, rs = rn(T, r).bfloat16(), rn(n), rn(T).abs()
    p0, g0 = rn(1000), rn(1000)

    def run():
        o = {k: torch.zeros(T, n, dtype=torch.bfloat16, device="cuda") for k in ("h", "y", "gx")}
        o |= {"rstd": torch.zeros(T, device="cuda"), "q": torch.zeros(T, n, device="cuda").to(torch.float8_e4m3fn),
              "scale": torch.zeros(T, 3, device="cuda"), "dg": torch.ones(n, device="cuda"), "out": torch.zeros(2, device="cuda"),
              "p": p0.clone(), "m": torch.zeros(1000, device="cuda"), "v": torch.zeros(1000, device="cuda")}
        P = L.adamw_plan([o["p"]], [g0], [o["m"]], [o["v"]])
        ws, gws = L.norm_workspace(T, n, "cuda"), L.grad_norm_workspace(P)
        hyp = torch.tensor([0.01, 2.0], dtype=torch.float64, device="cuda")
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            L.skip_norm_fwd(x, gamma, o["y"], res=res, b=b, h=o["h"], rstd=o["rstd"], eps=1e-6)
            L.skip_norm_q8_fwd(x, gamma, o["q"], o["scale"], res=res)
            L.skip_norm_bwd(x, gamma, rs, gy, o["gx"], o["dg"], g_h=res, accumulate=True, ws=ws)
            L.grad_norm(P, 1.0, o["out"], ws=gws)
            L.adamw_update(P, 0.01, 1, grad_scale=o["out"][1:])
            L.adamw_update(P, lr_step=hyp, betas=(0.8, 0.9), eps=1e-6)
        torch.cuda.current_stream().wait_stream(st)
        torch.cuda.synchronize()
        return o

    fast = run()
    calls = R._marshal
    assert calls.skip_norm_fwd(L._at["resbm_skip_norm_fwd"], L.io_code, x, gamma, None, None, None, None, 1e-5,
                               torch.zeros_like(x)) == R.OK
    P = L.adamw_plan([p0], [g0], [p0.clone()], [p0.abs()])
    assert calls.adamw_update(L._at["resbm_adamw_update"], P.host_ptr, P.table, 0.0, 1, (0.9, 0.95), 1e-8, None, None) == R.OK
    assert calls.grad_norm(L._at["resbm_grad_norm"], P.host_ptr, P.table, 1.0, fast["out"], L.grad_norm_workspace(P)) == R.OK
    with pytest.raises(ValueError, match="y: expected shape"):
        L.skip_norm_fwd(x, gamma, fast["y"][:3])
    with pytest.raises(ValueError, match="grad_scale"):
        L.adamw_update(P, 0.01, 1, grad_scale=fast["out"])
    with pytest.raises(R.ResbmError, match="resbm_adamw_update"):
        L.adamw_update(P, 0.01, 0)
    with pytest.raises(ValueError, match="out: expected"):
        L.grad_norm(P, 1.0, fast["rstd"])
    monkeypatch.setattr(R, "_marshal", None)
    for k, t in run().items():
        assert torch.equal(t.view(torch.uint8), fast[k].view(torch.uint8)), k
