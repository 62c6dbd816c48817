"""The operators together, as a stage's training step has them: decoder, residual norm, its backward,
decoder backward with the norm's gradient as the skip's, gradient norm, Muon on W_d and AdamW on the
gain; against the float64 oracles, eager and as one replayed graph."""
import numpy as np
import pytest
import torch

from gpu_helpers import check, f64, lib, say
from oracle import resbm_oracle as O
from oracle import stage_oracle as S

pytestmark = pytest.mark.gpu

EPS = 1e-5


class Stage:
    def __init__(self, L, T, n, r, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
        io = L.io_dtype
        self.L, self.T, self.n, self.r = L, T, n, r
        self.b, self.attn, self.gy, self.gs = rn(T, r).to(io), rn(T, n).to(io), (0.1 * rn(T, n)).to(io), (0.1 * rn(T, n)).to(io)
        self.W_d, self.gamma = rn(r, n) / r ** 0.5, 1 + 0.1 * rn(n)
        e = lambda *s, dt=io: torch.empty(*s, dtype=dt, device="cuda")
        self.zt, self.h, self.y, self.rstd = e(T, n), e(T, n), e(T, n), e(T, dt=torch.float32)
        self.g_h, self.g_b, self.dW_d, self.dgamma = e(T, n), e(T, r), e(r, n, dt=torch.float32), e(n, dt=torch.float32)
        self.M = torch.zeros(r, n, device="cuda")
        self.m, self.v, self.copy = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), e(n, dt=torch.bfloat16)
        self.norm = torch.empty(2, device="cuda")
        self.plan = L.adamw_plan([self.gamma], [self.dgamma], [self.m], [self.v], copy=[self.copy])
        self.grads = L.grad_plan([self.dW_d, self.dgamma])
        self.ws, self.nws = L.workspace(T, n, r, "cuda"), L.norm_workspace(T, n, "cuda")
        self.mws, self.gws = L.matrix_workspace(r, n, "cuda"), L.grad_norm_workspace(self.grads)

    def run(self):
        L = self.L
        L.decode_fwd(self.b, self.W_d, self.zt, ws=self.ws)
        L.skip_norm_fwd(self.zt, self.gamma, self.y, res=self.attn, b=self.b, h=self.h, rstd=self.rstd, eps=EPS)
        L.skip_norm_bwd(self.h, self.gamma, self.rstd, self.gy, self.g_h, self.dgamma, g_h=self.gs, ws=self.nws)
        L.decode_bwd(self.b, self.W_d, self.g_h, self.g_h, self.g_b, self.dW_d, ws=self.ws)
        L.grad_norm(self.grads, 1.0, self.norm, ws=self.gws)
        L.muon_update(self.W_d, self.dW_d, self.M, 1e-2, ws=self.mws)
        L.adamw_update(self.plan, 1e-2, 1, grad_scale=self.norm[1:])


def values(s):
    return {k: getattr(s, k).clone() for k in ("h", "y", "rstd", "g_h", "g_b", "dW_d", "dgamma", "W_d", "gamma", "m", "v", "copy", "norm")}


@pytest.mark.parametrize("variant", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(300, 512, 32), (77, 2112, 20), (1, 64, 4)], ids=lambda s: "x".join(map(str, s)))
def test_training_step(shape, variant):
    T, n, r = shape
    say(f"stage step {variant} T={T} n={n} r={r}")
    L = lib(variant)
    s = Stage(L, T, n, r, 21)
    W0, g0 = f64(s.W_d), f64(s.gamma)
    s.run()
    torch.cuda.synchronize()
    bf = variant == "bf16"
    bound = 2e-2 if bf else 1e-5  # the framework's bounds: of RMS(ref), half a bf16 step discounted
    zt = O.decode_fwd(f64(s.b), W0, False)
    check("z~", s.zt, zt, bf, bound)
    h = S.stream(f64(s.zt), f64(s.attn), f64(s.b))
    check("h", s.h, h, bf, bound)
    check("y", s.y, S.norm(f64(s.h), g0, EPS), bf, bound)
    gx, dg = S.norm_bwd(f64(s.h), g0, f64(s.rstd), f64(s.gy), f64(s.gs))
    check("g_h", s.g_h, gx, bf, bound)
    xh = f64(s.h) * f64(s.rstd)[:, None]
    check("dgamma", s.dgamma, dg, False, bound, scale=float(np.sqrt(np.mean(np.sum(np.abs(f64(s.gy) * xh), axis=0) ** 2))))
    check("g_b", s.g_b, f64(s.g_h) @ W0.T + f64(s.g_h)[:, :r], bf, bound)
    norm, f = S.grad_norm([f64(s.dW_d), f64(s.dgamma)], 1.0)
    assert abs(float(s.norm[0]) - norm) <= 2.0 ** -23 * norm
    rp, rm, rv = S.adamw(g0, f64(s.dgamma), np.zeros(n), np.zeros(n), 1e-2, 1, 0.9, 0.95, 1e-8, 0.0, f)
    # at step 1 the update is lr sign(g): 40 roundings of it and of gamma
    assert np.max(np.abs(f64(s.gamma) - rp)) <= 40 * 2.0 ** -24 * (1.5 + 1e-2)
    assert torch.equal(s.copy, s.gamma.bfloat16())
    assert bool(s.W_d.isfinite().all()) and not np.array_equal(f64(s.W_d), W0)


def test_the_step_as_a_graph():
    """Captured once and replayed from the same start, eager work in between: the eager results each time."""
    L = lib()
    s = Stage(L, 333, 512, 32, 22)
    start = {k: getattr(s, k).clone() for k in ("W_d", "gamma", "M", "m", "v")}

    def back():
        for k, t in start.items():
            getattr(s, k).copy_(t)

    s.run()
    torch.cuda.synchronize()
    ref = values(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    torch.cuda.synchronize()
    for rep in range(4):
        back()
        for k in ("h", "y", "rstd", "g_h", "g_b", "dW_d", "dgamma", "copy", "norm"):
            getattr(s, k).fill_(float("nan"))
        for ws in (s.ws, s.nws, s.mws, s.gws):
            ws.fill_(0x5A)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, t in values(s).items():
            assert torch.equal(t.view(torch.uint8), ref[k].view(torch.uint8)), (rep, k)


def test_two_graphs_share_a_workspace():
    """Two captured backward passes of different sizes on one workspace, replayed in turn."""
    L = lib()
    g = torch.Generator(device="cuda").manual_seed(23)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    ws = L.norm_workspace(900, 1024, "cuda")
    jobs = []
    for T, n in ((900, 1024), (130, 512)):
        a = dict(h=rn(T, n).bfloat16(), gamma=1 + 0.1 * rn(n), rstd=rn(T).abs(), g_y=rn(T, n).bfloat16(),
                 g_x=torch.empty(T, n, dtype=torch.bfloat16, device="cuda"), dgamma=torch.empty(n, device="cuda"))
        L.skip_norm_bwd(**a, ws=ws)
        torch.cuda.synchronize()
        ref = a["g_x"].clone(), a["dgamma"].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            L.skip_norm_bwd(**a, ws=ws)
        jobs.append((graph, a, ref))
    for rep in range(3):
        for graph, a, ref in jobs:
            a["g_x"].zero_()
            a["dgamma"].fill_(float("nan"))
            graph.replay()
        torch.cuda.synchronize()
        for _, a, ref in jobs:
            assert torch.equal(a["g_x"], ref[0]) and torch.equal(a["dgamma"], ref[1])
