"""Random shapes, strides, options and places of the residual norm's three ops and of AdamW, from fixed
seeds, against the float64 oracle.  Bounds as derived in test_gpu_norm.py and test_gpu_adamw.py."""
import random

import numpy as np
import pytest
import torch

import test_gpu_adamw as A
from gpu_helpers import f64, lib, say, strided
from oracle import stage_oracle as S
from test_gpu_norm import EPS, U, check_h, inputs, store, within

pytestmark = pytest.mark.gpu


def logint(rng, lo, hi, step=1):
    return max(lo, min(hi, int(np.exp(rng.uniform(np.log(lo), np.log(hi)))) // step * step))


@pytest.mark.parametrize("seed", range(48))
def test_norm(seed):
    rng = random.Random(seed)
    L = lib(rng.choice(["bf16", "bf16", "f32"]))
    io = L.io_dtype
    n = logint(rng, 8, 40000, 8)
    T = logint(rng, 1, max(1, min(3000, 2_000_000 // n)))
    group = rng.choice([0, 32, 64, 128, 256])
    if group:
        n = max(group, n // group * group)
    r = logint(rng, 4, min(n, 256), 4) if rng.random() < 0.7 else 0
    res, place, acc = rng.random() < 0.7, rng.choice([None, None, "x", "res"]), rng.random() < 0.5
    pads = [8 * rng.randrange(4) for _ in range(8)]
    say(f"random norm {seed}: T={T} n={n} r={r} group={group} res={res} place={place} acc={acc} pads={pads}")
    d = inputs(T, n, r, io, 1000 + seed)
    x, rs = strided(d["x"], pads[0]), strided(d["res"], pads[1]) if res else None
    h = x if place == "x" else rs if place == "res" and res else strided(torch.zeros_like(d["x"]), pads[2])
    y, rstd = strided(torch.zeros_like(d["x"]), pads[3]), torch.empty(T, device="cuda")
    if rng.random() < 0.5:
        q = torch.zeros(T, n + 16, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :n]
        sc = torch.empty(T, n // (group or n), device="cuda")
        L.skip_norm_q8_fwd(strided(d["x"], pads[0]), d["gamma"], q, sc, res=rs if h is not rs else strided(d["res"], 8), b=d["b"], eps=EPS)
    else:
        q = None
    L.skip_norm_fwd(x, d["gamma"], y, res=rs, b=d["b"], h=h, rstd=rstd, eps=EPS)
    torch.cuda.synchronize()
    check_h(d, h, io, res, r > 0)
    H = f64(h)
    ref = S.rstd(H, EPS)
    within("rstd", rstd, ref, 2.0 ** -18 * ref)
    ry = S.norm(H, f64(d["gamma"]), EPS)
    within("y", y, ry, (store(io) + 2.0 ** -17) * np.abs(ry) + 2.0 ** -133)
    if q is not None:
        rsc = S.scales(ry.reshape(T, -1, group or n))
        within("scale", sc, rsc, 2.0 ** -17 * rsc)
        s = np.repeat(f64(sc), group or n, axis=1)
        within("y8", torch.from_numpy(f64(q.float()) * s), ry, np.maximum(2.0 ** -4 * np.abs(ry), 2.0 ** -10 * s) * (1 + 2.0 ** -10)
               + 2.0 ** -16 * np.abs(ry))
    gy, gh = strided(d["gy"], pads[4]), strided(d["gh"], pads[5]) if rng.random() < 0.7 else None
    out = rng.choice([gy, gh, None])
    out = strided(torch.zeros_like(d["x"]), pads[6]) if out is None else out
    old = torch.linspace(-1, 1, n, device="cuda")
    dg = old.clone()
    L.skip_norm_bwd(h, d["gamma"], rstd, gy, out, dg, g_h=gh, accumulate=acc)
    torch.cuda.synchronize()
    G, R_, GY, GH = f64(d["gamma"]), f64(rstd), f64(d["gy"]), f64(d["gh"]) if gh is not None else None
    gx, ref = S.norm_bwd(H, G, R_, GY, GH)
    ref = ref + (f64(old) if acc else 0)
    xh, w = H * R_[:, None], GY * G
    terms = R_[:, None] * (np.abs(w) + np.abs(xh) * np.mean(np.abs(w * xh), axis=1, keepdims=True)) + (0 if GH is None else np.abs(GH))
    within("g_x", out, gx, store(io) * np.abs(gx) + 128 * U * terms + 2.0 ** -133)
    within("dgamma", dg, ref, (T + 4) * U * np.sum(np.abs(GY * xh), axis=0) + 2 * U * np.abs(ref) + 2.0 ** -133)


@pytest.mark.parametrize("seed", range(24))
def test_adamw(seed):
    rng = random.Random(100 + seed)
    L = lib()
    parts, wd = [], []
    for k in range(rng.randrange(1, 5)):
        sizes = [logint(rng, 1, rng.choice([40, 3000, 200000])) for _ in range(rng.randrange(1, 8))]
        parts.append(A.make(sizes, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.7, 50 * seed + k, rng.randrange(5)))
        wd += [rng.choice([0.0, 0.1, 0.5]) for _ in sizes]
    d = {k: sum((p[k] for p in parts), []) for k in parts[0]}
    say(f"random adamw {seed}: {[t.numel() for t in d['p']]}")
    P = A.plan(L, d, wd)
    out = torch.empty(2, device="cuda")
    for step in (1, rng.randrange(2, 5000)):
        L.grad_norm(P, 0.1, out)
        norm, f = S.grad_norm([f64(g) for g in d["g"]], 0.1)
        assert abs(float(out[0]) - norm) <= 1.01 * U * norm
        A.step_and_check(L, d, P, wd, 10.0 ** -rng.randrange(1, 5), step, gs=float(out[1]), grad_scale=out[1:])
