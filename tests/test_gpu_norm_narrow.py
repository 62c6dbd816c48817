"""The residual norm on narrow rows, several of which share a wave: widths around the borders of 16, 32
and 64 lanes a row, token counts around a wave's and a block's rows, strided rows, ranks that end inside
eight columns, and rows far apart.  Bounds as derived in test_gpu_norm.py."""
import numpy as np
import pytest
import torch

from gpu_helpers import f64, guarded, lib, say, strided
from oracle import stage_oracle as S
from test_gpu_norm import EPS, U, check_h, inputs, store, within

pytestmark = pytest.mark.gpu

WIDTHS = [8, 16, 72, 120, 128, 136, 200, 256, 264, 512]
TOKENS = [1, 2, 3, 4, 7, 15, 16, 17, 31, 33, 1000]


@pytest.mark.parametrize("variant", ["bf16", "f32"])
@pytest.mark.parametrize("n", WIDTHS)
def test_forward(n, variant):
    L = lib(variant)
    io = L.io_dtype
    for T in TOKENS:
        r = 4 * ((n // 4 + T) % (n // 4 + 1))
        pad = 8 * (T % 3)
        say(f"narrow forward {variant} T={T} n={n} r={r} pad={pad}")
        d = inputs(T, n, r, io, T)
        x, rs = strided(d["x"], pad), strided(d["res"], pad + 8)
        h, _, hg = guarded((T, n), io, "cuda", pad=pad)
        y, _, yg = guarded((T, n), io, "cuda", pad=16)
        buf = torch.full((T + 3, n + 8), 0x55, dtype=torch.uint8, device="cuda")
        q, sc = buf.view(torch.float8_e4m3fn)[2:T + 2, :n], torch.full((T + 1, 1), -1.0, device="cuda")
        rstd = torch.full((T + 1,), -1.0, device="cuda")
        L.skip_norm_fwd(x, d["gamma"], y, res=rs, b=d["b"], h=h, rstd=rstd[:T], eps=EPS)
        L.skip_norm_q8_fwd(x, d["gamma"], q, sc[:T], res=rs, b=d["b"], eps=EPS)
        torch.cuda.synchronize()
        hg(), yg()
        assert rstd[T] == -1 and sc[T] == -1
        assert bool((buf[:2] == 0x55).all()) and bool((buf[T + 2] == 0x55).all()) and bool((buf[:, n:] == 0x55).all())
        check_h(d, h, io, True, r > 0)
        ref = S.rstd(f64(h), EPS)
        within("rstd", rstd[:T], ref, 2.0 ** -18 * ref)
        ry = S.norm(f64(h), f64(d["gamma"]), EPS)
        within("y", y, ry, (store(io) + 2.0 ** -17) * np.abs(ry) + 2.0 ** -133)
        rsc = S.scales(ry)[:, None]
        within("scale", sc[:T], rsc, 2.0 ** -17 * rsc)
        s = f64(sc[:T])
        within("y8", torch.from_numpy(f64(q.float()) * s), ry, np.maximum(2.0 ** -4 * np.abs(ry), 2.0 ** -10 * s) * (1 + 2.0 ** -10)
               + 2.0 ** -16 * np.abs(ry))


@pytest.mark.parametrize("n,group", [(64, 32), (128, 32), (128, 64), (192, 64), (256, 32), (256, 64), (256, 128), (512, 256), (96, 32)])
def test_groups(n, group):
    L = lib()
    for T in (1, 3, 17, 100):
        d = inputs(T, n, 0, L.io_dtype, T + n)
        q, sc = torch.empty(T, n, device="cuda").to(torch.float8_e4m3fn), torch.full((T, n // group), float("nan"), device="cuda")
        L.skip_norm_q8_fwd(d["x"], d["gamma"], q, sc, eps=EPS)
        ry = S.norm(f64(d["x"]), f64(d["gamma"]), EPS)
        rs = S.scales(ry.reshape(T, -1, group))
        within("scale", sc, rs, 2.0 ** -17 * rs)
        s = np.repeat(f64(sc), group, axis=1)
        within("y8", torch.from_numpy(f64(q.float()) * s), ry, np.maximum(2.0 ** -4 * np.abs(ry), 2.0 ** -10 * s) * (1 + 2.0 ** -10)
               + 2.0 ** -16 * np.abs(ry))


@pytest.mark.parametrize("variant", ["bf16", "f32"])
@pytest.mark.parametrize("n", WIDTHS)
def test_backward(n, variant):
    L = lib(variant)
    io = L.io_dtype
    for T in TOKENS + [9000]:
        pad, acc = 8 * (T % 3), T % 2 == 0
        say(f"narrow backward {variant} T={T} n={n} pad={pad}")
        d = inputs(T, n, 0, io, T)
        rs = torch.from_numpy(S.rstd(f64(d["x"]), EPS)).float().cuda()
        H, G, R_, GY, GH = f64(d["x"]), f64(d["gamma"]), f64(rs), f64(d["gy"]), f64(d["gh"])
        old = torch.linspace(-1, 1, n, device="cuda")
        dg = old.clone() if acc else torch.full((n,), float("nan"), device="cuda")
        out, _, check = guarded((T, n), io, "cuda", pad=pad)
        L.skip_norm_bwd(strided(d["x"], pad), d["gamma"], rs, strided(d["gy"], 16), out, dg, g_h=strided(d["gh"], pad),
                        accumulate=acc, ws=L.norm_workspace(T, n, "cuda"))
        torch.cuda.synchronize()
        check()
        xh, w = H * R_[:, None], GY * G
        gx, ref = S.norm_bwd(H, G, R_, GY, GH)
        ref = ref + (f64(old) if acc else 0)
        terms = R_[:, None] * (np.abs(w) + np.abs(xh) * np.mean(np.abs(w * xh), axis=1, keepdims=True)) + np.abs(GH)
        within("g_x", out, gx, store(io) * np.abs(gx) + 128 * U * terms + 2.0 ** -133)
        within("dgamma", dg, ref, (T + 4) * U * np.sum(np.abs(GY * xh), axis=0) + 2 * U * np.abs(ref) + 2.0 ** -133)


def test_rows_that_are_far_apart():
    """Rows that share a wave lie up to 8 GiB apart: the same results, bit for bit, as packed ones."""
    L = lib()
    T, n = 6, 128
    for ld in (136, (1 << 26) + 8, 1 << 29):
        d = inputs(T, n, 8, L.io_dtype, 3)
        x = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda").view(T, ld)[:, :n]
        x.copy_(d["x"])
        out = []
        for src in (x, d["x"]):
            y, rs, h = torch.empty_like(d["x"]), torch.empty(T, device="cuda"), torch.empty_like(d["x"])
            L.skip_norm_fwd(src, d["gamma"], y, b=d["b"], h=h, rstd=rs)
            gx, dg = torch.empty_like(y), torch.empty(n, device="cuda")
            L.skip_norm_bwd(src, d["gamma"], rs, d["gy"], gx, dg, ws=L.norm_workspace(T, n, "cuda"))
            L.skip_norm_bwd(d["x"], d["gamma"], rs, src, gx, dg, accumulate=True)
            out.append((h, y, gx, dg, rs))
        assert all(torch.equal(a, b) for a, b in zip(*out))
        del x
