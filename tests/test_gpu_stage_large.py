"""The residual norm and AdamW on the routes that only larger calls take: the one-pass backward of rows wider than
4096, tensors that are streamed past the caches (over 120 MB a call) in every form of a row, and dgamma sums in
which every row counts.  The reference is float64 torch on the device, in elementary operations.

Bounds as derived in test_gpu_norm.py and test_gpu_adamw.py, but for dgamma, whose chain of additions is counted:
a product of two roundings, T / 256 rows at most one after the other in a block (at least 256 blocks, or a row
each), 16 rows of a block, 16 partial sums (1024 at most, 64 side by side), and 2 + 16 sums of those: (T / 256 + 64) u."""
import numpy as np
import pytest
import torch

import test_gpu_adamw as A
from gpu_helpers import f64, lib, say, strided
from oracle import stage_oracle as S
from test_gpu_norm import EPS, U, inputs, store

pytestmark = pytest.mark.gpu


def within(name, got, ref, bound):
    bad = ~((got.double() - ref).abs() <= bound)
    assert not bool(bad.any()), (name, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), ref[bad][:4].tolist())


def check_backward(L, T, n, gh, acc, place=None, pad=0, seed=1):
    io = L.io_dtype
    d = inputs(T, n, 0, io, seed)
    h, gy, ghv = strided(d["x"], pad), strided(d["gy"], pad), strided(d["gh"], 8) if gh else None
    rs = (1 / (d["x"].double().square().mean(1) + EPS).sqrt()).float()
    out = {"gy": gy, "gh": ghv}.get(place)
    out = strided(torch.zeros_like(d["x"]), 16) if out is None else out
    old = torch.linspace(-1, 1, n, device="cuda")
    dg = old.clone() if acc else torch.full((n,), float("nan"), device="cuda")
    L.skip_norm_bwd(h, d["gamma"], rs, gy, out, dg, g_h=ghv, accumulate=acc)
    r = rs.double()[:, None]
    xh = d["x"].double().mul_(r)
    q = d["gy"].double().mul_(xh)
    ref = q.sum(0) + (old.double() if acc else 0)
    within("dgamma", dg, ref, (T / 256 + 64) * U * q.abs().sum(0) + 2 * U * ref.abs() + 2.0 ** -133)
    q.mul_(d["gamma"].double())
    c, ca = q.mean(1, keepdim=True), q.abs_().mean(1, keepdim=True)
    w = d["gy"].double().mul_(d["gamma"].double())
    gx, terms = (w - xh * c).mul_(r), w.abs_().add_(xh.abs_().mul_(ca)).mul_(r)
    if gh:
        gx += d["gh"]
        terms += d["gh"].abs()
    within("g_x", out, gx, store(io) * gx.abs() + 128 * U * terms + 2.0 ** -133)


@pytest.mark.parametrize("variant", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(257, 4104), (300, 4104), (611, 6152), (700, 8192), (520, 16384), (1300, 16376)],
                         ids=lambda s: "x".join(map(str, s)))
def test_one_pass_backward_of_wide_rows(shape, variant):
    say(f"one-pass backward {variant} {shape}")
    L = lib(variant)
    for gh, acc, place, pad in ((True, False, None, 8), (False, True, None, 0), (True, True, "gy", 0), (True, False, "gh", 24)):
        check_backward(L, *shape, gh, acc, place, pad)


# over 120 MB in three 16-bit tensors: each form of a row (16, 32 and 64 lanes; a block with one, two,
# four and eight chunks a lane)
LARGE = [(172_003, 128), (86_001, 256), (43_003, 512), (10_703, 2056), (5_501, 4096), (2_703, 8192), (1_351, 16384),
         (895, 24584), (341, 65536)]


@pytest.mark.parametrize("shape", LARGE, ids=lambda s: "x".join(map(str, s)))
def test_streamed_forward(shape):
    T, n = shape
    say(f"streamed forward {shape}")
    L = lib()
    io = L.io_dtype
    assert 3 * T * n * 2 > 120 << 20
    r = 20
    d = inputs(T, n, r, io, 2)
    h, y, rstd = strided(torch.zeros_like(d["x"]), 8), strided(torch.zeros_like(d["x"]), 16), torch.empty(T, device="cuda")
    L.skip_norm_fwd(d["x"], d["gamma"], y, res=d["res"], b=d["b"], h=h, rstd=rstd, eps=EPS)
    ref, mags = d["x"].double().add_(d["res"]), d["x"].double().abs_().add_(d["res"].abs())
    ref[:, :r] += d["b"]
    mags[:, :r] += d["b"].abs()
    within("h", h, ref, store(io) * ref.abs() + 2 * U * (1 + store(io)) * mags)
    ref = h.double()
    rs = 1 / (ref.square().mean(1) + EPS).sqrt()
    within("rstd", rstd, rs, 2.0 ** -18 * rs)
    ref.mul_(rs[:, None]).mul_(d["gamma"].double())
    within("y", y, ref, (store(io) + 2.0 ** -17) * ref.abs() + 2.0 ** -133)
    groups = [n] + [g for g in (32, 256) if n % g == 0 and n != g]
    for group in groups:
        q = torch.empty(T, n + 8, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :n]
        sc = torch.empty(T, n // group, device="cuda")
        h.zero_()
        L.skip_norm_q8_fwd(d["x"], d["gamma"], q, sc, res=d["res"], b=d["b"], h=h, eps=EPS)
        rsc = (ref.abs().view(T, -1, group).amax(2) / 448).clamp_(min=2.0 ** -126)
        within("scale", sc, rsc, 2.0 ** -17 * rsc)
        s = sc.double().repeat_interleave(group, 1)
        within("y8", q.float().double() * s, ref, torch.maximum(2.0 ** -4 * ref.abs(), 2.0 ** -10 * s) * (1 + 2.0 ** -10)
               + 2.0 ** -16 * ref.abs())
    within("h", h, d["x"].double().add_(d["res"]).add_(torch.nn.functional.pad(d["b"].double(), (0, n - r))),
           store(io) * h.double().abs() * (1 + 2 * store(io)) + 2 * U * (1 + store(io)) * mags)


@pytest.mark.parametrize("shape", LARGE, ids=lambda s: "x".join(map(str, s)))
def test_streamed_backward(shape):
    say(f"streamed backward {shape}")
    for gh, acc, place in ((True, False, None), (False, True, None), (True, False, "gy")):
        check_backward(lib(), *shape, gh, acc, place)


@pytest.mark.parametrize("shape", [((1 << 22) + 4100, 8), (9000, 8), (300_007, 128), (9001, 136), (100_003, 256), (50_001, 512),
                                   (1000, 512), (20_001, 520), (9_001, 2112), (257, 4096), (4_099, 4096), (3_001, 8192), (700, 16384), (700, 16392),
                                   (129, 65536), (5, 4096), (200, 1024), (256, 512)], ids=lambda s: "x".join(map(str, s)))
def test_every_row_counts(shape):
    """dgamma of h = +-1, rstd = 1 and whole g_y of -2 to 2: every partial sum is a whole number below 2^24,
    so the result is exact, and wrong by one where a single row is left out or taken twice."""
    T, n = shape
    say(f"every row counts {shape}")
    L = lib()
    g = torch.Generator(device="cuda").manual_seed(T)
    io = L.io_dtype
    h = (torch.randint(0, 2, (T, n), generator=g, device="cuda", dtype=torch.int8) * 2 - 1).to(io)
    gy = torch.randint(-2, 3, (T, n), generator=g, device="cuda", dtype=torch.int8).to(io)
    old = torch.randint(-9, 10, (n,), generator=g, device="cuda").float()
    ref = (h.float() * gy.float()).sum(0, dtype=torch.float64)
    assert bool((ref != 0).any()) and 2 * T + 9 < 1 << 24
    rs, gamma, gx = torch.ones(T, device="cuda"), torch.ones(n, device="cuda"), torch.empty_like(h)
    for acc in (False, True):
        dg = old.clone()
        L.skip_norm_bwd(h, gamma, rs, gy, gx, dg, accumulate=acc)
        assert torch.equal(dg.double(), ref + old.double() * acc)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("q8,g16,copy", [(True, False, True), (True, True, True), (True, False, False), (False, True, True),
                                         (False, False, True)])
def test_streamed_adamw(q8, g16, copy, offset):
    """Over 120 MB a step, aligned and not, whole chunks and tails, small tensors among them."""
    sizes = [3_000_001, 777, 256 * 12_000, 1, 2_500_003, 2048]
    say(f"streamed adamw q8={q8} g16={g16} copy={copy} offset={offset}")
    assert sum(sizes) * ((2 if g16 else 4) + 8 + (4 if q8 else 16) + 2 * copy) > 120 << 20
    L = lib()
    d = A.make(sizes, g16, q8, copy, seed=3, offset=offset)
    wd = [0.1, 0.0, 0.2, 0.1, 0.0, 0.3]
    P = A.plan(L, d, wd)
    out = torch.empty(2, device="cuda")
    L.grad_norm(P, 0.3, out)
    norm, f = S.grad_norm([f64(g) for g in d["g"]], 0.3)
    assert abs(float(out[0]) - norm) <= 1.01 * U * norm and abs(float(out[1]) - f) <= 1.01 * U * f
    A.step_and_check(L, d, P, wd, 1e-2, 3, gs=float(out[1]), grad_scale=out[1:])
