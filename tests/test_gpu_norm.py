"""The residual addition with its RMS norm, 16- and 8-bit output, and its backward, against the
float64 oracle.

Bounds, all counted from roundings (u = 2^-24, float32; a stored act adds half a step, 2^-8 of
the value in bf16, u in float32).
  h     three terms added in float32: 2 u (|x| + |res| + |b|), and the store.
  rstd  the float32 sum of n squares in any order of at most 64 terms a lane and a tree of 16
        levels has relative error under 80 u + u; half of it passes the root; eps, division and
        root add three: under 64 u = 2^-18.
  y     against the oracle on the op's own h: rstd's 2^-18, two products, and the store.
  scale y's error before its store, and one division: 2^-17.
  code  half a step of e4m3 (2^-4 of the value, 2^-10 of the scale below the normals), moved by the
        errors of y, scale and the product with 1 / scale: 2^-16 of the value.
  g_x   c is a float32 sum of n products: at most (80 + 4) u of mean |w xh|; the few operations
        around it add under 8 u of each term: 128 u (rstd (|w| + |xh| mean |w xh|) + |g_h|), and the store.
  dgamma  a float32 sum of T products in any order: (T + 4) u sum |g_y xh|, and u of an old value.
"""
import numpy as np
import pytest
import torch

from gpu_helpers import f64, guarded, lib, say, strided
from oracle import stage_oracle as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5


def store(io):
    return 2.0 ** -8 if io == torch.bfloat16 else U


def inputs(T, n, r, io, seed, spread=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    tok = torch.exp(rn(T, 1)) if spread else 1.0
    return {"x": (rn(T, n) * tok).to(io), "res": (rn(T, n) * tok).to(io), "b": rn(T, r).to(io) if r else None,
            "gamma": 1 + 0.1 * rn(n), "gy": (0.1 * rn(T, n)).to(io), "gh": (0.1 * rn(T, n)).to(io)}


def within(name, got, ref, bound):
    d = np.abs(f64(got) - ref)
    bad = ~(d <= bound)
    say(f"    {name}: worst {np.max(d / np.maximum(bound, 1e-300)) if d.size else 0:.3f} of the bound")
    assert not bad.any(), (name, np.argwhere(bad)[:4], f64(got)[bad][:4], ref[bad][:4])


def check_h(d, h, io, res, b):
    x, rs, bb = f64(d["x"]), f64(d["res"]) if res else 0.0, 0.0
    ref = S.stream(d["x"].cpu().double().numpy(), f64(d["res"]) if res else None, f64(d["b"]) if b else None)
    if b:
        bb = np.zeros_like(x)
        bb[:, :d["b"].shape[1]] = np.abs(f64(d["b"]))
    within("h", h, ref, store(io) * np.abs(ref) * (1 + 2.0 ** -8) + 3 * U * (np.abs(x) + np.abs(rs) + bb) + 2.0 ** -133)


SHAPES = [(1, 8, 0), (1, 8, 8), (3, 64, 4), (5, 504, 20), (7, 512, 512), (4, 520, 12), (129, 1000, 0), (2, 1032, 36),
          (1, 4096, 32), (33, 2048, 16), (6, 2056, 100), (9, 4096, 32), (3, 4104, 64), (2, 8192, 64), (2, 8200, 8),
          (3, 16384, 0), (1, 16392, 128), (2, 32768, 4), (2, 32776, 256), (2, 65536, 64)]
IDS = ["x".join(map(str, s)) for s in SHAPES]


@pytest.mark.parametrize("variant", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_forward(shape, variant):
    T, n, r = shape
    say(f"norm forward {variant} T={T} n={n} r={r}")
    L = lib(variant)
    io = L.io_dtype
    d = inputs(T, n, r, io, 1)
    for res, pad in ((True, 8), (False, 0)):
        x, rs = strided(d["x"], pad), strided(d["res"], pad) if res else None
        h, _, hg = guarded((T, n), io, "cuda", pad=pad)
        y, _, yg = guarded((T, n), io, "cuda", pad=pad)
        rstd = torch.full((T,), float("nan"), device="cuda")
        L.skip_norm_fwd(x, d["gamma"], y, res=rs, b=d["b"], h=h, rstd=rstd, eps=EPS)
        torch.cuda.synchronize()
        hg(), yg()
        check_h(d, h, io, res, r > 0)
        hs = f64(h)
        ref = S.rstd(hs, EPS)
        within("rstd", rstd, ref, 2.0 ** -18 * ref)
        ry = S.norm(hs, f64(d["gamma"]), EPS)
        within("y", y, ry, (store(io) + 2.0 ** -17) * np.abs(ry) + 2.0 ** -133)
        y2 = torch.empty_like(y)
        L.skip_norm_fwd(x, d["gamma"], y2, res=rs, b=d["b"], eps=EPS)  # h and rstd not written: the same y
        assert torch.equal(y, y2)


@pytest.mark.parametrize("variant", ["bf16", "f32"])
@pytest.mark.parametrize("shape,group", [((1, 8, 0), 8), ((5, 504, 20), 504), ((3, 64, 4), 32), ((1, 64, 4), 64), ((9, 2112, 20), 64),
                                         ((33, 2048, 16), 128), ((7, 2048, 16), 2048), ((4, 512, 0), 256), ((3, 4096, 32), 256),
                                         ((1, 4096, 32), 4096), ((2, 8192, 64), 128), ((2, 8224, 8), 32), ((3, 16384, 0), 16384),
                                         ((2, 32768, 4), 64), ((1, 65536, 64), 256), ((1, 65536, 64), 65536), ((2, 264, 4), 264)])
def test_forward_8bit(shape, group, variant):
    T, n, r = shape
    say(f"norm 8 bits {variant} T={T} n={n} r={r} group={group}")
    L = lib(variant)
    d = inputs(T, n, r, L.io_dtype, 2)
    buf = torch.full((T, n + 8), 0x55, dtype=torch.uint8, device="cuda")
    y = buf.view(torch.float8_e4m3fn)[:, :n]
    scale = torch.full((T, n // group), float("nan"), device="cuda")
    h, rstd = torch.empty(T, n, dtype=L.io_dtype, device="cuda"), torch.empty(T, device="cuda")
    L.skip_norm_q8_fwd(d["x"], d["gamma"], y, scale, res=d["res"], b=d["b"], h=h, rstd=rstd, eps=EPS)
    torch.cuda.synchronize()
    assert bool((buf[:, n:] == 0x55).all())
    check_h(d, h, L.io_dtype, True, r > 0)
    ry = S.norm(f64(h), f64(d["gamma"]), EPS)
    rs = S.scales(ry.reshape(T, -1, group))
    within("scale", scale, rs, 2.0 ** -17 * rs)
    sc = np.repeat(f64(scale), group, axis=1)
    back = f64(y.float()) * sc
    within("y", torch.from_numpy(back), ry, np.maximum(2.0 ** -4 * np.abs(ry), 2.0 ** -10 * sc) * (1 + 2.0 ** -10)
           + 2.0 ** -16 * np.abs(ry))
    assert np.abs(f64(y.float())).max() == 448.0


@pytest.mark.parametrize("variant", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES + [(300, 512, 0), (1111, 264, 0), (517, 2112, 0), (130, 4096, 0)],
                         ids=lambda s: "x".join(map(str, s)))
def test_backward(shape, variant):
    T, n, _ = shape
    say(f"norm backward {variant} T={T} n={n}")
    L = lib(variant)
    io = L.io_dtype
    d = inputs(T, n, 0, io, 3)
    rs = torch.from_numpy(S.rstd(f64(d["x"]), EPS)).float().cuda()
    H, G, R_, GY, GH = f64(d["x"]), f64(d["gamma"]), f64(rs), f64(d["gy"]), f64(d["gh"])
    old = torch.randn(n, generator=torch.Generator().manual_seed(5)).cuda()
    xh, w = H * R_[:, None], GY * G
    terms = R_[:, None] * (np.abs(w) + np.abs(xh) * np.mean(np.abs(w * xh), axis=1, keepdims=True))
    for gh, acc, pad, place in ((True, False, 8, None), (False, True, 0, None), (True, True, 0, "g_y"), (True, False, 0, "g_h")):
        h, gy, ghv = strided(d["x"], pad), strided(d["gy"], pad), strided(d["gh"], pad) if gh else None
        out, check = {"g_y": gy, "g_h": ghv}.get(place), None
        if out is None:
            out, _, check = guarded((T, n), io, "cuda", pad=pad)
        dg = old.clone() if acc else torch.full((n,), float("nan"), device="cuda")
        L.skip_norm_bwd(h, d["gamma"], rs, gy, out, dg, g_h=ghv, accumulate=acc)
        torch.cuda.synchronize()
        if check:
            check()
        gx, dgam = S.norm_bwd(H, G, R_, GY, GH if gh else None)
        within("g_x", out, gx, store(io) * np.abs(gx) + 128 * U * (terms + (np.abs(GH) if gh else 0)) + 2.0 ** -133)
        ref = dgam + (f64(old) if acc else 0)
        within("dgamma", dg, ref, (T + 4) * U * np.sum(np.abs(GY * xh), axis=0) + 2 * U * np.abs(ref) + 2.0 ** -133)


def test_backward_against_differences():
    """The float32 build's own forward, in differences: dL along random directions."""
    L = lib("f32")
    T, n = 5, 72
    d = inputs(T, n, 0, torch.float32, 6, spread=False)
    y, rs = torch.empty(T, n, device="cuda"), torch.empty(T, device="cuda")
    L.skip_norm_fwd(d["x"], d["gamma"], y, rstd=rs, eps=EPS)
    gx, dg = torch.empty(T, n, device="cuda"), torch.empty(n, device="cuda")
    L.skip_norm_bwd(d["x"], d["gamma"], rs, d["gy"], gx, dg)
    H, G, GY = f64(d["x"]), f64(d["gamma"]), f64(d["gy"])
    rng = np.random.default_rng(7)
    for _ in range(4):
        dh, dga = rng.standard_normal((T, n)), rng.standard_normal(n)
        s = 1e-6
        num = np.sum(GY * (S.norm(H + s * dh, G + s * dga, EPS) - S.norm(H - s * dh, G - s * dga, EPS))) / (2 * s)
        ana = np.sum(f64(gx) * dh) + np.sum(f64(dg) * dga)
        # g_x and dgamma carry 128 u and (T + 4) u of terms of size 0.1; 1e-7 of the differences' own error
        assert abs(num - ana) <= 128 * U * 0.1 * 8 * T * n + 1e-6


@pytest.mark.parametrize("which", ["x", "res"])
def test_stream_in_place(which):
    L = lib()
    for T, n, r in ((5, 2056, 8), (3, 512, 4), (2, 16392, 4)):
        d = inputs(T, n, r, L.io_dtype, 8)
        h, y, y2 = torch.empty_like(d["x"]), torch.empty_like(d["x"]), torch.empty_like(d["x"])
        L.skip_norm_fwd(d["x"], d["gamma"], y, res=d["res"], b=d["b"], h=h)
        L.skip_norm_fwd(d["x"], d["gamma"], y2, res=d["res"], b=d["b"], h=d[which])
        torch.cuda.synchronize()
        assert torch.equal(d[which], h) and torch.equal(y, y2)


def test_many_rows():
    """More rows than one launch has blocks for, the last rows among them; and rows behind T stay as they were."""
    L = lib()
    T, n = (1 << 22) + 4100, 8
    x = torch.randn(T + 3, n, device="cuda").bfloat16()
    g = torch.ones(n, device="cuda")
    y, rs = torch.full_like(x, 7.0), torch.full((T,), -1.0, device="cuda")
    L.skip_norm_fwd(x[:T], g, y[:T], rstd=rs)
    xf = x[:T].float()
    ref = torch.rsqrt((xf * xf).mean(1) + EPS)
    assert bool(((rs - ref).abs() <= 2.0 ** -17 * ref).all()) and bool((y[T:] == 7.0).all())
    assert bool(((y[:T].float() - xf * ref[:, None]).abs() <= 2.0 ** -7 * (xf * ref[:, None]).abs()).all())
    gx, dg = torch.full_like(x, 7.0), torch.empty(n, device="cuda")
    L.skip_norm_bwd(x[:T], g, rs, y[:T], gx[:T], dg)
    xh = xf.double() * rs.double()[:, None]
    ref = (y[:T].double() * xh).sum(0)
    assert bool(((dg.double() - ref).abs() <= T * U * (y[:T].double() * xh).abs().sum(0)).all())
    assert bool((gx[T:] == 7.0).all())
    w = y[:T].double()
    rx = rs.double()[:, None] * (w - xh * (w * xh).mean(1, keepdim=True))
    lim = 2.0 ** -8 * rx.abs() + 128 * U * rs.double()[:, None] * (w.abs() + xh.abs() * (w * xh).abs().mean(1, keepdim=True))
    assert bool(((gx[:T].double() - rx).abs() <= lim).all())


def test_offsets_beyond_32_bits():
    """Rows so far apart that byte offsets pass 4 GiB."""
    L = lib()
    T, n, ld = 5, 64, (1 << 29) + 64
    x = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda").view(T, ld)[:, :n]
    v = torch.randn(T, n, device="cuda").bfloat16()
    x.copy_(v)
    g, y, y2 = torch.ones(n, device="cuda"), torch.empty(T, n, dtype=torch.bfloat16, device="cuda"), None
    L.skip_norm_fwd(x, g, y)
    y2 = torch.empty_like(y)
    L.skip_norm_fwd(v, g, y2)
    assert torch.equal(y, y2)
    q, s = torch.empty(T, n, device="cuda").to(torch.float8_e4m3fn), torch.empty(T, 2, device="cuda")
    L.skip_norm_q8_fwd(x, g, q, s, h=x, res=x)  # the stream doubled in place
    assert torch.equal(x, v + v)
    rs = torch.ones(T, device="cuda")
    gx, gx2, dg, dg2 = torch.empty_like(y), torch.empty_like(y), torch.empty_like(g), torch.empty_like(g)
    L.skip_norm_bwd(x, g, rs, y, gx, dg)
    L.skip_norm_bwd((v + v).contiguous(), g, rs, y, gx2, dg2)
    assert torch.equal(gx, gx2) and torch.equal(dg, dg2)


def test_zeros_infinities_and_nans():
    L = lib()
    T, n = 6, 256
    x = torch.randn(T, n, device="cuda").bfloat16()
    x[0] = 0
    x[1, 5] = float("nan")
    x[2, 7] = float("inf")
    x[3] = 1e-30
    x[4] = 1e30  # mean square beyond float32: rstd = 0
    g = torch.ones(n, device="cuda")
    y, rs = torch.empty_like(x), torch.empty(T, device="cuda")
    L.skip_norm_fwd(x, g, y, rstd=rs, eps=EPS)
    torch.cuda.synchronize()
    y, rs = y.float().cpu(), rs.cpu()
    assert bool((y[0] == 0).all()) and rs[0] == np.float32(1.0) / np.sqrt(np.float32(EPS))
    assert bool(y[1].isnan().all()) and bool(rs[1].isnan())
    assert bool(y[2, 7].isnan()) and bool((y[2].nan_to_num(0.0) == 0).all()) and rs[2] == 0
    assert bool((y[3] != 0).all()) and bool((y[4] == 0).all()) and bool(y[5].isfinite().all())
    for group in (32, 256):
        q, s = torch.empty(T, n, device="cuda").to(torch.float8_e4m3fn), torch.empty(T, n // group, device="cuda")
        L.skip_norm_q8_fwd(x, g, q, s, eps=EPS)
        back = (q.float() * s.repeat_interleave(group, 1)).cpu()
        assert bool((back[0] == 0).all()) and s[0, 0] == 2.0 ** -126 and bool(back[1].isnan().all())
        assert bool(back[2, :group].isnan().all()) and bool((back[2, group:] == 0).all())
        assert bool(back[5].isfinite().all())


def test_eps_zero_and_the_gain():
    L = lib("f32")
    x = torch.full((2, 64), 3.0, device="cuda")
    g = torch.arange(64, device="cuda", dtype=torch.float32)
    y = torch.empty_like(x)
    L.skip_norm_fwd(x, g, y, eps=0.0)
    assert bool(((y - g).abs() <= 2.0 ** -20 * g).all())


def test_other_stream_and_no_workspace_race():
    """Two calls at once on two streams with workspaces of their own, against the same calls alone."""
    L = lib()
    d = [inputs(700, 1024, 0, L.io_dtype, s) for s in (11, 12)]
    rs = [torch.rsqrt((e["x"].float() ** 2).mean(1) + EPS) for e in d]
    alone, both = [], []
    for e, r in zip(d, rs):
        gx, dg = torch.empty_like(e["x"]), torch.empty(1024, device="cuda")
        L.skip_norm_bwd(e["x"], e["gamma"], r, e["gy"], gx, dg, g_h=e["gh"])
        alone.append((gx, dg))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(5):
        both = []
        for e, r, s in zip(d, rs, streams):
            gx, dg = torch.empty_like(e["x"]), torch.empty(1024, device="cuda")
            ws = L.norm_workspace(700, 1024, "cuda")
            torch.cuda.synchronize()
            L.skip_norm_bwd(e["x"], e["gamma"], r, e["gy"], gx, dg, g_h=e["gh"], ws=ws, stream=s)
            both.append((gx, dg, ws))
        torch.cuda.synchronize()
        for a, b in zip(alone, both):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_no_rows_and_host_tensors():
    """T = 0 is no work (dgamma stays), and a host tensor among the operands is refused, native path or not."""
    L = lib()
    n = 64
    x, g = torch.zeros(0, n, dtype=torch.bfloat16, device="cuda"), torch.ones(n, device="cuda")
    dg = torch.full((n,), 3.0, device="cuda")
    L.skip_norm_fwd(x, g, torch.zeros_like(x), rstd=torch.zeros(0, device="cuda"))
    L.skip_norm_q8_fwd(x, g, x.to(torch.float8_e4m3fn), torch.zeros(0, 2, device="cuda"))
    L.skip_norm_bwd(x, g, torch.zeros(0, device="cuda"), x, torch.zeros_like(x), dg)
    torch.cuda.synchronize()
    assert bool((dg == 3.0).all())
    x = torch.ones(4, n, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    with pytest.raises(ValueError, match="one GPU"):
        L.skip_norm_fwd(x, g.cpu(), y)
    with pytest.raises(ValueError, match="one GPU"):
        L.skip_norm_fwd(x, g, y, res=x.cpu())
    with pytest.raises(ValueError, match="one GPU"):
        L.skip_norm_bwd(x, g, torch.ones(4, device="cuda"), x, y, dg, ws=torch.zeros(1 << 16, dtype=torch.uint8))


@pytest.mark.parametrize("T", [2, 3, 4, 5])
def test_backward_of_few_wide_rows_is_one_block_or_many(T):
    """Around the row count from which dgamma takes a second launch, on a workspace of the smallest size."""
    L = lib()
    for n in (2056, 4096, 16384):
        d = inputs(T, n, 0, L.io_dtype, 30 + T)
        rs = torch.rsqrt((d["x"].float() ** 2).mean(1) + EPS)
        H, G, R_, GY = f64(d["x"]), f64(d["gamma"]), f64(rs), f64(d["gy"])
        old = torch.randn(n, device="cuda")
        for acc in (False, True):
            dg, gx = old.clone(), torch.empty_like(d["x"])
            L.skip_norm_bwd(d["x"], d["gamma"], rs, d["gy"], gx, dg, accumulate=acc, ws=L.norm_workspace(T, n, "cuda"))
            _, ref = S.norm_bwd(H, G, R_, GY)
            ref = ref + (f64(old) if acc else 0)
            within("dgamma", dg, ref, (T + 4) * U * np.sum(np.abs(GY * H * R_[:, None]), axis=0) + 2 * U * np.abs(ref) + 2.0 ** -133)


@pytest.mark.parametrize("T", [1, 8, 128, 129, 192, 193, 256, 257, 600])
def test_backward_around_the_rows_that_take_one_launch(T):
    """dgamma beside the rows, or from partial sums: the bounds hold, and g_x in g_y's or g_h's place
    gives the same bits."""
    L = lib()
    for n in (128, 512, 1024, 1544, 4096, 16392):
        d = inputs(T, n, 0, L.io_dtype, 40 + T)
        rs = torch.rsqrt((d["x"].float() ** 2).mean(1) + EPS)
        out = []
        for place in (None, "gy", "gh"):
            e = {k: d[k].clone() for k in ("gy", "gh")}
            gx = torch.empty_like(d["x"]) if place is None else e[place]
            dg = torch.full((n,), 2.0, device="cuda")
            L.skip_norm_bwd(d["x"], d["gamma"], rs, e["gy"], gx, dg, g_h=e["gh"], accumulate=True)
            out.append((gx, dg))
        for gx, dg in out[1:]:
            assert torch.equal(gx, out[0][0]) and torch.equal(dg, out[0][1])
        H, G, R_, GY, GH = f64(d["x"]), f64(d["gamma"]), f64(rs), f64(d["gy"]), f64(d["gh"])
        gx, ref = S.norm_bwd(H, G, R_, GY, GH)
        xh, w = H * R_[:, None], GY * G
        terms = R_[:, None] * (np.abs(w) + np.abs(xh) * np.mean(np.abs(w * xh), axis=1, keepdims=True)) + np.abs(GH)
        within("g_x", out[0][0], gx, store(L.io_dtype) * np.abs(gx) + 128 * U * terms + 2.0 ** -133)
        within("dgamma", out[0][1], ref + 2, (T + 4) * U * np.sum(np.abs(GY * xh), axis=0) + 2 * U * np.abs(ref + 2))


def test_workspace_of_a_call_on_another_stream():
    """Without a workspace argument, on a stream that is still busy, by object and by handle: what the caller's
    stream allocates and writes meanwhile does not reach the sums."""
    L = lib()
    T, n = 2000, 2048
    d = inputs(T, n, 0, L.io_dtype, 50)
    rs = torch.rsqrt((d["x"].float() ** 2).mean(1) + EPS)
    ref, gx = torch.empty(n, device="cuda"), torch.empty_like(d["x"])
    L.skip_norm_bwd(d["x"], d["gamma"], rs, d["gy"], gx, ref)
    P, out, norm = L.grad_plan([d["gamma"]] * 40), torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    L.grad_norm(P, 1.0, norm)
    torch.cuda.synchronize()
    size = L.norm_workspace(T, n, "cuda").numel() + 256
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        dg = torch.empty(n, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(2_000_000)
        L.skip_norm_bwd(d["x"], d["gamma"], rs, d["gy"], gx, dg, stream=stream)
        L.grad_norm(P, 1.0, out, stream=stream)
        for _ in range(200):
            torch.empty(size, dtype=torch.uint8, device="cuda").fill_(0xFF)
        torch.cuda.synchronize()
        assert torch.equal(dg, ref) and torch.equal(out, norm)
