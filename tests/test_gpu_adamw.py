"""AdamW over many tensors and the gradient norm, against the float64 oracle.

Bounds (u = 2^-24).  Every operation is a float32 one and the constants are rounded to float32:
  m   4 u (b1 |m| + (1 - b1) |g|)       v   6 u v (all terms positive), and u^2-sized underflow
  p   3 u |p| + rate / den (e_m + 16 u |m|): sqrt(v), its product, eps, the division, the rate and
      the two constants behind them are at most 12 roundings on top of m's error e_m
  copy  half a bf16 step of p, on top of p's bound
8-bit states: what they stand for against the oracle's unrounded m and u = sqrt(v): half a step
  (2^-4 of the value, 2^-10 of the scale below the normals) and 2^-20 of it; a non-zero u below half
  the smallest code is that code: the error is at most 2^-9 of the scale.  scale: 2^-20.
"""
import numpy as np
import pytest
import torch

from gpu_helpers import f64, lib, say
from oracle import stage_oracle as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
B1, B2, EPS = 0.9, 0.95, 1e-8


def within(name, got, ref, bound):
    d = np.abs(got - ref)
    bad = ~(d <= bound)
    assert not bad.any(), (name, np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4], bound[bad][:4])


def make(sizes, g16=False, q8=False, copy=True, seed=0, offset=0):
    """Tensors of the given sizes, each starting `offset` elements into its allocation."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = {k: [] for k in ("p", "g", "m", "v", "m_scale", "v_scale", "copy")}

    def put(name, t):
        buf = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
        out[name].append(buf[offset:])
        buf[offset:].copy_(t)

    for i, k in enumerate(sizes):
        s = 10.0 ** (-(i % 4))
        grad = torch.randn(k, generator=g, device="cuda") * s
        put("p", torch.randn(k, generator=g, device="cuda"))
        put("g", grad.bfloat16() if g16 else grad)
        m = torch.randn(k, generator=g, device="cuda") * s * 0.3
        v = (torch.rand(k, generator=g, device="cuda") * s) ** 2
        if q8:
            for nm, t in (("m", m), ("v", v.sqrt())):
                nb = -(-k // 256)
                sc = torch.zeros(nb * 256, device="cuda")
                sc[:k] = t.abs()
                sc = (sc.view(nb, 256).amax(1) / 448).clamp(min=2.0 ** -126)
                put(nm, (t / sc.repeat_interleave(256)[:k]).to(torch.float8_e4m3fn).view(torch.uint8))
                out[nm][-1] = out[nm][-1].view(torch.float8_e4m3fn)
                out[nm + "_scale"].append(sc)
        else:
            put("m", m)
            put("v", v)
            out["m_scale"].append(None)
            out["v_scale"].append(None)
        put("copy", torch.zeros(k, device="cuda", dtype=torch.bfloat16))
        if not copy:
            out["copy"][-1] = None
    return out


def state(d, i):
    m, v = f64(d["m"][i].float()), f64(d["v"][i].float())
    if d["m_scale"][i] is not None:
        rep = lambda s: np.repeat(f64(s), 256)[:m.size]
        m, v = m * rep(d["m_scale"][i]), (v * rep(d["v_scale"][i])) ** 2
    return m, v


def plan(L, d, wd):
    return L.adamw_plan(d["p"], d["g"], d["m"], d["v"], m_scale=d["m_scale"], v_scale=d["v_scale"], copy=d["copy"],
                        weight_decay=wd)


def step_and_check(L, d, P, wd, lr, step, gs=None, **kw):
    n = len(d["p"])
    before = [(f64(d["p"][i]), f64(d["g"][i]), *state(d, i)) for i in range(n)]
    L.adamw_update(P, lr, step, betas=(B1, B2), eps=EPS, **kw)
    torch.cuda.synchronize()
    for i, (p, g, m, v) in enumerate(before):
        rp, rm, rv = S.adamw(p, g, m, v, lr, step, B1, B2, EPS, wd[i], 1.0 if gs is None else gs)
        g = np.abs(g * (1.0 if gs is None else gs))
        em = 4 * U * (B1 * np.abs(m) + (1 - B1) * g) + 2.0 ** -148
        den = np.sqrt(rv / (1 - B2 ** step)) + EPS
        ep = 3 * U * np.abs(p) + lr / (1 - B1 ** step) / den * (em + 16 * U * np.abs(rm)) + 2.0 ** -148
        within(f"p[{i}]", f64(d["p"][i]), rp, ep)
        if d["copy"][i] is not None:
            assert torch.equal(d["copy"][i], d["p"][i].bfloat16())
        if d["m_scale"][i] is None:
            within(f"m[{i}]", f64(d["m"][i]), rm, em)
            within(f"v[{i}]", f64(d["v"][i]), rv, 6 * U * rv + 2.0 ** -147)
            continue
        for nm, ref in (("m", rm), ("v", np.sqrt(rv))):
            sc = f64(d[nm + "_scale"][i])
            rs = S.scales(S.blocks(ref))
            within(f"{nm}_scale[{i}]", sc, rs, 2.0 ** -20 * rs)
            rep = np.repeat(sc, 256)[:ref.size]
            low = 2.0 ** -10 if nm == "m" else 2.0 ** -9
            q = f64(d[nm][i].float())
            within(f"{nm}8[{i}]", q * rep, ref, np.maximum(2.0 ** -4 * np.abs(ref), low * rep) * (1 + 2.0 ** -18)
                   + 2.0 ** -20 * np.abs(ref))
            if nm == "v":
                assert np.all((q > 0) == (ref > 0)) and np.all((q == 0) | (q >= S.TINY))


SIZES = [1, 3, 4, 5, 255, 256, 257, 511, 1023, 1024, 1025, 2047, 2048, 2049, 5000, 0, 12289, 7]


@pytest.mark.parametrize("variant", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1, 3, 4])
@pytest.mark.parametrize("g16", [False, True], ids=["g32", "g16"])
@pytest.mark.parametrize("q8", [False, True], ids=["s32", "s8"])
def test_two_steps(q8, g16, offset, variant):
    say(f"adamw q8={q8} g16={g16} offset={offset} {variant}")
    L = lib(variant)
    d = make(SIZES, g16, q8, seed=1, offset=offset)
    wd = [0.1 * (i % 3) for i in range(len(SIZES))]
    P = plan(L, d, wd)
    for s in (1, 2):
        step_and_check(L, d, P, wd, 1e-2, s)


def test_mixed_states_gradients_and_copies_in_one_plan():
    L = lib()
    parts = [make([777, 4096], False, False, True, 2), make([2050], True, True, False, 3, 1), make([1, 600], False, True, True, 4),
             make([9000], True, False, False, 5)]
    d = {k: sum((q[k] for q in parts), []) for k in parts[0]}
    wd = [0.0, 0.1, 0.2, 0.0, 0.1, 0.3]
    P = plan(L, d, wd)
    for s in (1, 7, 100000):
        step_and_check(L, d, P, wd, 3e-3, s)


def test_what_lies_around_the_tensors_stays():
    L = lib()
    for q8 in (False, True):
        bufs = {k: torch.full((3000,), 9.0, device="cuda").to(dt) for k, dt in
                (("p", torch.float32), ("m", torch.float8_e4m3fn if q8 else torch.float32),
                 ("v", torch.float8_e4m3fn if q8 else torch.float32), ("copy", torch.bfloat16))}
        sc = {k: torch.full((20,), 9.0, device="cuda") for k in ("ms", "vs")}
        lo, k = 101, 2051
        view = {n: [t[lo:lo + k]] for n, t in bufs.items()}
        g = torch.randn(k, device="cuda")
        more = dict(m_scale=[sc["ms"][3:3 + 9]], v_scale=[sc["vs"][3:3 + 9]]) if q8 else {}
        P = L.adamw_plan(view["p"], [g], view["m"], view["v"], copy=view["copy"], **more)
        L.adamw_update(P, 1e-2, 1)
        torch.cuda.synchronize()
        for n, t in bufs.items():
            t = t.float()
            assert bool((t[:lo] == 9).all()) and bool((t[lo + k:] == 9).all())
            # 8-bit states: p moves by 0.02, which bf16 (a step of 2^-4 below 9) rounds back to 9
            assert torch.equal(t, bufs["p"].bfloat16().float()) if n == "copy" else bool((t[lo:lo + k] != 9).any())
        if q8:
            for t in sc.values():
                assert bool((t[:3] == 9).all()) and bool((t[12:] == 9).all()) and bool((t[3:12] != 9).all())


def test_many_tensors_and_chunks():
    L = lib()
    sizes = [(37 * i) % 4099 + 1 for i in range(400)] + [3_000_001]
    d = make(sizes, seed=6)
    P = plan(L, d, [0.1] * len(sizes))
    step_and_check(L, d, P, [0.1] * len(sizes), 1e-3, 4)
    q = make(sizes, q8=True, seed=6)
    step_and_check(L, q, plan(L, q, [0.1] * len(sizes)), [0.1] * len(sizes), 1e-3, 4)


def test_a_tensor_beyond_32_bit_offsets():
    """2^30 + 77 elements: float32 byte offsets pass 4 GiB; ends and a middle stretch are checked."""
    L = lib()
    k = (1 << 30) + 77
    t = {n: torch.empty(k, device="cuda") for n in ("p", "g", "m", "v")}
    t["p"].normal_(), t["g"].normal_(), t["m"].zero_(), t["v"].zero_()
    pick = torch.cat([torch.arange(3000), torch.arange((1 << 29) - 1500, (1 << 29) + 1500), torch.arange(k - 3000, k)]).cuda()
    before = {n: f64(x[pick]) for n, x in t.items()}
    P = L.adamw_plan([t["p"]], [t["g"]], [t["m"]], [t["v"]], weight_decay=0.1)
    L.adamw_update(P, 1e-2, 1, betas=(B1, B2), eps=EPS)
    rp, rm, rv = S.adamw(before["p"], before["g"], before["m"], before["v"], 1e-2, 1, B1, B2, EPS, 0.1)
    within("p", f64(t["p"][pick]), rp, 4 * U * np.abs(before["p"]) + 0.1 * 32 * U)
    within("m", f64(t["m"][pick]), rm, 4 * U * np.abs(before["g"]))
    within("v", f64(t["v"][pick]), rv, 6 * U * rv)
    out = torch.empty(2, device="cuda")
    L.grad_norm(P, 1.0, out)
    ref = float(torch.linalg.vector_norm(t["g"], dtype=torch.float64))
    assert abs(float(out[0]) - ref) <= 2 * U * ref


def test_zero_gradients_and_states():
    """Nothing but decay, and 8-bit states of zeros that stay zeros."""
    L = lib()
    for q8 in (False, True):
        d = make([1000], q8=q8, seed=7)
        for n in ("g", "m", "v"):
            d[n][0].view(torch.uint8).zero_()
        p = d["p"][0].clone()
        L.adamw_update(plan(L, d, [0.5]), 0.1, 3)
        assert torch.equal(d["p"][0], p * np.float32(0.95))
        assert not bool(d["m"][0].view(torch.uint8).any()) and not bool(d["v"][0].view(torch.uint8).any())


def test_roots_that_are_small_beside_their_block():
    """A first step with gradients over twelve decades: no element moves further than lr (1 + a half step)
    at the next one, as its own gradient alone would have it."""
    L = lib()
    g = torch.logspace(-12, 0, 256, device="cuda")
    d = make([256], q8=True, seed=8)
    for n in ("m", "v"):
        d[n][0].view(torch.uint8).zero_()
    d["g"][0].copy_(g)
    P = plan(L, d, [0.0])
    step_and_check(L, d, P, [0.0], 1e-3, 1)
    before = d["p"][0].clone()
    d["g"][0].zero_()
    L.adamw_update(P, 1e-3, 2, betas=(B1, B2), eps=EPS)
    # m <= 7 u before the rounding (b1 and b2 as here: 0.1 g against sqrt(0.05) g), each rounded by at most
    # its half step, u upwards only below the smallest code
    assert float((d["p"][0] - before).abs().max()) <= 1e-3 * 2


def test_clip_factor_and_skip():
    L = lib()
    d = make([5000, 31], seed=9)
    P = plan(L, d, [0.1, 0.0])
    out = torch.empty(2, device="cuda")
    L.grad_norm(P, 0.5, out)
    norm, f = S.grad_norm([f64(g) for g in d["g"]], 0.5)
    assert abs(float(out[0]) - norm) <= 2 * U * norm and abs(float(out[1]) - f) <= 2 * U * f
    step_and_check(L, d, P, [0.1, 0.0], 1e-2, 5, gs=float(out[1]), grad_scale=out[1:])
    for bad in (float("inf"), float("nan")):
        d["g"][1][30] = bad
        L.grad_norm(P, 0.5, out)
        keep = [t.clone() for k in ("p", "m", "v", "copy") for t in d[k]]
        L.adamw_update(P, 1e-2, 6, grad_scale=out[1:])
        torch.cuda.synchronize()
        assert bool(out[1].isnan())
        assert all(torch.equal(a, b) for a, b in zip(keep, [t for k in ("p", "m", "v", "copy") for t in d[k]]))


def test_nonfinite_gradient_without_a_norm():
    L = lib()
    for q8 in (False, True):
        d = make([1024], q8=q8, seed=10)
        d["g"][0][300] = float("nan")
        L.adamw_update(plan(L, d, [0.0]), 1e-2, 1)
        nan = d["p"][0].isnan()
        assert int(nan.sum()) == 1 and bool(nan[300])
        m, _ = state(d, 0)
        bad = np.isnan(m)
        assert bad[300] and (bad[256:512].all() and bad.sum() == 256 if q8 else bad.sum() == 1)


@pytest.mark.parametrize("g16", [False, True])
@pytest.mark.parametrize("sizes", [[1], [5, 0, 3], SIZES, [(37 * i) % 4099 + 1 for i in range(700)], [6_000_003, 17]],
                         ids=["one", "three", "edges", "many", "long"])
def test_grad_norm(sizes, g16):
    L = lib()
    for offset in (0, 1):
        d = make([max(s, 1) for s in sizes], g16, seed=11, offset=offset)["g"]
        d = [g[:s] for g, s in zip(d, sizes)]
        P = L.grad_plan(d)
        out = torch.empty(2, device="cuda")
        for mx in (1e-3, 1e9, float("inf")):
            L.grad_norm(P, mx, out)
            norm, f = S.grad_norm([f64(g) for g in d], mx)
            # float64 sums, rounded once; the factor's float64 value too
            assert abs(float(out[0]) - norm) <= 1.01 * U * norm and abs(float(out[1]) - f) <= 1.01 * U * f


def test_grad_norm_around_the_chunks_that_take_one_launch():
    """One chunk a tensor or sixteen in one, plus and minus one, gradients of a plan with states among them."""
    L = lib()
    out = torch.empty(2, device="cuda")
    for count, size in ((15, 700), (16, 4096), (17, 4096), (16, 1), (17, 3), (1, 16 * 4096), (1, 16 * 4096 + 1), (1, 4097)):
        for g16 in (False, True):
            d = make([size] * count, g16, seed=count)
            for P in (L.grad_plan(d["g"]), plan(L, d, [0.0] * count)):
                L.grad_norm(P, 2.0, out)
                norm, f = S.grad_norm([f64(g) for g in d["g"]], 2.0)
                assert abs(float(out[0]) - norm) <= 1.01 * U * norm and abs(float(out[1]) - f) <= 1.01 * U * f
    d = make([512] * 5, seed=3)
    d["g"][4][511] = float("nan")
    L.grad_norm(L.grad_plan(d["g"]), 1.0, out)
    assert bool(out.isnan().all())


def test_grad_norm_of_nothing_zeros_and_large_values():
    L = lib()
    out = torch.empty(2, device="cuda")
    L.grad_norm(L.grad_plan([]), 1.0, out)
    assert out.tolist() == [0.0, 1.0]
    L.grad_norm(L.grad_plan([torch.zeros(100, device="cuda")]), 1.0, out)
    assert out.tolist() == [0.0, 1.0]
    L.grad_norm(L.grad_plan([torch.full((4,), 1e30, device="cuda")]), 1.0, out)  # squares beyond float32
    assert abs(float(out[0]) - 2e30) <= 2e30 * 2 * U and abs(float(out[1]) - 5e-31) <= 5e-31 * 4 * U


def test_captured_step_follows_device_lr_and_step():
    """Clip factor and step in one graph, replayed with other learning rates, steps and gradients, eager
    work in between; each replay against the eager calls on a copy."""
    L = lib()
    for q8 in (False, True):
        a, b = (make(SIZES, q8=q8, seed=12) for _ in range(2))
        wd = [0.1] * len(SIZES)
        P, Q = plan(L, a, wd), plan(L, b, wd)
        hyp = torch.tensor([1e-3, 1.0], dtype=torch.float64, device="cuda")
        out, out2, ws = torch.empty(2, device="cuda"), torch.empty(2, device="cuda"), L.grad_norm_workspace(P)
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            L.grad_norm(P, 0.25, out, ws=ws)
            L.adamw_update(P, grad_scale=out[1:], lr_step=hyp)
        torch.cuda.synchronize()
        for rep in range(1, 5):
            lr = 1e-3 * rep
            hyp.copy_(torch.tensor([lr, float(rep)], dtype=torch.float64))
            for x, y in zip(a["g"], b["g"]):
                x.mul_(1.5)
                y.mul_(1.5)
            ws.fill_(0x5A)
            torch.cuda.synchronize()
            graph.replay()
            L.grad_norm(Q, 0.25, out2)
            L.adamw_update(Q, lr, rep, grad_scale=out2[1:])
            torch.cuda.synchronize()
            assert torch.equal(out, out2)
            for k in ("p", "m", "v", "copy"):
                for x, y in zip(a[k], b[k]):
                    assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), (rep, k)


def test_same_results_whatever_the_alignment():
    L = lib()
    res = []
    for offset in (0, 1):
        d = make([4000], q8=True, seed=13, offset=offset)
        L.adamw_update(plan(L, d, [0.1]), 1e-2, 3)
        res.append([d[k][0].view(torch.uint8).clone() for k in ("m", "v")] + [d["p"][0].clone(), d["m_scale"][0], d["v_scale"][0]])
    assert all(torch.equal(x, y) for x, y in zip(*res))
