"""Refusals of the residual norm, of the AdamW plan and step, and of the gradient norm: every
call here is turned away by host checks before any HIP call, or is a host query.  The addresses
are made up, so the file is skipped where a GPU is visible."""
import ctypes
import os

import pytest
import torch

from paper_2604_11947_amd import build as B
from paper_2604_11947_amd import resbm as R

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up device addresses")

A = 0x10000000
T, N, RR = 64, 256, 32


@pytest.fixture(scope="module", params=["bf16", "f32"])
def lib(request):
    if not os.path.exists(B.lib_path(request.param)):
        B.build_all()
    return R.Library(request.param)


def args(names, vals, over):
    vals = list(vals)
    for k, v in over.items():
        vals[names.index(k)] = v
    return vals


FWD = ["T", "n", "r", "x", "ldx", "res", "ldr", "b", "gamma", "eps", "h", "ldh", "y", "ldy", "rstd", "s"]
FWD_V = [T, N, RR, A, N, 2 * A, N, 3 * A, 4 * A, 1e-5, 5 * A, N, 6 * A, N, 7 * A, None]
NAN = float("nan")

COMMON = [
    (dict(T=-1), R.E_SHAPE), (dict(T=1 << 31), R.E_SHAPE), (dict(n=4), R.E_SHAPE), (dict(n=0), R.E_SHAPE),
    (dict(n=260), R.E_SHAPE), (dict(n=65544, ldx=65544, ldr=65544, ldh=65544, ldy=65544), R.E_SHAPE),
    (dict(r=-4), R.E_SHAPE), (dict(r=6), R.E_SHAPE), (dict(r=260), R.E_SHAPE), (dict(eps=-1e-5), R.E_SHAPE),
    (dict(eps=NAN), R.E_SHAPE), (dict(eps=float("inf")), R.E_SHAPE),
    (dict(x=None), R.E_NULL), (dict(gamma=None), R.E_NULL), (dict(y=None), R.E_NULL), (dict(b=None), R.E_NULL),
    (dict(ldx=N - 8), R.E_SHAPE), (dict(ldr=N + 4), R.E_SHAPE), (dict(ldh=N - 8), R.E_SHAPE), (dict(ldy=N + 2), R.E_SHAPE),
    (dict(x=A + 8), R.E_ALIGN), (dict(res=2 * A + 2), R.E_ALIGN), (dict(b=3 * A + 8), R.E_ALIGN),
    (dict(gamma=4 * A + 4), R.E_ALIGN), (dict(h=5 * A + 8), R.E_ALIGN), (dict(y=6 * A + 8), R.E_ALIGN),
    (dict(rstd=7 * A + 2), R.E_ALIGN),
    (dict(y=A), R.E_ALIAS), (dict(y=2 * A), R.E_ALIAS), (dict(y=5 * A), R.E_ALIAS), (dict(h=A + 16), R.E_ALIAS),
    (dict(h=A, ldh=N + 8), R.E_ALIAS), (dict(h=3 * A), R.E_ALIAS), (dict(rstd=4 * A), R.E_ALIAS), (dict(rstd=5 * A + 64), R.E_ALIAS),
    (dict(y=3 * A), R.E_ALIAS),
]


@pytest.mark.parametrize("over,status", COMMON)
def test_norm_forward_refusals(lib, over, status):
    assert lib.cdll.resbm_skip_norm_fwd(*args(FWD, FWD_V, over)) == status


Q8 = FWD[:3] + ["group"] + FWD[3:14] + ["scale", "rstd", "s"]
Q8_V = FWD_V[:3] + [64] + FWD_V[3:14] + [8 * A, 7 * A, None]


@pytest.mark.parametrize("over,status", COMMON + [
    (dict(group=0), R.E_SHAPE), (dict(group=-1), R.E_SHAPE), (dict(group=16), R.E_SHAPE), (dict(group=48), R.E_SHAPE),
    (dict(group=512), R.E_SHAPE), (dict(n=96, r=0, group=64), R.E_SHAPE), (dict(scale=None), R.E_NULL),
    (dict(scale=8 * A + 2), R.E_ALIGN), (dict(scale=6 * A), R.E_ALIAS), (dict(scale=7 * A), R.E_ALIAS), (dict(scale=A), R.E_ALIAS),
])
def test_norm_8bit_refusals(lib, over, status):
    assert lib.cdll.resbm_skip_norm_q8_fwd(*args(Q8, Q8_V, over)) == status


BWD = ["T", "n", "h", "ldh", "gamma", "rstd", "gy", "ldgy", "gh", "ldgh", "gx", "ldgx", "dg", "acc", "ws", "wsb", "s"]
BWD_V = [T, N, A, N, 2 * A, 3 * A, 4 * A, N, 5 * A, N, 6 * A, N, 7 * A, 0, 8 * A, 1 << 24, None]


@pytest.mark.parametrize("over,status", [
    (dict(T=-1), R.E_SHAPE), (dict(n=12), R.E_SHAPE), (dict(h=None), R.E_NULL), (dict(gamma=None), R.E_NULL),
    (dict(rstd=None), R.E_NULL), (dict(gy=None), R.E_NULL), (dict(gx=None), R.E_NULL), (dict(dg=None), R.E_NULL),
    (dict(ws=None), R.E_NULL), (dict(ldh=N - 8), R.E_SHAPE), (dict(ldgy=N + 1), R.E_SHAPE), (dict(ldgh=0), R.E_SHAPE),
    (dict(ldgx=8), R.E_SHAPE), (dict(h=A + 2), R.E_ALIGN), (dict(gh=5 * A + 8), R.E_ALIGN), (dict(dg=7 * A + 4), R.E_ALIGN),
    (dict(ws=8 * A + 16), R.E_ALIGN), (dict(wsb=64), R.E_WORKSPACE), (dict(gx=A), R.E_ALIAS),
    (dict(gx=4 * A, ldgx=N + 8), R.E_ALIAS), (dict(gx=4 * A + 16), R.E_ALIAS), (dict(gx=5 * A + 512), R.E_ALIAS),
    (dict(dg=2 * A), R.E_ALIAS), (dict(dg=6 * A), R.E_ALIAS), (dict(ws=A), R.E_ALIAS), (dict(ws=7 * A), R.E_ALIAS),
    (dict(ws=6 * A), R.E_ALIAS), (dict(dg=3 * A), R.E_ALIAS),
])
def test_norm_backward_refusals(lib, over, status):
    assert lib.cdll.resbm_skip_norm_bwd(*args(BWD, BWD_V, over)) == status


def test_no_tokens_is_no_work(lib):
    c = lib.cdll
    assert c.resbm_skip_norm_fwd(0, N, 0, None, 0, None, 0, None, None, 0.0, None, 0, None, 0, None, None) == R.OK
    assert c.resbm_skip_norm_q8_fwd(0, N, 0, N, None, 0, None, 0, None, None, 0.0, None, 0, None, 0, None, None, None) == R.OK
    assert c.resbm_skip_norm_bwd(0, N, None, 0, None, None, None, 0, None, 0, None, 0, None, 0, None, 0, None) == R.OK
    assert c.resbm_skip_norm_fwd(0, 100, 0, None, 0, None, 0, None, None, 0.0, None, 0, None, 0, None, None) == R.E_SHAPE


def test_norm_workspace(lib):
    c = lib.cdll
    assert c.resbm_norm_workspace_bytes(-1, N) == 0 and c.resbm_norm_workspace_bytes(4, 12) == 0
    for t in (0, 1, 63, 64, 1000, 1 << 20):
        w = c.resbm_norm_workspace_bytes(t, 4096)
        assert w % 256 == 0 and 0 < w <= 64 << 20


# ---------------------------------------------------------------- plans
def entry(**over):
    e = dict(numel=1000, p=A, g=2 * A, m=3 * A, v=4 * A, m_scale=None, v_scale=None, copy=5 * A, g_type=0, state=0,
             weight_decay=0.1, reserved=0)
    e.update(over)
    return R.AdamWTensor(**e)


def plan_of(lib, *entries, room=None):
    arr = (R.AdamWTensor * max(1, len(entries)))(*entries)
    n = int(lib.cdll.resbm_adamw_plan_bytes(arr, len(entries)))
    host = (ctypes.c_int64 * (max(n, 4096) // 8))()
    return lib.cdll.resbm_adamw_plan(arr, len(entries), host, n if room is None else room), host, n


def moved(k, **over):
    return entry(**{**{f: k * A * 16 + getattr(entry(), f) for f in ("p", "g", "m", "v", "copy")}, **over})


@pytest.mark.parametrize("over,status", [
    (dict(), R.OK), (dict(copy=None), R.OK), (dict(numel=0, p=None, g=None, m=None, v=None, copy=None), R.OK),
    (dict(p=A + 4, g=2 * A + 12), R.OK), (dict(g_type=1, g=2 * A + 2), R.OK), (dict(numel=1), R.OK),
    (dict(numel=-1), R.E_SHAPE), (dict(numel=1 << 43), R.E_SHAPE), (dict(weight_decay=-0.1), R.E_SHAPE),
    (dict(weight_decay=NAN), R.E_SHAPE), (dict(g_type=2), R.E_KIND), (dict(state=2), R.E_KIND),
    (dict(p=None), R.E_NULL), (dict(g=None), R.E_NULL), (dict(m=None), R.E_NULL), (dict(v=None), R.E_NULL),
    (dict(state=1), R.E_NULL), (dict(state=1, m_scale=6 * A), R.E_NULL), (dict(state=1, m_scale=6 * A, v_scale=7 * A), R.OK),
    (dict(state=1, m=3 * A + 1, m_scale=6 * A, v_scale=7 * A), R.OK),
    (dict(state=1, m_scale=6 * A + 2, v_scale=7 * A), R.E_ALIGN), (dict(p=A + 2), R.E_ALIGN), (dict(g=2 * A + 2), R.E_ALIGN),
    (dict(m=3 * A + 1), R.E_ALIGN), (dict(copy=5 * A + 1), R.E_ALIGN),
    (dict(m=A), R.E_ALIAS), (dict(g=A + 2000), R.E_ALIAS), (dict(copy=4 * A + 3996), R.E_ALIAS), (dict(copy=4 * A + 4000), R.OK),
    (dict(state=1, m_scale=6 * A, v_scale=6 * A + 12), R.E_ALIAS), (dict(state=1, m_scale=6 * A, v_scale=6 * A + 16), R.OK),
])
def test_plan_refusals(lib, over, status):
    assert plan_of(lib, entry(**over))[0] == status


def test_entry_layout():
    assert ctypes.sizeof(R.AdamWTensor) == 80 and R.AdamWTensor.weight_decay.offset == 72 and R.AdamWTensor.copy.offset == 56


def test_plan_of_many(lib):
    assert plan_of(lib)[0] == R.OK
    assert plan_of(lib, entry(), moved(1))[0] == R.OK
    assert plan_of(lib, entry(), moved(1), entry())[0] == R.E_ALIAS          # the same tensor twice
    assert plan_of(lib, entry(), moved(1, p=A + 3996))[0] == R.E_ALIAS       # the last element of another's
    assert plan_of(lib, entry(), moved(1, g=2 * A))[0] == R.OK               # a gradient that two share
    assert plan_of(lib, entry(), moved(1, g=3 * A))[0] == R.E_ALIAS          # a gradient that is another's state
    st, host, n = plan_of(lib, entry())
    assert n % 256 == 0 and lib.cdll.resbm_adamw_plan((R.AdamWTensor * 1)(entry()), 1, host, n - 1) == R.E_WORKSPACE
    assert lib.cdll.resbm_adamw_plan((R.AdamWTensor * 1)(entry()), 1, None, n) == R.E_NULL
    assert lib.cdll.resbm_adamw_plan(None, 1, host, n) == R.E_NULL
    assert lib.cdll.resbm_adamw_plan(None, -1, host, n) == R.E_SHAPE
    assert lib.cdll.resbm_adamw_plan((R.AdamWTensor * 1)(entry()), 1, ctypes.addressof(host) + 4, n) == R.E_ALIGN
    bare = dict(p=None, m=None, v=None, copy=None)
    assert plan_of(lib, entry(**bare), moved(1, **bare))[0] == R.OK
    assert plan_of(lib, entry(**bare), moved(1))[0] == R.E_NULL
    empty = dict(numel=0, g=None, **bare)
    assert plan_of(lib, entry(), entry(**empty))[0] == R.OK                  # one without elements beside others
    assert plan_of(lib, entry(**empty), entry(**bare))[0] == R.OK


def test_a_clash_far_from_its_neighbour_is_found(lib):
    """A long tensor that covers several later ones by address, read-only ones in between."""
    big = moved(1, numel=1 << 20, p=A)
    assert plan_of(lib, big, moved(3, g=A * 16 * 9), moved(4, p=A + (4 << 20) - 4))[0] == R.E_ALIAS
    assert plan_of(lib, big, moved(3, g=A * 16 * 9), moved(4, p=A + (4 << 20)))[0] == R.OK


UPD = ["plan", "dev", "lr", "b1", "b2", "eps", "step", "lr_step", "gs", "s"]


@pytest.mark.parametrize("over,status", [
    (dict(plan=None), R.E_NULL), (dict(dev=None), R.E_NULL), (dict(b1=1.0), R.E_SHAPE), (dict(b1=-0.1), R.E_SHAPE),
    (dict(b2=NAN), R.E_SHAPE), (dict(b2=1.5), R.E_SHAPE), (dict(eps=-1.0), R.E_SHAPE), (dict(step=0), R.E_SHAPE),
    (dict(lr=NAN), R.E_SHAPE), (dict(lr=float("inf")), R.E_SHAPE), (dict(dev=A + 128), R.E_ALIGN),
    (dict(lr_step=A + 4), R.E_ALIGN), (dict(gs=A + 2), R.E_ALIGN),
])
def test_update_refusals(lib, over, status):
    _, host, _ = plan_of(lib, entry())
    vals = [ctypes.addressof(host), 9 * A, 1e-3, 0.9, 0.95, 1e-8, 1, None, None, None]
    assert lib.cdll.resbm_adamw_update(*args(UPD, vals, over)) == status


def test_plans_that_are_none_or_have_no_work(lib):
    c = lib.cdll
    zero = (ctypes.c_int64 * 64)()
    assert c.resbm_adamw_update(zero, 9 * A, 1e-3, 0.9, 0.95, 1e-8, 1, None, None, None) == R.E_KIND
    assert c.resbm_grad_norm(zero, 9 * A, 1.0, A, 2 * A, 1 << 20, None) == R.E_KIND
    assert c.resbm_grad_norm_workspace_bytes(zero) == 0 and c.resbm_grad_norm_workspace_bytes(None) == 0
    _, empty, _ = plan_of(lib)
    assert c.resbm_adamw_update(empty, None, 1e-3, 0.9, 0.95, 1e-8, 1, None, None, None) == R.OK
    _, bare, _ = plan_of(lib, entry(p=None, m=None, v=None, copy=None))
    assert c.resbm_adamw_update(bare, 9 * A, 1e-3, 0.9, 0.95, 1e-8, 1, None, None, None) == R.E_NULL


NRM = ["plan", "dev", "max", "out", "ws", "wsb", "s"]


@pytest.mark.parametrize("over,status", [
    (dict(plan=None), R.E_NULL), (dict(dev=None), R.E_NULL), (dict(out=None), R.E_NULL), (dict(ws=None), R.E_NULL),
    (dict(max=0.0), R.E_SHAPE), (dict(max=-1.0), R.E_SHAPE), (dict(max=NAN), R.E_SHAPE), (dict(dev=A + 16), R.E_ALIGN),
    (dict(out=2 * A + 2), R.E_ALIGN), (dict(ws=3 * A + 8), R.E_ALIGN), (dict(wsb=0), R.E_WORKSPACE),
    (dict(out=3 * A), R.E_ALIAS), (dict(out=A), R.E_ALIAS), (dict(ws=A), R.E_ALIAS),
])
def test_grad_norm_refusals(lib, over, status):
    _, host, _ = plan_of(lib, entry())
    vals = [ctypes.addressof(host), A, 1.0, 2 * A, 3 * A, 1 << 20, None]
    assert lib.cdll.resbm_grad_norm(*args(NRM, vals, over)) == status


# ---------------------------------------------------------------- the binding's own checks
def test_binding_refuses_wrong_tensors(lib):
    io = lib.io_dtype
    x, g, y = torch.zeros(4, 64, dtype=io), torch.ones(64), torch.zeros(4, 64, dtype=io)
    with pytest.raises(TypeError, match="gamma"):
        lib.skip_norm_fwd(x, g.double(), y)
    with pytest.raises(ValueError, match="gamma"):
        lib.skip_norm_fwd(x, g[:32], y)
    with pytest.raises(ValueError, match="y: expected shape"):
        lib.skip_norm_fwd(x, g, y[:3])
    with pytest.raises(ValueError, match="res"):
        lib.skip_norm_fwd(x, g, y, res=torch.zeros(4, 128, dtype=io)[:, ::2])
    with pytest.raises(ValueError, match="b: expected"):
        lib.skip_norm_fwd(x, g, y, b=torch.zeros(3, 8, dtype=io))
    q = torch.zeros(4, 64).to(torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="scale"):
        lib.skip_norm_q8_fwd(x, g, q, torch.zeros(4, 3))
    with pytest.raises(TypeError, match="y: expected"):
        lib.skip_norm_q8_fwd(x, g, y, torch.zeros(4, 1))
    with pytest.raises(ValueError, match="rstd"):
        lib.skip_norm_bwd(x, g, torch.ones(3), x, y, torch.zeros(64))
    p = [torch.zeros(300)]
    with pytest.raises(ValueError, match="lengths"):
        lib.adamw_plan(p, p, p, [])
    with pytest.raises(ValueError, match="contiguous tensor of 300"):
        lib.adamw_plan(p, [torch.zeros(299)], p, p)
    with pytest.raises(TypeError, match=r"m\[0\]"):
        lib.adamw_plan(p, p, p, p, m_scale=[torch.zeros(2)], v_scale=[torch.zeros(2)])
    with pytest.raises(TypeError, match=r"g\[0\]"):
        lib.adamw_plan(p, [torch.zeros(300).half()], p, p)
    e = [torch.zeros(300).to(torch.float8_e4m3fn)]
    with pytest.raises(ValueError, match="m_scale"):
        lib.adamw_plan(p, p, e, e, m_scale=[torch.zeros(1)], v_scale=[torch.zeros(2)])
    with pytest.raises(ValueError, match="both or neither"):
        lib.adamw_plan(p, p, p, p, v_scale=[torch.zeros(2)])
    sc, big = torch.zeros(4, 1), torch.zeros(1 << 16, dtype=torch.uint8)
    for call in (lambda: lib.skip_norm_fwd(x, g, y), lambda: lib.skip_norm_q8_fwd(x, g, q, sc),
                 lambda: lib.skip_norm_bwd(x, g, torch.ones(4), x, y, torch.zeros(64), ws=big)):
        with pytest.raises(ValueError, match="one GPU"):  # host memory never reaches a kernel
            call()
    with pytest.raises(ValueError, match="one GPU"):
        lib.adamw_plan(p, [torch.ones(300)], [torch.ones(300)], [torch.ones(300)])
