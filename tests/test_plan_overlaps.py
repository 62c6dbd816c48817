"""Operands of an AdamW step or a gradient norm that lie in the plan's own tensors: refused by host checks
before any HIP call.  The addresses are made up, so the file is skipped where a GPU is visible."""
import ctypes
import os

import pytest
import torch

from paper_2604_11947_amd import build as B
from paper_2604_11947_amd import resbm as R

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up device addresses")

A = 0x10000000
FIELDS = ("p", "g", "m", "v", "m_scale", "v_scale", "copy")
N = (1000, 700, 512)


def at(i, field):
    return A * (1 + 8 * i + FIELDS.index(field))


FAR = A * 64


@pytest.fixture(scope="module")
def cdll():
    if not os.path.exists(B.lib_path("bf16")):
        B.build_all()
    return R.Library("bf16").cdll


@pytest.fixture(scope="module")
def plan(cdll):
    """float32 states and gradients; the same with bf16 gradients and without a copy; 8-bit states."""
    arr = (R.AdamWTensor * 3)()
    for i, n in enumerate(N):
        e = {f: at(i, f) for f in FIELDS}
        if i == 1:
            e["copy"] = None
        arr[i] = R.AdamWTensor(numel=n, g_type=int(i == 1), state=int(i == 2), weight_decay=0.0, reserved=0, **e)
    n = int(cdll.resbm_adamw_plan_bytes(arr, 3))
    host = (ctypes.c_int64 * (n // 8))()
    assert cdll.resbm_adamw_plan(arr, 3, host, n) == R.OK
    return host


def ends(i):
    """(field, first byte, end) of a tensor's memory."""
    n, q8 = N[i], i == 2
    size = {"p": 4 * n, "m": n if q8 else 4 * n, "v": n if q8 else 4 * n, "copy": 0 if i == 1 else 2 * n,
            "m_scale": 8 if q8 else 0, "v_scale": 8 if q8 else 0, "g": 2 * n if i == 1 else 4 * n}
    return [(f, at(i, f), at(i, f) + b) for f, b in size.items() if b]


def test_scale_and_step_in_what_the_step_writes(cdll, plan):
    def update(gs=None, ls=None, dev=FAR):
        return cdll.resbm_adamw_update(plan, dev, 1e-3, 0.9, 0.95, 1e-8, 1, ls, gs, None)

    for i in range(3):
        for f, lo, end in ends(i):
            if f == "g":
                continue
            assert update(gs=lo) == update(gs=(end - 1) // 4 * 4) == R.E_ALIAS, (i, f)
            assert update(ls=lo - 8) == update(ls=(end - 1) // 8 * 8) == R.E_ALIAS, (i, f)
            assert update(dev=lo) == update(dev=lo - 256) == R.E_ALIAS, (i, f)


def test_scale_and_step_beside_it(cdll, plan):
    """Taken: the call goes on to the launch, which has no GPU here."""
    for i in range(3):
        for f, lo, end in ends(i):
            end = (end + 7) // 8 * 8
            if f != "g":
                assert cdll.resbm_adamw_update(plan, FAR, 1e-3, 0.9, 0.95, 1e-8, 1, end, lo - 4, None) == R.E_HIP
    # a gradient is only read
    assert cdll.resbm_adamw_update(plan, FAR, 1e-3, 0.9, 0.95, 1e-8, 1, None, at(0, "g"), None) == R.E_HIP


def test_norm_and_workspace_in_a_gradient(cdll, plan):
    need = int(cdll.resbm_grad_norm_workspace_bytes(plan))
    norm = lambda out=FAR + A, ws=FAR + 2 * A: cdll.resbm_grad_norm(plan, FAR, 1.0, out, ws, need, None)
    for i in range(3):
        (lo, end), = [(lo, end) for f, lo, end in ends(i) if f == "g"]
        assert norm(out=lo) == norm(out=lo - 4) == norm(out=(end - 1) // 4 * 4) == R.E_ALIAS
        assert need == 256 and norm(ws=lo) == norm(ws=(end - 1) // 256 * 256) == R.E_ALIAS
        assert norm(ws=lo - 256) == norm(out=lo - 8) == norm(out=(end + 3) // 4 * 4) == norm(ws=(end + 255) // 256 * 256) == R.E_HIP
    assert norm() == R.E_HIP
