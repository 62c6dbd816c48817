"""8-bit AdamW states and the betas they follow: where half of a block changes, what nearest rounding
keeps up with and what it does not (on the oracle, on the CPU), and the refusal of the rest."""
import ctypes
import os
from types import SimpleNamespace

import numpy as np
import pytest

from oracle import stage_oracle as S
from paper_2604_11947_amd import build as B
from paper_2604_11947_amd import resbm as R


class States:
    """float32-like and 8-bit states of the same gradients."""

    def __init__(self, n, b1, b2):
        self.b = b1, b2
        self.m = self.v = self.m8 = self.v8 = np.zeros(n)

    def step(self, g):
        b1, b2 = self.b
        self.m, self.v = b1 * self.m + (1 - b1) * g, b2 * self.v + (1 - b2) * g * g
        m8, v8 = b1 * self.m8 + (1 - b1) * g, b2 * self.v8 + (1 - b2) * g * g
        q, s = S.state8(m8)
        self.m8 = q * np.repeat(s, S.BLOCK)
        q, s = S.state8(v8, root=True)
        self.v8 = (q * np.repeat(s, S.BLOCK)) ** 2
        return m8 / np.sqrt(v8)


def median_root(b1, b2, factor):
    """Every second element's gradients change their size by `factor` after 4 / (1 - b2) steps: the median of
    u8 / u over them 8 / (1 - b2) steps later."""
    rng = np.random.default_rng(21)
    n, turn = S.BLOCK * 8, round(4 / (1 - b2))
    sigma, moves = np.exp(rng.standard_normal(n)), np.arange(n) % 2 == 1
    s = States(n, b1, b2)
    for t in range(3 * turn):
        s.step(np.where(moves & (t >= turn), factor, 1.0) * sigma * rng.standard_normal(n))
    return float(np.median(np.sqrt(s.v8 / s.v)[moves]))


@pytest.mark.parametrize("factor", [0.1, 3.0])
def test_roots_follow_a_part_of_their_block_up_to_the_limit(factor):
    """Within half a step, 2^-4, of the float32 state's."""
    assert abs(median_root(*R.STATE8_BETAS, factor) - 1) <= 2.0 ** -4


@pytest.mark.parametrize("b2", [0.98, 0.99])
def test_roots_stand_still_beyond(b2):
    """Why larger betas are refused: u stays a multiple of what it should be."""
    assert median_root(0.9, b2, 0.1) >= 2


@pytest.mark.parametrize("b1", [0.9, 0.95])
def test_first_moment_beside_steady_gradients(b1):
    """Gradients of 1 / 100 to 1 of their block's largest, all steady; then every second one becomes zero.
    m falls by 1 - b1 a step until half a step is more: at 0.9 below five of the smallest codes, 2^-9 (0.1 x 5 =
    0.5 goes to the even 4); u is frozen within a half step of its start, 448 / 100 at least.  So an element
    still moves by 4 x 2^-9 / (4.48 (1 - 2^-4)) lr a step at most.  At 0.95 m stops at once."""
    g = np.logspace(-2, 0, S.BLOCK)
    dead = np.arange(S.BLOCK) % 2 == 0
    s = States(S.BLOCK, b1, 0.95)
    for t in range(80):
        s.step(g)
    for t in range(300):
        move = s.step(np.where(dead, 0.0, g))
    most = np.abs(move[dead]).max()
    limit = 4 * S.TINY / (4.48 * (1 - 2.0 ** -4))
    assert most <= limit if b1 <= R.STATE8_BETAS[0] else most > 100 * limit


A = 0x10000000


@pytest.fixture(scope="module")
def cdll():
    if not os.path.exists(B.lib_path("bf16")):
        B.build_all()
    return R.Library("bf16").cdll


def host_plan(cdll, *entries):
    """Each entry with addresses of its own; never launched."""
    arr = (R.AdamWTensor * len(entries))()
    for i, over in enumerate(entries):
        e = dict(numel=1000, g_type=0, state=0, weight_decay=0.0, reserved=0)
        e |= {f: A * (16 * i + k) for k, f in enumerate(("p", "g", "m", "v", "m_scale", "v_scale"), 1)}
        arr[i] = R.AdamWTensor(**(e | over))
    n = int(cdll.resbm_adamw_plan_bytes(arr, len(entries)))
    host = (ctypes.c_int64 * (n // 8))()
    assert cdll.resbm_adamw_plan(arr, len(entries), host, n) == R.OK
    return host


@pytest.mark.parametrize("betas", [(0.91, 0.95), (0.9, 0.96), (0.95, 0.9), (0.9, 0.999), (0.0, 0.99)])
def test_larger_betas_are_refused(cdll, betas):
    up = lambda host, b: cdll.resbm_adamw_update(host, None, 1e-3, *b, 1e-8, 1, None, None, None)
    for entries in ((dict(state=1),), (dict(), dict(state=1)), (dict(state=1), dict())):
        host = host_plan(cdll, *entries)
        assert up(host, betas) == R.E_SHAPE
        # taken: the next check, of the missing table, is reached
        assert up(host, (0.9, 0.95)) == R.E_NULL and up(host, (0.0, 0.5)) == R.E_NULL
    # states in float32, and entries without elements, take any
    assert up(host_plan(cdll, dict()), betas) == R.E_NULL
    assert up(host_plan(cdll, dict(), dict(state=1, numel=0)), betas) == R.E_NULL


def test_the_binding_says_so():
    L = R.Library.__new__(R.Library)
    with pytest.raises(ValueError, match="8-bit states take betas"):
        L.adamw_update(SimpleNamespace(q8=True), 1e-3, 1, betas=(0.9, 0.999))
