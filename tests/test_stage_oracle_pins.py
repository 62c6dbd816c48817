"""Pins of the oracle of the operators next to the boundary: differences, torch's
float64 autograd, closed forms and torch's e4m3 rounding.  All on the CPU."""
import numpy as np
import pytest
import torch

from oracle import stage_oracle as S

EPS = 1e-5


@pytest.mark.parametrize("shape", [(1, 8), (3, 24), (5, 40)])
def test_norm_backward_against_differences_and_autograd(shape):
    rng = np.random.default_rng(1)
    T, n = shape
    h, gamma = rng.standard_normal((T, n)), 1 + 0.1 * rng.standard_normal(n)
    gy, gh = rng.standard_normal((T, n)), rng.standard_normal((T, n))
    gx, dg = S.norm_bwd(h, gamma, S.rstd(h, EPS), gy, gh)

    def loss(h, gamma):
        return np.sum(gy * S.norm(h, gamma, EPS)) + np.sum(gh * h)

    for _ in range(4):
        dh, dga = rng.standard_normal((T, n)), rng.standard_normal(n)
        s = 1e-6
        num = (loss(h + s * dh, gamma + s * dga) - loss(h - s * dh, gamma - s * dga)) / (2 * s)
        assert abs(num - (np.sum(gx * dh) + np.sum(dg * dga))) <= 1e-7 * (np.abs(num) + T * n)
    ht, gt = torch.tensor(h, requires_grad=True), torch.tensor(gamma, requires_grad=True)
    y = ht * torch.rsqrt((ht * ht).mean(1, keepdim=True) + EPS) * gt
    ((y * torch.tensor(gy)).sum() + (ht * torch.tensor(gh)).sum()).backward()
    np.testing.assert_allclose(gx, ht.grad.numpy(), rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(dg, gt.grad.numpy(), rtol=1e-10, atol=1e-12)


def test_stream_puts_the_payload_into_the_first_columns():
    x, res, b = np.ones((2, 8)), 2 * np.ones((2, 8)), 4 * np.ones((2, 4))
    assert np.array_equal(S.stream(x, res, b), [[7] * 4 + [3] * 4] * 2)
    assert np.array_equal(S.stream(x), x)


def test_norm_of_a_constant_row():
    np.testing.assert_allclose(S.norm(np.full((1, 16), 3.0), np.ones(16), 0.0), 1.0, rtol=1e-15)


def test_e4m3_is_torchs_rounding():
    x = torch.randn(200_000, generator=torch.Generator().manual_seed(0), dtype=torch.float64).float() * 30
    x = torch.cat([x.clamp(-448, 448), torch.tensor([0.0, 448.0, -448.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2 ** -9, 17.0, 19.0])])
    assert np.array_equal(S.e4m3(x.double().numpy()), x.to(torch.float8_e4m3fn).double().numpy())


def test_adamw_against_a_scalar_loop_and_its_first_step():
    rng = np.random.default_rng(2)
    p, g = rng.standard_normal(5), rng.standard_normal(5)
    m = v = np.zeros(5)
    q, mm, vv = p.copy(), [0.0] * 5, [0.0] * 5
    for step in range(1, 4):
        p, m, v = S.adamw(p, g, m, v, 0.01, step, 0.9, 0.95, 1e-8, 0.1)
        for i in range(5):
            mm[i] = 0.9 * mm[i] + 0.1 * g[i]
            vv[i] = 0.95 * vv[i] + 0.05 * g[i] ** 2
            q[i] = q[i] * (1 - 0.001) - 0.01 * (mm[i] / (1 - 0.9 ** step)) / ((vv[i] / (1 - 0.95 ** step)) ** 0.5 + 1e-8)
    np.testing.assert_allclose(p, q, rtol=1e-13)
    one, _, _ = S.adamw(np.zeros(5), g, np.zeros(5), np.zeros(5), 0.01, 1, 0.9, 0.95, 0.0, 0.0)
    np.testing.assert_allclose(one, -0.01 * np.sign(g), rtol=1e-12)  # bias correction makes the first step lr sign(g)


def test_adamw_against_torch():
    rng = np.random.default_rng(3)
    w = torch.tensor(rng.standard_normal(64), requires_grad=True)
    opt = torch.optim.AdamW([w], lr=3e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    p, m, v = w.detach().numpy().copy(), np.zeros(64), np.zeros(64)
    for step in range(1, 6):
        g = rng.standard_normal(64)
        w.grad = torch.tensor(g)
        opt.step()
        p, m, v = S.adamw(p, g, m, v, 3e-3, step, 0.9, 0.95, 1e-8, 0.1)
    np.testing.assert_allclose(p, w.detach().numpy(), rtol=1e-12)


def test_state8_keeps_every_nonzero_root_and_half_a_step():
    rng = np.random.default_rng(4)
    x = rng.standard_normal(600) * np.exp(3 * rng.standard_normal(600))
    q, s = S.state8(x)
    back = q * np.repeat(s, 256)[:600]
    assert np.all(np.abs(back - x) <= np.maximum(np.abs(x) * 2.0 ** -4, np.repeat(s, 256)[:600] * 2.0 ** -10) * (1 + 1e-9))
    v = x ** 2 * np.where(np.arange(600) % 5 == 0, 1e-12, 1.0)
    v[7] = 0.0
    q, s = S.state8(v, root=True)
    assert q[7] == 0 and np.all(q[v > 0] >= S.TINY)
    assert np.array_equal(S.state8(np.zeros(3))[1], [S.SCALE_FLOOR])


def test_grad_norm():
    n, f = S.grad_norm([np.full(4, 3.0), np.full(7, 4.0) * 0, np.array([8.0])], 5.0)
    assert n == 10.0 and abs(f - 0.5) < 1e-7
    assert S.grad_norm([np.zeros(3)], 1.0) == (0.0, 1.0)
    assert np.isnan(S.grad_norm([np.array([np.inf])], 1.0)[1])


def test_8bit_states_follow_a_noisy_gradient():
    """Nearest rounding freezes a value that moves by less than half a step at a time, as u = sqrt(v) does
    (1 - sqrt(b2) = 2.5 %, against 3 to 6 %).  The scales, which follow each block's largest element exactly,
    move with it and shift the others over their codes: u stays within a half step, 2^-4, of the float32
    state's on average, also after the gradients have become ten times smaller."""
    rng = np.random.default_rng(6)
    n, b1, b2 = 256 * 16, 0.9, 0.95
    sigma = np.exp(rng.standard_normal(n))
    m = v = m8 = v8 = np.zeros(n)
    for size in (1.0, 0.1):
        for _ in range(200):
            g = size * sigma * rng.standard_normal(n)
            m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
            m8, v8 = b1 * m8 + (1 - b1) * g, b2 * v8 + (1 - b2) * g * g
            q, s = S.state8(m8)
            m8 = q * np.repeat(s, 256)
            q, s = S.state8(v8, root=True)
            v8 = (q * np.repeat(s, 256)) ** 2
        ratio = np.sqrt(v8 / v)
        assert abs(ratio.mean() - 1) <= 2.0 ** -4, (size, ratio.mean())
        step, step8 = m / np.sqrt(v), m8 / np.sqrt(v8)
        assert np.corrcoef(step, step8)[0, 1] >= 0.98


def test_planted_mistakes_fail_a_pin():
    """A dropped projection term, a mean over the wrong axis, an uncorrected bias, a root that rounds to zero."""
    rng = np.random.default_rng(5)
    h, gamma, gy = rng.standard_normal((3, 16)), np.ones(16), rng.standard_normal((3, 16))
    rs = S.rstd(h, EPS)
    good, _ = S.norm_bwd(h, gamma, rs, gy)
    d = rng.standard_normal((3, 16))
    num = (np.sum(gy * S.norm(h + 1e-6 * d, gamma, EPS)) - np.sum(gy * S.norm(h - 1e-6 * d, gamma, EPS))) / 2e-6
    xh = h * rs[:, None]
    for bad in (rs[:, None] * gy, rs[:, None] * (gy - xh * np.mean(gy * xh, axis=0, keepdims=True))):
        assert abs(num - np.sum(bad * d)) > 1e-3
    assert abs(num - np.sum(good * d)) < 1e-6
    g = rng.standard_normal(5)
    m, v = 0.1 * g, 0.05 * g * g
    assert not np.allclose(-0.01 * m / np.sqrt(v), -0.01 * np.sign(g))
    t = np.array([1.0, 1e-9])
    assert S.e4m3(t / S.scales(t)).min() == 0 and S.state8(t * t, root=True)[0].min() > 0
