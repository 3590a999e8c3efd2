"""The oracle of rotary positions, residual norms and AdamW against what they have to be: rotations that depend on distances alone, autograd and
differences, torch's own optimizer, the table of 8-bit numbers.  No GPU needed."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_turns_by_distance(interleaved):
    r = np.random.default_rng(1)
    f = 100.0 ** (-np.arange(4) / 4)
    q, k = r.standard_normal((1, 1, 11)), r.standard_normal((1, 1, 11))
    at = lambda x, p: L.rotary(x, [p], f, 10 ** 6, interleaved)  # noqa: E731
    for p, s in ((5, 2), (1000, 77)):
        for shift in (0, 3, 4000):   # a score depends on the distance only
            np.testing.assert_allclose((at(q, p + shift) * at(k, s + shift)).sum(), (at(q, p) * at(k, s)).sum(), rtol=1e-9)
    np.testing.assert_allclose(at(q, 0), q, rtol=0, atol=0)
    np.testing.assert_allclose(np.linalg.norm(at(q, 12345)), np.linalg.norm(q), rtol=1e-12)
    np.testing.assert_array_equal(at(q, 7)[..., 8:], q[..., 8:])
    back = L.rotary(at(q, 99), [99], f, 10 ** 6, interleaved, transpose=True)
    np.testing.assert_allclose(back, q, rtol=1e-12, atol=1e-13)
    np.testing.assert_array_equal(L.rotary(q, [-1], f, 10, interleaved), q)
    np.testing.assert_array_equal(L.rotary(q, [10], f, 10, interleaved), q)
    # one pair by hand: (1, 0) goes to (cos, sin)
    e = np.zeros((1, 1, 8))
    e[0, 0, 2 if interleaved else 1] = 1.0
    out = L.rotary(e, [3], f, 10, interleaved, magnitude=2.0)[0, 0]
    pair = out[[2, 3]] if interleaved else out[[1, 5]]
    np.testing.assert_allclose(pair, 2 * np.array([np.cos(3 * f[1]), np.sin(3 * f[1])]), rtol=1e-14)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_and_its_gradient(kind):
    r = np.random.default_rng(2)
    x, w, b, g = r.standard_normal((5, 7)) + 0.3, r.standard_normal(7), r.standard_normal(7), r.standard_normal((5, 7))
    f = lambda x: L.normed(x, L.statistics(x, kind, 1e-3), w, b)  # noqa: E731
    tx = torch.from_numpy(x).requires_grad_()
    tw, tb = torch.from_numpy(w), torch.from_numpy(b)
    t = torch.nn.functional.layer_norm(tx, (7,), tw, tb, 1e-3) if kind == "layer" else torch.nn.functional.rms_norm(tx, (7,), tw, 1e-3) + tb
    np.testing.assert_allclose(f(x), t.detach().numpy(), rtol=1e-12, atol=1e-13)
    t.backward(torch.from_numpy(g))
    back = L.norm_back(g * w, x, L.statistics(x, kind, 1e-3), kind)
    np.testing.assert_allclose(back, tx.grad.numpy(), rtol=1e-10, atol=1e-12)
    for i, j in ((0, 0), (3, 5), (4, 6)):
        d = np.zeros_like(x)
        d[i, j] = 1e-5
        np.testing.assert_allclose(((f(x + d) - f(x - d)) * g).sum() / 2e-5, back[i, j], rtol=1e-6, atol=1e-8)


def test_codes_are_the_type():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    np.testing.assert_array_equal(L.CODES, every[torch.isfinite(every)].abs().unique().numpy())


def test_scales():
    for top, e in ((1.0, 0), (1.9999, 0), (2.0, 1), (3e-5, -16), (1e30, 99), (2.0 ** -119, -119), (2.0 ** -125, -119), (0.0, -119)):
        assert L.block_scale(np.array([0.0, -top, top / 3])) == 2.0 ** (e - 7)
    assert L.block_scale(np.array([np.nan, np.inf, -4.0])) == 2.0 ** -5


def test_rounding_up_and_down_is_even_over_steps():
    """Over N steps of an entry the mean of its codes is the value: the share of ups is within the sequence's discrepancy, well under 1 in 100 at 4096."""
    r = np.random.default_rng(3)
    n = 4096
    for i in (0, 1, 255, 12345, 2 ** 32 - 1):
        u = [np.array([L.spread(i, k, *ab) for k in range(n)]) for ab in ((L.A, L.B), (L.B, L.A))]
        for _ in range(5):
            m = float(r.uniform(-250, 250)) * 2.0 ** -float(r.integers(0, 20))
            lo, hi = L.neighbours(abs(m))
            assert abs(np.mean([L.code_m(m, 1.0, x) for x in u[0]]) - m) <= 0.01 * (hi - lo)
            v = m * m
            if np.sqrt(v) >= L.CODES[1]:
                codes = np.array([L.code_v(v, 1.0, x) for x in u[1]])
                assert abs(np.mean(codes ** 2) - v) <= 0.01 * (hi ** 2 - lo ** 2)
    assert L.code_v(1e-30, 1.0, 0.5) == L.CODES[1] and L.code_v(0.0, 1.0, 0.0) == 0.0
    for x in L.CODES[L.CODES < 256]:   # what is a code stays one, whatever decides
        assert L.code_m(-x, 1.0, 0.0) == -x and L.code_m(x, 1.0, 1 - 2.0 ** -24) == x and L.code_v(x * x, 1.0, 0.0) == x


def test_adamw_is_torchs():
    r = np.random.default_rng(4)
    w, m, v = r.standard_normal(50), np.zeros(50), np.zeros(50)
    p = torch.from_numpy(w.copy()).requires_grad_()
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.8, 0.9), eps=1e-6, weight_decay=0.3)
    for step in range(1, 6):
        g = r.standard_normal(50)
        p.grad = torch.from_numpy(g)
        opt.step()
        w, m, v = L.adamw(w, g, m, v, step, 0.01, 0.8, 0.9, 1e-6, 0.3)
        np.testing.assert_allclose(w, p.detach().numpy(), rtol=1e-10, atol=1e-13)
