"""Pins of the oracle of the pipeline's ends: torch's own functions in fp64, central differences, and closed forms."""
import numpy as np
import pytest
import torch

from oracle import ends_oracle as E


def _rng(seed):
    return np.random.Generator(np.random.Philox(key=[seed, 2111]))


@pytest.mark.parametrize("smoothing", [0.0, 0.3, 1.0])
def test_cross_entropy_is_torchs_with_autograd(smoothing):
    r = _rng(1)
    x, y = r.standard_normal((9, 13)) * 3, r.integers(0, 13, 9)
    y[4] = -100
    loss, dx, _ = E.cross_entropy(x, y, smoothing, 0.25)
    t = torch.from_numpy(x).requires_grad_()
    ref = torch.nn.functional.cross_entropy(t, torch.from_numpy(y), reduction="none", ignore_index=-100, label_smoothing=smoothing)
    (0.25 * ref.sum()).backward()
    np.testing.assert_allclose(loss, ref.detach().numpy(), rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(dx, t.grad.numpy(), rtol=1e-12, atol=1e-13)


def test_cross_entropy_gradient_is_its_difference():
    r = _rng(2)
    x, y = r.standard_normal((3, 5)), np.array([0, 4, 7])
    _, dx, _ = E.cross_entropy(x, y, 0.1, 2.0)
    for i in range(3):
        for j in range(5):
            step = np.zeros_like(x)
            step[i, j] = 1e-5
            d = (E.cross_entropy(x + step, y, 0.1)[0].sum() - E.cross_entropy(x - step, y, 0.1)[0].sum()) / 2e-5
            assert abs(2.0 * d - dx[i, j]) < 1e-8


def test_cross_entropy_of_equal_logits_is_log_vocab_and_masked_entries_do_not_count():
    loss, dx, p = E.cross_entropy(np.zeros((1, 8)), np.array([3]))
    assert abs(loss[0] - np.log(8)) < 1e-14 and abs(dx.sum()) < 1e-15
    x = np.zeros((1, 8))
    x[0, 4:] = -np.inf
    loss, dx, p = E.cross_entropy(x, np.array([3]))
    assert abs(loss[0] - np.log(4)) < 1e-14 and (dx[0, 4:] == 0).all()


def test_embedding_and_its_gradient_are_torchs():
    r = _rng(3)
    table, ids, dy = r.standard_normal((11, 6)), r.integers(0, 11, 40), r.standard_normal((40, 6))
    places, at = r.standard_normal((7, 6)), r.integers(0, 7, 40)
    t = torch.from_numpy(table).requires_grad_()
    out = 1.5 * torch.nn.functional.embedding(torch.from_numpy(ids), t) + torch.from_numpy(places)[torch.from_numpy(at)]
    out.backward(torch.from_numpy(dy))
    np.testing.assert_allclose(E.embedding_fwd(ids, table, 1.5, at, places), out.detach().numpy(), rtol=1e-14)
    grad, n, mag = E.embedding_bwd(ids, dy, 11, 1.5)
    np.testing.assert_allclose(grad, t.grad.numpy(), rtol=1e-12, atol=1e-13)
    assert n.sum() == 40 and (mag >= np.abs(grad) - 1e-12).all()
    ids[5], ids[6] = -1, 11
    assert (E.embedding_fwd(ids, table)[5:7] == 0).all() and E.embedding_bwd(ids, dy, 11)[1].sum() == 38


def test_norm_and_clipping_are_torchs():
    r = _rng(4)
    ts = [r.standard_normal(n) for n in (3, 100, 17)]
    p = [torch.nn.Parameter(torch.zeros(len(t), dtype=torch.float64)) for t in ts]
    for q, t in zip(p, ts):
        q.grad = torch.from_numpy(t.copy())
    norm = torch.nn.utils.clip_grad_norm_(p, 2.0)
    s, bad = E.grad_norm(ts)
    assert bad == 0 and abs(np.sqrt(s) - float(norm)) < 1e-12
    c = E.clip_factor(s, 2.0, 1e-6)
    for q, t in zip(p, ts):
        np.testing.assert_allclose(q.grad.numpy(), c * t, rtol=1e-12)
    ts[1][7], ts[2][0] = np.nan, np.inf
    assert E.grad_norm(ts)[1] == 2 and np.isfinite(E.grad_norm(ts)[0])
