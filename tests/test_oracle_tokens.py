"""Pins of the token models' oracle: torch autograd in float64, central differences, and the
definition of the 8-bit form."""

import numpy as np
import pytest

from oracle import tokens

torch = pytest.importorskip("torch")


def _scan_torch(x, g, bias, h0, length):
    h, out = h0, []
    for t in range(x.shape[0]):
        if t < length:
            a = torch.sigmoid(g[t] + bias)
            h = a * h + (1 - a) * x[t]
            out.append(h)
        else:
            out.append(torch.zeros_like(h))
    return (torch.stack(out) if out else x), h


@pytest.mark.parametrize("T,C,length", [(1, 3, 1), (7, 2, 7), (9, 4, 5), (6, 1, 0)])
def test_scan_against_autograd(T, C, length):
    rng = np.random.default_rng(T)
    x, g, dh = rng.normal(size=(3, T, C))
    bias, h0, last = rng.normal(size=(3, C))
    leaves = [torch.tensor(v, requires_grad=True) for v in (x, g, bias, h0)]
    h, s = _scan_torch(*leaves, length)
    ((h * torch.tensor(dh))[:length].sum() + (s * torch.tensor(last)).sum()).backward()
    (ho, before, so), _ = tokens.scan(x, g, bias, h0, length)
    np.testing.assert_allclose(ho, h.detach().numpy(), atol=1e-12)
    np.testing.assert_allclose(so, s.detach().numpy(), atol=1e-12)
    np.testing.assert_allclose(before[0], h0)
    (dx, dg, dh0, db), _ = tokens.scan_grad(x, g, bias, h0, length, dh, last)
    for got, leaf in zip((dx, dg, db, dh0), leaves):
        want = np.zeros(leaf.shape) if leaf.grad is None else leaf.grad.numpy()
        np.testing.assert_allclose(got, want, atol=1e-12)


def test_scan_gradient_against_differences():
    rng = np.random.default_rng(3)
    T, C, eps = 6, 3, 1e-5
    x, g, dh = rng.normal(size=(3, T, C))
    bias, h0, last = rng.normal(size=(3, C))

    def loss(g_, b_):
        (h, _, s), _ = tokens.scan(x, g_, b_, h0, T)
        return (h * dh).sum() + (s * last).sum()

    (_, dg, _, db), _ = tokens.scan_grad(x, g, bias, h0, T, dh, last)
    for t, c in ((0, 0), (3, 1), (5, 2)):
        d = np.zeros_like(g)
        d[t, c] = eps
        np.testing.assert_allclose((loss(g + d, bias) - loss(g - d, bias)) / (2 * eps), dg[t, c], rtol=1e-6,
                                   atol=1e-8)
    d = np.array([0, eps, 0])
    np.testing.assert_allclose((loss(g, bias + d) - loss(g, bias - d)) / (2 * eps), db[1], rtol=1e-6)


def test_embed_against_autograd():
    rng = np.random.default_rng(0)
    E = torch.tensor(rng.normal(size=(5, 3)), requires_grad=True)
    tok, dY = np.array([4, 0, 4, -1, 2, 5, 4]), rng.normal(size=(7, 3))
    inside = torch.tensor((tok >= 0) & (tok < 5))
    Y = torch.where(inside[:, None], 2.5 * E[torch.tensor(tok).clamp(0, 4)], 0.0)
    (Y * torch.tensor(dY)).sum().backward()
    np.testing.assert_allclose(tokens.embed(E.detach().numpy(), tok, 2.5), Y.detach().numpy())
    np.testing.assert_allclose(tokens.embed_grad(dY, tok, 5, 2.5)[0], E.grad.numpy(), atol=1e-14)


def test_act8_steps():
    A = np.zeros((40, 4))
    A[:32, 0] = np.linspace(-1, 1, 32)
    A[3, 1] = 127.5          # rounds to 128 on a step of one
    A[35, 2] = 2.0 ** -130   # below every step
    A[2, 3] = np.inf
    q, step = tokens.act8(A)
    assert step[0, 0] == 2.0 ** -6 and np.abs(q[:32, 0]).max() == 64
    assert step[3, 1] == 2.0 and q[3, 1] == 64
    assert step[35, 2] == 2.0 ** -126 and q[35, 2] == 0
    assert np.isnan(step[5, 3]) and step[33, 3] == 2.0 ** -126
    ok = ~np.isnan(step)
    assert (np.abs(q * step - A)[ok] <= step[ok] / 2).all()
