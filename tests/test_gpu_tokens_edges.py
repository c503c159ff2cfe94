"""The token models' kernels where their ways meet and at the ends of their ranges."""

import numpy as np
import pytest

import paper_2211_00889_amd as nb
from oracle import tokens as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_tokens import BF16, DEV, SENTINEL, _close, _np, _say, _ws  # noqa: E402


# --------------------------------------------- 8-bit weight gradient, its range
def _act8(A):
    """``orc.act8`` for whole arrays [T, dim]: (whole numbers, steps)."""
    T = len(A)
    q, step = np.zeros(A.shape), np.zeros(A.shape)
    for t in range(0, T, orc.BLOCK):
        v = A[t:t + orc.BLOCK]
        peak = np.abs(v).max(0)
        k = np.full(peak.shape, 121)
        for e in range(120, -127, -1):
            k = np.where(np.rint(peak / 2.0 ** e) <= 127, e, k)
        s = np.where(np.isfinite(peak), 2.0 ** k, np.nan)
        with np.errstate(invalid="ignore"):
            q[t:t + orc.BLOCK] = np.where(np.isfinite(peak), np.clip(np.rint(v / s), -127, 127), 0)
        step[t:t + orc.BLOCK] = s
    return q, step


# just at the largest step, just below it, and beyond; the smallest steps; ordinary ones
PEAKS = [127.5 * 2.0 ** 120, 127.49 * 2.0 ** 120, 2.0 ** 127, 3.3895e38, 3.4028234e38, 2.0 ** -126, 2.0 ** -120, 1.0, 0.0,
         -3e38, -127.5 * 2.0 ** 119]

GRAD_TILES = [
    # n, m, T, dim, out: the small tile, whole and in four parts; the middle one; the large one
    (1, 1, 77, 60, 50), (1, 1, 4100, 40, 72), (8, 8, 131, 384, 300), (8, 8, 130, 512, 512),
]


@pytest.mark.parametrize("n,m,T,dim,out", GRAD_TILES)
def test_act_grad_over_the_steps(n, m, T, dim, out):
    """Peaks up to the largest finite value and down to the smallest step, against the definition and
    against what ``act_unpack`` says that the bytes stand for."""
    rng = np.random.default_rng(T)
    _say(f"act_grad steps {n}x{m} T={T} dim={dim} out={out}")
    gen = torch.Generator(device=DEV).manual_seed(T)
    peaks = torch.tensor([PEAKS[c % len(PEAKS)] for c in range(dim)], device=DEV)
    A = (torch.rand((n, m, T, dim), generator=gen, device=DEV) * 2 - 1) * peaks
    A[:, :, 5::32] = peaks
    A[:, :, 9::32] = 0
    dY = (torch.randn((n, m, T, out), generator=gen, device=DEV) * 2.0 ** -24).to(BF16)
    packed = torch.empty((n, m, nb.act_bytes(T, dim)), dtype=torch.uint8, device=DEV)
    mask = np.ones((n, m), np.uint8)
    nb.act_pack(A, mask, packed)
    values = torch.empty_like(A)
    nb.act_unpack(packed, mask, values)
    G = torch.full((n, m, dim * out), SENTINEL, device=DEV)
    nb.act_grad(packed, dY, mask, G, 0, dim, _ws(nb.act_workspace_bytes(n, m, T, dim, out)))
    for i, j in {(0, 0), (n - 1, m - 1), (n // 2, int(rng.integers(m)))}:
        q, step = _act8(_np(A[i, j]))
        assert (step == 2.0 ** 121).any() and (step == 2.0 ** -126).any()
        assert np.array_equal(_np(values[i, j]), q * step)
        want, bound = orc.act_grad(q * step, _np(dY[i, j]))
        _close("G", G[i, j].view(dim, out), want, bound)


@pytest.mark.parametrize("n,m,T,dim,out", GRAD_TILES)
def test_act_grad_of_nan_blocks(n, m, T, dim, out):
    """A block that holds an infinity or a NaN makes its own channel's row of the gradient NaN."""
    _say(f"act_grad NaN blocks {n}x{m} T={T} dim={dim} out={out}")
    gen = torch.Generator(device=DEV).manual_seed(T)
    A = torch.randn((n, m, T, dim), generator=gen, device=DEV)
    bad = {1: 3, 17: T - 1, dim - 1: 40}  # channel: token
    for c, t in bad.items():
        A[..., t, c] = float("nan") if c == 17 else float("inf") if c == 1 else -float("inf")
    dY = torch.randn((n, m, T, out), generator=gen, device=DEV).to(BF16)
    packed = torch.empty((n, m, nb.act_bytes(T, dim)), dtype=torch.uint8, device=DEV)
    mask = np.ones((n, m), np.uint8)
    nb.act_pack(A, mask, packed)
    G = torch.full((n, m, dim * out), SENTINEL, device=DEV)
    nb.act_grad(packed, dY, mask, G, 0, dim, _ws(nb.act_workspace_bytes(n, m, T, dim, out)))
    others = np.array([c not in bad for c in range(dim)])
    for i, j in {(0, 0), (n - 1, m - 1)}:
        q, step = _act8(_np(A[i, j]))
        got = G[i, j].view(dim, out)
        assert torch.isnan(got[sorted(bad)]).all()
        want, bound = orc.act_grad((q * step)[:, others], _np(dY[i, j]))
        _close("G", got[torch.from_numpy(others).to(DEV)], want, bound)
