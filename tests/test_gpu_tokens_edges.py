"""The token models' kernels where their ways meet and at the ends of their ranges."""

import numpy as np
import pytest

import paper_2211_00889_amd as nb
from oracle import tokens as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_tokens import BF16, DEV, F32, SENTINEL, _close, _np, _rows, _say, _tokens, _ws  # noqa: E402


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


# ------------------------------------------------- a mini-batch's results are its own
def _bits(t):
    return t.contiguous().view(torch.int32 if t.dtype is F32 else torch.int16)


def _scan_both(x, g, dh, X, h0, dl, lengths):
    """Every output of the two passes."""
    n, m, b, T, C = x.shape
    mask, ws = np.ones((n, m), np.uint8), _ws(nb.scan_workspace_bytes(n, m, b, T, C))
    o = {k: torch.empty_like(x) for k in ("h", "dx", "dg")}
    o["last"], o["dh0"] = torch.empty_like(h0), torch.empty_like(h0)
    o["states"] = torch.empty((n, m, b, -(-T // nb.SCAN_INTERVAL), C), device=DEV)
    o["G"] = torch.zeros((n, m, X.shape[1]), device=DEV)
    nb.scan(x, g, mask, o["h"], X=X, h0=h0, h_last=o["last"], lengths=lengths, states=o["states"], workspace=ws)
    nb.scan_grad(x, g, o["states"], dh, mask, o["dx"], o["dg"], ws, X=X, G=o["G"], dh_last=dl, dh0=o["dh0"], lengths=lengths)
    return o


def _scan_some(seed, n, m, b, T, C, dtype):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    shape = (n, m, b, T, C)
    x, g, dh = (torch.randn(shape, generator=gen, device=DEV, dtype=F32 if dtype is F32 else BF16) for _ in range(3))
    h0, dl = (torch.randn((n, m, b, C), generator=gen, device=DEV) for _ in range(2))
    X = torch.randn((n, (C + 3) // 4 * 4), generator=gen, device=DEV) + 2
    lengths = torch.randint(0, T + 1, (n, m, b), generator=gen, device=DEV, dtype=torch.int32)
    lengths[..., 0] = T
    return x, g, dh, X, h0, dl, lengths


def _against_oracle(o, data, at, few, dtype):
    """One sequence's channels `few` of every output."""
    x, g, dh, X, h0, dl, lengths = data
    L = int(lengths[at])
    args = [_np(x[at][..., few]), _np(g[at][..., few]), _np(X[at[0], few]), _np(h0[at][few]), L]
    (ho, before, s), (eh, eb, es) = orc.scan(*args)
    _close("h", o["h"][at][..., few], ho, eh, dtype)
    _close("h_last", o["last"][at][few], s, es)
    _close("states", o["states"][at][..., few], before[::nb.SCAN_INTERVAL], eb[::nb.SCAN_INTERVAL])
    (gx, gg, g0, _), (ex, eg, e0, _) = orc.scan_grad(*args, _np(dh[at][..., few]), _np(dl[at][few]))
    _close("dx", o["dx"][at][..., few], gx, ex, dtype)
    _close("dg", o["dg"][at][..., few], gg, eg, dtype)
    _close("dh0", o["dh0"][at][few], g0, e0)


@pytest.mark.parametrize("n,m,b,T,C,dtype", [
    # walked whole with the others; alone a tile a workgroup, or three and two (the last ones)
    (4, 4, 8, 700, 136, F32), (4, 4, 8, 700, 198, BF16), (4, 8, 8, 520, 1024, BF16), (4, 1, 2, 5000, 4096, BF16),
    (4, 2, 2, 5000, 1030, F32),
])
def test_scan_of_many_and_alone(n, m, b, T, C, dtype):
    """One mini-batch of a call whose sequences are walked whole, against the same one in a call that
    splits them: bit for bit."""
    _say(f"scan many and alone {n}x{m}x{b} T={T} dim={C} {dtype}")
    data = _scan_some(T + C, n, m, b, T, C, dtype)
    x, g, dh, X, h0, dl, lengths = data
    lengths[n - 1, 0, 1] = 2 * T // 3
    whole = _scan_both(*data)
    for i, j in ((0, 0), (n - 1, m - 1)):
        own = [t[i:i + 1, j:j + 1].contiguous() for t in (x, g, dh)]
        one = _scan_both(*own, X[i:i + 1].contiguous(), *(t[i:i + 1, j:j + 1].contiguous() for t in (h0, dl, lengths)))
        differ = {k: int((_bits(one[k][0, 0]) != _bits(whole[k][i, j])).sum()) for k in one}
        assert not any(differ.values()), differ
    _against_oracle(whole, data, (n - 1, 0, 1), slice(C - 9, C), dtype)
    _against_oracle(whole, data, (0, 0, 0), slice(0, 7), dtype)


@pytest.mark.parametrize("T", [12, 300, 1500])
def test_a_state_keeps_its_sign(T):
    """A state of -0 of an ended sequence, in a call that walks its sequences whole and in one that
    splits them, forward and backward."""
    n, m, b, C = 8, 8, 8, 4
    x, g, dh, X, h0, dl, lengths = _scan_some(T, n, m, b, T, C, F32)
    h0.fill_(-0.0), dl.fill_(-0.0), lengths.zero_()
    whole = _scan_both(x, g, dh, X, h0, dl, lengths)
    one = _scan_both(*(t[:1, :1].contiguous() for t in (x, g, dh)), X[:1].contiguous(),
                     *(t[:1, :1].contiguous() for t in (h0, dl, lengths)))
    for o in (whole, one):
        for k in ("last", "dh0", "states"):
            assert torch.equal(_bits(o[k]), _bits(torch.full_like(o[k], -0.0))), k


# ------------------------------------------------------------------ embeddings
@pytest.mark.parametrize("T", [5, 128, 129, 1500])
@pytest.mark.parametrize("scale", [float("inf"), float("nan"), -2.0, 0.0])
def test_rows_without_tokens_are_zero(T, scale):
    """Whatever the scale is, and +0: a few tokens and sorted ones alike."""
    rng = np.random.default_rng(T)
    V, D = 300, 21
    tok = rng.integers(0, V // 2, (1, 1, T)).astype(np.int32)
    dY, _ = _rows((1, 1, T, D), F32, rng=rng)
    G = torch.full((1, 1, (V * D + 3) // 4 * 4), SENTINEL, device=DEV)
    nb.embed_grad(dY, torch.from_numpy(tok).to(DEV), [[1]], G, 0, V, _ws(nb.embed_workspace_bytes(1, 1, T, V, D)), scale=scale)
    rows = G[0, 0, :V * D].view(V, D)
    empty = torch.from_numpy(~np.isin(np.arange(V), tok)).to(DEV)
    assert (_bits(rows[empty]) == 0).all()
    if np.isfinite(scale):
        want, bound = orc.embed_grad(_np(dY[0, 0]), tok[0, 0], V, scale)
        _close("G", rows, want, bound)
    else:
        assert not torch.isfinite(rows[~empty]).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind,T,vocab,dim", [("zipf", 40001, 300, 5), ("uniform", 33000, 70000, 3), ("one", 50000, 9, 4),
                                              ("zipf", 32768, 5000, 8), ("uniform", 262144, 40, 2)])
def test_embed_grad_of_many_tokens(kind, T, vocab, dim, dtype):
    """More than four sorted runs to join."""
    rng = np.random.default_rng(T)
    _say(f"embed_grad {kind} T={T} vocab={vocab} dim={dim} {dtype}")
    tok = _tokens(rng, kind, (1, 1, T), vocab)
    dY, _ = _rows((1, 1, T, dim), dtype, rng=rng)
    G = torch.full((1, 1, (vocab * dim + 3) // 4 * 4), SENTINEL, device=DEV)
    nb.embed_grad(dY, torch.from_numpy(tok).to(DEV), [[1]], G, 0, vocab, _ws(nb.embed_workspace_bytes(1, 1, T, vocab, dim)))
    want, bound = orc.embed_grad(_np(dY[0, 0]), tok[0, 0], vocab, 1.0)
    _close("G", G[0, 0, :vocab * dim].view(vocab, dim), want, bound)


# -------------------------------------------------- sequences of many tiles
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,m,b,T,C,ends", [
    # 64 tiles, 65, 79: one and two rounds of the tiles' states; then two tiles a workgroup
    (1, 1, 1, 16384, 7, ()), (1, 1, 2, 16385, 24, (16384,)), (1, 1, 3, 20000, 64, (17001, 3)),
    (1, 2, 32, 5000, 40, (4999, 257, 256, 0, 1300)),
])
def test_scan_of_many_tiles(n, m, b, T, C, ends, dtype):
    """More tiles than one round of the tiles' states takes, and more than one tile a workgroup, with
    lengths that end inside them."""
    _say(f"scan many tiles {n}x{m}x{b} T={T} dim={C} {dtype}")
    data = _scan_some(T, n, m, b, T, C, dtype)
    lengths = data[-1]
    for k, e in enumerate(ends):
        lengths[n - 1, m - 1, k + 1] = e
    o = _scan_both(*data)
    for k in range(min(b, len(ends) + 1)):
        _against_oracle(o, data, (n - 1, m - 1, k), slice(max(0, C - 5), C), dtype)


# ------------------------------------------------------------ gates in 32 bits
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [1, 40])
def test_gates_in_32_bits(T, dtype):
    """The state after one token from a state of 1 and an x of 0 is the gate, in fp32 of bf16 rows too.
    With u = 2^-24: the exponential's argument is off by |z| u (a product) and 0.25 |z| u (log2 e), it by 2 u
    (its last place), 1 + e by u, the reciprocal by 2 u, a product by u.  So the smaller of gate and
    complement is off by (1.25 |z| + 6) u of its value, and the larger, bf16 rows' 1 - e r, by that and half
    a step of [1/2, 1]; fp32 rows' 1 / (1 + e) by the rounding of 1 + e, u of the value, besides."""
    C = 4096
    g = torch.linspace(-20, 20, C, device=DEV).to(dtype).view(1, 1, 1, 1, C).expand(1, 1, 1, T, C).contiguous()
    h, last = torch.empty_like(g), torch.empty((1, 1, 1, C), device=DEV)
    one = torch.ones((1, 1, 1), dtype=torch.int32, device=DEV)
    nb.scan(torch.zeros_like(g), g, [[1]], h, h0=torch.ones_like(last), h_last=last, lengths=one,
            workspace=_ws(nb.scan_workspace_bytes(1, 1, 1, T, C)))
    z = _np(g[0, 0, 0, 0])
    want, small = 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(np.abs(z)))
    room = small * (1.25 * np.abs(z) + 6) * orc.U + np.where(z > 0, orc.U / 2 + (orc.U * want if dtype is F32 else 0), 0)
    off = np.abs(_np(last[0, 0, 0]) - want) / room
    assert off.max() <= 1, (off.max(), z[off.argmax()], int((off > 1).sum()))


# ------------------------------------------------ infinities and NaNs in live values
BAD = [float("inf"), -float("inf"), float("nan")]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,at", [(12, 5), (200, 70), (600, 258), (600, 0), (600, 599)])
def test_infinities_stay_behind_their_token(T, at, dtype):
    """An infinite or NaN x, h0, dh or dh_last: forward the tokens before it, backward the ones after it,
    and every other channel are as the formula has them."""
    _say(f"infinities T={T} at={at} {dtype}")
    C = 9
    data = _scan_some(T, 1, 1, 1, T, C, dtype)
    x, g, dh, X, h0, dl, lengths = data
    finite = [t.clone() for t in data]
    want, none = _scan_both(*finite), slice(6, C)

    def same(a, b):
        assert torch.equal(_bits(a), _bits(b))

    for c, v in enumerate(BAD):
        x[0, 0, 0, at, c] = v
        h0[0, 0, 0, 3 + c] = v
    got = _scan_both(*data)
    for k in want:
        if k != "G":
            same(got[k][..., none], want[k][..., none])
    same(got["G"][..., none.start:C], want["G"][..., none.start:C])
    same(got["h"][0, 0, 0, :at, :3], want["h"][0, 0, 0, :at, :3])
    same(got["dg"][0, 0, 0, :at, :3], want["dg"][0, 0, 0, :at, :3])
    for k in ("dx", "dh0"):  # x and h0 are not in them
        same(got[k], want[k])
    assert not torch.isfinite(got["h"][0, 0, 0, at:, :3].float()).any() and not torch.isfinite(got["last"][..., :6]).any()
    assert not torch.isfinite(got["h"][0, 0, 0, :, 3:6].float()).any() and not torch.isfinite(got["G"][..., :6]).any()

    x, g, dh, X, h0, dl, lengths = data = finite
    for c, v in enumerate(BAD):
        dh[0, 0, 0, at, c] = v
        dl[0, 0, 0, 3 + c] = v
    got = _scan_both(*data)
    for k in ("h", "last", "states"):
        same(got[k], want[k])
    for k in ("dx", "dg", "dh0", "G"):
        same(got[k][..., none], want[k][..., none])
    for k in ("dx", "dg"):
        same(got[k][0, 0, 0, at + 1:, :3], want[k][0, 0, 0, at + 1:, :3])
    assert not torch.isfinite(got["dx"][0, 0, 0, :at + 1, :3].float()).any()
    assert not torch.isfinite(got["dx"][0, 0, 0, :, 3:6].float()).any()
    assert not torch.isfinite(got["dh0"][..., :6]).any() and not torch.isfinite(got["G"][..., :6]).any()
