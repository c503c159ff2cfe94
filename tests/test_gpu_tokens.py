"""The token models' kernels against the fp64 oracle, element by element within the bound that
the oracle carries beside each result, at the sizes and masks where they can go wrong; then a
mini-batch in calls of its own and of many, captured and replayed, on another stream, and the
calls together as a training iteration uses them.

A bf16 result may be off by half a step of bf16 (2^-8 of its size) on top of the bound."""

import numpy as np
import pytest

import paper_2211_00889_amd as nb
from oracle import step as ostep
from oracle import tokens as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
SENTINEL = 7.0


def _say(msg):
    print(f"[case] {msg}", flush=True)


def _np(t):
    return t.detach().double().cpu().numpy()


def _close(name, got, want, bound, dtype=F32):
    """|got - want| <= bound + half a step of the result (and of what rounding the bound adds)."""
    got = _np(got)
    room = bound + HALF[dtype] * (np.abs(want) + bound) + 1e-37
    bad = ~(np.abs(got - want) <= room)
    assert not bad.any(), (f"{name}: {bad.sum()} of {bad.size} off, worst "
                           f"{np.nanmax(np.abs(got - want) / room):.3g} of the bound, first at "
                           f"{np.argwhere(bad)[0].tolist()}: {got[bad][0]} for {want[bad][0]}")


def _rows(shape, dtype, gap=0, shift=0, fill=None, rng=None, std=1.0):
    """A tensor of rows with `gap` untouched elements behind each and `shift` before the first;
    (view, whole buffer)."""
    width = shape[-1]
    rows = int(np.prod(shape[:-1]))
    whole = torch.full((shift + rows * (width + gap) + 8,), SENTINEL, dtype=dtype, device=DEV)
    view = whole[shift:shift + rows * (width + gap)].view(*shape[:-1], width + gap)[..., :width]
    if rng is not None:
        view.copy_(torch.from_numpy(rng.normal(0, std, shape).astype(np.float32)).to(dtype))
    elif fill is not None:
        view.fill_(fill)
    return view, whole


def _gaps_untouched(view, whole):
    probe = whole.clone()
    torch.as_strided(probe, view.shape, view.stride(), view.storage_offset()).fill_(SENTINEL)
    assert (probe == SENTINEL).all(), "written outside the rows"


def _mask(rng, n, m):
    mask = (rng.random((n, m)) < 0.6).astype(np.uint8)
    mask[rng.integers(n), rng.integers(m)] = 1
    return mask


def _ws(size):
    return torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------------ embeddings
EMBED = [
    # n, m, T, vocab, dim, gap, shift, offset
    (1, 1, 1, 1, 1, 0, 0, 0), (2, 3, 5, 7, 3, 2, 1, 4), (3, 2, 97, 50, 60, 0, 0, 8), (1, 2, 130, 33, 65, 3, 1, 4),
    (2, 2, 64, 300, 512, 8, 0, 0), (1, 1, 33, 1000, 513, 1, 3, 4), (2, 1, 300, 20, 1032, 0, 0, 0),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,m,T,vocab,dim,gap,shift,offset", EMBED)
def test_embed(n, m, T, vocab, dim, gap, shift, offset, dtype):
    rng = np.random.default_rng(T * dim)
    _say(f"embed {n}x{m} T={T} vocab={vocab} dim={dim} {dtype}")
    ld = (offset + vocab * dim + 3) // 4 * 4 + 4
    X = torch.from_numpy(rng.normal(0, 1, (n, ld)).astype(np.float32)).to(DEV)
    tok = rng.integers(-1, vocab + 1, (n, m, T)).astype(np.int32)
    mask = _mask(rng, n, m)
    Y, whole = _rows((n, m, T, dim), dtype, gap, shift)
    nb.embed(X, offset, vocab, torch.from_numpy(tok).to(DEV), mask, Y, scale=1.75)
    for i in range(n):
        E = _np(X[i, offset:offset + vocab * dim]).reshape(vocab, dim)
        for j in range(m):
            if mask[i, j]:
                want = orc.embed(E, tok[i, j], 1.75)
                _close("Y", Y[i, j], want, orc.U * np.abs(want), dtype)
            else:
                assert (Y[i, j] == SENTINEL).all()
    _gaps_untouched(Y, whole)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim,gap", [(64, 0), (64, 64), (192, 0), (520, 56), (1024, 0), (1000, 24)])
def test_embed_rows_on_lines(dim, gap, dtype):
    """Rows of whole 128-byte lines, with and without elements behind the last channel."""
    n, m, T, vocab = 2, 2, 133, 90
    rng = np.random.default_rng(dim)
    X = torch.from_numpy(rng.normal(0, 1, (n, vocab * dim)).astype(np.float32)).to(DEV)
    tok = rng.integers(-1, vocab + 1, (n, m, T)).astype(np.int32)
    Y, whole = _rows((n, m, T, dim), dtype, gap)
    nb.embed(X, 0, vocab, torch.from_numpy(tok).to(DEV), np.ones((n, m), np.uint8), Y, scale=0.5)
    for i in range(n):
        for j in range(m):
            want = orc.embed(_np(X[i]).reshape(vocab, dim), tok[i, j], 0.5)
            _close("Y", Y[i, j], want, orc.U * np.abs(want), dtype)
    _gaps_untouched(Y, whole)
    A = torch.full((n, m, T, dim), float("nan"), dtype=dtype, device=DEV)
    packed = torch.empty((n, m, nb.act_bytes(T, dim)), dtype=torch.uint8, device=DEV)
    nb.act_pack(Y, np.ones((n, m), np.uint8), packed)
    nb.act_unpack(packed, np.ones((n, m), np.uint8), A)
    back, whole = _rows((n, m, T, dim), dtype, gap + 1)
    nb.act_unpack(packed, np.ones((n, m), np.uint8), back)
    assert torch.equal(A, back)
    line, whole = _rows((n, m, T, dim), dtype, gap)
    nb.act_unpack(packed, np.ones((n, m), np.uint8), line)
    assert torch.equal(A, line)
    _gaps_untouched(line, whole)


def _tokens(rng, kind, shape, vocab):
    if kind == "uniform":
        return rng.integers(-1, vocab + 1, shape).astype(np.int32)
    if kind == "one":      # every token the same: the longest run there is
        return np.full(shape, vocab // 2, np.int32)
    if kind == "padding":  # nothing inside the table
        return np.where(rng.random(shape) < 0.5, -7, vocab + 3).astype(np.int32)
    return np.minimum(rng.zipf(1.3, shape) - 1, vocab - 1).astype(np.int32)  # "zipf"


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind,n,m,T,vocab,dim,gap,shift", [
    ("uniform", 1, 1, 1, 1, 1, 0, 0), ("uniform", 2, 2, 0, 9, 5, 0, 0), ("uniform", 2, 3, 97, 50, 60, 0, 0),
    ("one", 2, 1, 300, 11, 33, 1, 1), ("padding", 1, 2, 70, 13, 24, 0, 0), ("zipf", 2, 2, 1000, 200, 64, 0, 0),
    ("zipf", 1, 2, 1025, 5000, 12, 4, 2), ("one", 1, 1, 9001, 3, 7, 0, 0), ("zipf", 1, 1, 8192, 700, 20, 0, 0),
    ("uniform", 1, 1, 8193, 70000, 3, 0, 0), ("zipf", 1, 1, 20011, 333, 17, 3, 1), ("uniform", 1, 2, 40, 1, 520, 0, 0),
    ("zipf", 1, 1, 500, 64, 1300, 0, 0), ("zipf", 3, 1, 129, 257, 513, 7, 1), ("one", 1, 1, 64, 100, 128, 0, 0),
    ("uniform", 1, 1, 4097, 66000, 9, 0, 0),
])
def test_embed_grad(kind, n, m, T, vocab, dim, gap, shift, dtype):
    rng = np.random.default_rng(T + dim)
    _say(f"embed_grad {kind} {n}x{m} T={T} vocab={vocab} dim={dim} {dtype}")
    tok = _tokens(rng, kind, (n, m, T), vocab)
    mask = _mask(rng, n, m)
    dY, _ = _rows((n, m, T, dim), dtype, gap, shift, rng=rng)
    outside = torch.from_numpy((tok < 0) | (tok >= vocab)).to(DEV)
    dY[outside] = float("nan")  # rows of padding are not read
    offset = 4
    ld = offset + (vocab * dim + 3) // 4 * 4 + 4
    G = torch.full((n, m, ld), SENTINEL, device=DEV)
    nb.embed_grad(dY, torch.from_numpy(tok).to(DEV), mask, G, offset, vocab,
                  _ws(nb.embed_workspace_bytes(n, m, T, vocab, dim)), scale=0.75)
    for i in range(n):
        for j in range(m):
            if mask[i, j]:
                want, bound = orc.embed_grad(_np(dY[i, j]), tok[i, j], vocab, 0.75)
                _close("G", G[i, j, offset:offset + vocab * dim].view(vocab, dim), want, bound)
            else:
                assert (G[i, j] == SENTINEL).all()
    assert (G[:, :, :offset] == SENTINEL).all() and (G[:, :, offset + vocab * dim:] == SENTINEL).all()


@pytest.mark.parametrize("T", [129, 700, 1023, 1024, 1500, 2047, 2048, 4100])
@pytest.mark.parametrize("rows", [-1, 0, 1, 37])  # of the table, beside twice the tokens
def test_embed_grad_keeps_to_its_workspace(T, rows):
    """Where the pieces' number changes with the sizes: nothing behind the stated bytes is written."""
    n, m, vocab, dim = 2, 1, 2 * T + rows, 20
    rng = np.random.default_rng(T)
    _say(f"embed_grad T={T} vocab={vocab}")
    tok = _tokens(rng, "zipf", (n, m, T), vocab)
    dY, _ = _rows((n, m, T, dim), F32, rng=rng)
    G = torch.full((n, m, vocab * dim), SENTINEL, device=DEV)
    size = nb.embed_workspace_bytes(n, m, T, vocab, dim)
    guard = torch.full((size + 65536,), 7, dtype=torch.uint8, device=DEV)
    nb.embed_grad(dY, torch.from_numpy(tok).to(DEV), np.ones((n, m), np.uint8), G, 0, vocab, guard[:size])
    assert (guard[size:] == 7).all()
    for i in range(n):
        want, bound = orc.embed_grad(_np(dY[i, 0]), tok[i, 0], vocab, 1.0)
        _close("G", G[i, 0].view(vocab, dim), want, bound)


# ------------------------------------------------------------------ recurrence
SCAN = [
    # n, m, batch, T, dim, joint, lengths, bias, h0
    (1, 1, 1, 1, 1, 0, "full", 1, 1), (2, 2, 3, 1, 70, 0, "full", 1, 1), (1, 2, 2, 2, 64, 1, "ragged", 0, 0),
    (2, 2, 2, 33, 60, 0, "ragged", 1, 1), (1, 1, 2, 16, 9, 1, "ragged", 1, 1), (1, 1, 2, 17, 130, 0, "full", 1, 0),
    (1, 2, 1, 255, 33, 1, "full", 1, 1), (1, 1, 2, 256, 64, 0, "full", 1, 1), (1, 1, 3, 257, 65, 0, "ragged", 1, 1),
    (2, 1, 2, 700, 24, 1, "ragged", 1, 1), (1, 1, 1, 1500, 67, 0, "full", 0, 1), (1, 1, 4, 300, 7, 0, "empty", 1, 1),
    (1, 1, 1, 0, 12, 0, "full", 1, 1), (1, 1, 2, 64, 4, 0, "odd", 1, 1), (1, 1, 1, 5000, 5, 0, "full", 1, 1),
    (1, 1, 2, 513, 136, 1, "odd", 1, 1), (2, 3, 1, 40, 200, 0, "full", 1, 1),
]


def _scan_inputs(rng, n, m, b, T, C, joint, lengths, bias, h0, dtype):
    d = {}
    if joint:
        xg, _ = _rows((n, m, b, T, 2 * C), dtype, rng=rng)
        d["x"], d["g"] = xg[..., :C], xg[..., C:]
    else:
        d["x"], _ = _rows((n, m, b, T, C), dtype, 3, 1, rng=rng)
        d["g"], _ = _rows((n, m, b, T, C), dtype, 3, 2, rng=rng)
    d["X"] = torch.from_numpy(rng.normal(0, 1, (n, (C + 3) // 4 * 4 + 8)).astype(np.float32)).to(DEV)
    d["X"][:, 4:4 + C] += torch.linspace(-1, 6, C, device=DEV)
    if not bias:
        d["X"] = None
    d["h0"] = torch.from_numpy(rng.normal(0, 1, (n, m, b, C)).astype(np.float32)).to(DEV) if h0 else None
    lens = {"full": np.full((n, m, b), T), "ragged": rng.integers(0, T + 1, (n, m, b)),
            "empty": np.zeros((n, m, b)), "odd": np.resize([-3, T + 9], (n, m, b))}[lengths].astype(np.int32)
    d["lengths"] = None if lengths == "full" else torch.from_numpy(lens).to(DEV)
    d["len"] = np.clip(lens, 0, T)
    past = torch.arange(T, device=DEV) >= torch.from_numpy(d["len"]).to(DEV)[..., None]
    d["past"] = past
    for k in ("x", "g"):
        d[k][past] = float("nan")  # not read
    return d


def _scan_call(d, mask, n, m, b, T, C, dtype, states=True):
    h, whole = _rows((n, m, b, T, C), dtype, 1, 1)
    last = torch.full((n, m, b, C), SENTINEL, device=DEV)
    st = torch.full((n, m, b, -(-T // nb.SCAN_INTERVAL), C), SENTINEL, device=DEV) if states else None
    ws = _ws(nb.scan_workspace_bytes(n, m, b, T, C))
    nb.scan(d["x"], d["g"], mask, h, X=d["X"], offset=4 if d["X"] is not None else 0, h0=d["h0"], h_last=last,
            lengths=d["lengths"], states=st, workspace=ws)
    return h, whole, last, st


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,m,b,T,C,joint,lengths,bias,h0", SCAN)
def test_scan(n, m, b, T, C, joint, lengths, bias, h0, dtype):
    rng = np.random.default_rng(T + C)
    _say(f"scan {n}x{m}x{b} T={T} dim={C} {lengths} {dtype}")
    d = _scan_inputs(rng, n, m, b, T, C, joint, lengths, bias, h0, dtype)
    mask = _mask(rng, n, m)
    h, whole, last, st = _scan_call(d, mask, n, m, b, T, C, dtype)
    dh, _ = _rows((n, m, b, T, C), dtype, 2, 1, rng=rng)
    dh[d["past"]] = float("nan")
    dlast = torch.from_numpy(rng.normal(0, 1, (n, m, b, C)).astype(np.float32)).to(DEV) if h0 else None
    if joint:
        dxg, _ = _rows((n, m, b, T, 2 * C), dtype)
        dx, dg = dxg[..., :C], dxg[..., C:]
    else:
        dx, wx = _rows((n, m, b, T, C), dtype, 3, 1)
        dg, wg = _rows((n, m, b, T, C), dtype, 3, 2)
    dh0 = torch.full((n, m, b, C), SENTINEL, device=DEV)
    G = torch.full((n, m, (C + 3) // 4 * 4 + 8), SENTINEL, device=DEV)
    off = 4 if bias else 0
    nb.scan_grad(d["x"], d["g"], st, dh, mask, dx, dg, _ws(nb.scan_workspace_bytes(n, m, b, T, C)), X=d["X"], G=G,
                 offset=off, dh_last=dlast, dh0=dh0, lengths=d["lengths"])
    for i in range(n):
        bv = _np(d["X"][i, 4:4 + C]) if bias else np.zeros(C)
        for j in range(m):
            if not mask[i, j]:
                for t in (h[i, j], last[i, j], st[i, j], dx[i, j], dg[i, j], dh0[i, j], G[i, j]):
                    assert (t == SENTINEL).all()
                continue
            db, edb = np.zeros(C), np.zeros(C)
            for k in range(b):
                at, L = (i, j, k), int(d["len"][i, j, k])
                x, g = np.nan_to_num(_np(d["x"][at])), np.nan_to_num(_np(d["g"][at]))
                s0 = _np(d["h0"][at]) if h0 else np.zeros(C)
                (ho, before, s), (eh, eb, es) = orc.scan(x, g, bv, s0, L)
                _close("h", h[at], ho, eh, dtype)
                _close("h_last", last[at], s, es)
                _close("states", st[at], before[::nb.SCAN_INTERVAL], eb[::nb.SCAN_INTERVAL])
                l0 = _np(dlast[at]) if h0 else np.zeros(C)
                (gx, gg, g0, gb), (ex, eg, e0, egb) = orc.scan_grad(x, g, bv, s0, L, np.nan_to_num(_np(dh[at])), l0)
                _close("dx", dx[at], gx, ex, dtype)
                _close("dg", dg[at], gg, eg, dtype)
                _close("dh0", dh0[at], g0, e0)
                db, edb = db + gb, edb + egb + b * orc.U * np.abs(gg).sum(0)
            _close("dbias", G[i, j, off:off + C], db, edb)
    _gaps_untouched(h, whole)
    if not joint:
        _gaps_untouched(dx, wx)
        _gaps_untouched(dg, wg)
    assert (G[:, :, off + C:] == SENTINEL).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [1, 2, 3, 5, 6, 31, 33, 63, 65, 66, 67, 131])
def test_scan_widths(C, dtype):
    """Rows shorter than a lane's 8 bytes, and ones whose last lane has any part of them."""
    test_scan(1, 2, 2, 290, C, C % 2, "ragged", 1, 1, dtype)


def test_scan_extreme_gates():
    """Gates of 0 and 1, and infinite ones: the state is replaced, kept, and never NaN."""
    g = torch.tensor([float("inf"), -float("inf"), 200.0, -200.0, 88.0, -104.0, 1e38, -1e38], device=DEV)
    x = torch.full((1, 1, 1, 8, 3), 2.0, device=DEV)
    gg = g.view(1, 1, 1, 8, 1).expand(1, 1, 1, 8, 3).contiguous()
    h = torch.zeros_like(x)
    st = torch.zeros((1, 1, 1, 1, 3), device=DEV)
    h0 = torch.full((1, 1, 1, 3), -5.0, device=DEV)
    ws = _ws(nb.scan_workspace_bytes(1, 1, 1, 8, 3))
    nb.scan(x, gg, [[1]], h, h0=h0, states=st, workspace=ws)
    assert _np(h[0, 0, 0, :, 0]).tolist() == [-5.0, 2.0, 2.0, 2.0, 2.0, 2.0, 2.0, 2.0]
    dh, dx, dg = torch.ones_like(x), torch.empty_like(x), torch.empty_like(x)
    nb.scan_grad(x, gg, st, dh, [[1]], dx, dg, ws)
    assert torch.isfinite(dx).all() and torch.isfinite(dg).all()
    assert dx[0, 0, 0, 1, 0] > 0.9 and dx[0, 0, 0, 0, 0] == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_token_by_token(dtype):
    """Served one token at a time, the state in place, against the whole sequence."""
    rng = np.random.default_rng(5)
    b, T, C = 5, 20, 77
    d = _scan_inputs(rng, 1, 1, b, T, C, 0, "full", 1, 1, dtype)
    h, _, last, _ = _scan_call(d, [[1]], 1, 1, b, T, C, dtype, states=False)
    state = d["h0"].clone()
    ws = _ws(nb.scan_workspace_bytes(1, 1, b, 1, C))
    for t in range(T):
        x, g = d["x"][:, :, :, t:t + 1].contiguous(), d["g"][:, :, :, t:t + 1].contiguous()
        one = torch.empty_like(x)
        nb.scan(x, g, [[1]], one, X=d["X"], offset=4, h0=state, h_last=state, workspace=ws)
        for k in range(b):
            (ho, _, _), (eh, _, _) = orc.scan(_np(d["x"][0, 0, k]), _np(d["g"][0, 0, k]), _np(d["X"][0, 4:4 + C]),
                                              _np(d["h0"][0, 0, k]), T)
            _close("h", one[0, 0, k, 0], ho[t], eh[t], dtype)
    assert torch.allclose(state, last, rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("n,m,b,T,C,dtype", [
    (1, 2, 3, 700, 64, BF16), (2, 1, 2, 300, 96, F32), (1, 1, 1, 1030, 128, BF16), (8, 8, 5, 40, 128, BF16),
    (4, 8, 4, 700, 64, F32), (4, 8, 8, 520, 1024, BF16), (4, 8, 4, 530, 1024, F32),
])
def test_scan_rows_on_lines_and_off(n, m, b, T, C, dtype):
    """Rows on whole 128-byte lines, few and many bytes of them, against the same rows 4 elements
    further apart: bit for bit the same."""
    _say(f"scan lines {n}x{m}x{b} T={T} dim={C} {dtype}")
    gen = torch.Generator(device=DEV).manual_seed(T)
    shape = (n, m, b, T, C)
    x, g, dh = (torch.randn(shape, generator=gen, device=DEV).to(dtype) for _ in range(3))
    h0, dl = (torch.randn((n, m, b, C), generator=gen, device=DEV) for _ in range(2))
    X = torch.randn((n, C), generator=gen, device=DEV)
    lengths = torch.randint(0, T + 1, (n, m, b), generator=gen, device=DEV, dtype=torch.int32)
    mask, ws, results = np.ones((n, m), np.uint8), _ws(nb.scan_workspace_bytes(n, m, b, T, C)), []
    for gap in (0, 4):
        def rows(t=None):
            view = torch.full((*shape[:-1], C + gap), SENTINEL, dtype=dtype, device=DEV)[..., :C]
            return view if t is None else view.copy_(t)
        px, pg, pd, h, dx, dg = rows(x), rows(g), rows(dh), rows(), rows(), rows()
        last, st, d0 = torch.empty_like(h0), torch.empty((n, m, b, -(-T // nb.SCAN_INTERVAL), C), device=DEV), torch.empty_like(dl)
        G = torch.empty((n, m, C), device=DEV)
        nb.scan(px, pg, mask, h, X=X, h0=h0, h_last=last, lengths=lengths, states=st, workspace=ws)
        nb.scan_grad(px, pg, st, pd, mask, dx, dg, ws, X=X, G=G, dh_last=dl, dh0=d0, lengths=lengths)
        results.append([t.contiguous() for t in (h, last, st, dx, dg, d0, G)])
        if gap:
            assert all((torch.as_strided(t, (*shape[:-1], gap), t.stride(), t.storage_offset() + C) == SENTINEL).all()
                       for t in (h, dx, dg))
    assert all(torch.equal(p, q) for p, q in zip(*results))
    i, j, k = n - 1, m - 1, b - 1  # one sequence's first channels against the oracle
    L, few = int(lengths[i, j, k]), slice(0, 40)
    args = [_np(t[i, j, k][..., few]) for t in (x, g)] + [_np(X[i, few]), _np(h0[i, j, k, few]), L]
    (ho, _, s), (eh, _, es) = orc.scan(*args)
    _close("h", results[0][0][i, j, k][:, few], ho, eh, dtype)
    _close("h_last", results[0][1][i, j, k, few], s, es)
    (gx, gg, g0, _), (ex, eg, e0, _) = orc.scan_grad(*args, _np(dh[i, j, k][..., few]), _np(dl[i, j, k, few]))
    _close("dx", results[0][3][i, j, k][:, few], gx, ex, dtype)
    _close("dg", results[0][4][i, j, k][:, few], gg, eg, dtype)
    _close("dh0", results[0][5][i, j, k, few], g0, e0)


# --------------------------------------------------------- 8-bit activations
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,m,T,dim,gap,shift", [
    (1, 1, 1, 1, 0, 0), (2, 2, 31, 7, 1, 1), (1, 2, 32, 64, 0, 0), (2, 1, 33, 65, 3, 1), (1, 1, 129, 300, 0, 0),
    (2, 2, 200, 40, 8, 0), (1, 1, 161, 257, 0, 1), (1, 1, 1000, 8, 0, 0), (1, 1, 70, 1030, 0, 0),
])
def test_act_pack(n, m, T, dim, gap, shift, dtype):
    rng = np.random.default_rng(T * dim)
    _say(f"act_pack {n}x{m} T={T} dim={dim} {dtype}")
    A, _ = _rows((n, m, T, dim), dtype, gap, shift, rng=rng)
    A *= torch.exp(torch.linspace(-20, 20, dim, device=DEV))
    A[..., 0, :] = 0
    mask = _mask(rng, n, m)
    packed = torch.full((n, m, nb.act_bytes(T, dim)), 99, dtype=torch.uint8, device=DEV)
    nb.act_pack(A, mask, packed)
    out, whole = _rows((n, m, T, dim), dtype, gap + 1, shift)
    nb.act_unpack(packed, mask, out)
    wide = torch.zeros((n, m, T, dim), device=DEV)
    nb.act_unpack(packed, mask, wide)
    for i in range(n):
        for j in range(m):
            if mask[i, j]:
                q, step = orc.act8(_np(A[i, j]))
                assert np.array_equal(_np(out[i, j]), q * step) and np.array_equal(_np(wide[i, j]), q * step)
                _packed_layout(packed[i, j].cpu().numpy(), q, step, T, dim)
            else:
                assert (out[i, j] == SENTINEL).all() and (packed[i, j] == 99).all()
    _gaps_untouched(out, whole)


def _packed_layout(raw, q, step, T, dim):
    """The documented layout: blocks of 32 tokens, channels, tokens; then steps, four blocks a channel."""
    blocks = -(-T // 32)
    want = np.zeros((blocks * 32, dim), np.int8)
    want[:T] = q
    want = want.reshape(blocks, 32, dim).transpose(0, 2, 1)
    assert np.array_equal(raw[:blocks * dim * 32].view(np.int8).reshape(blocks, dim, 32), want)
    steps = np.zeros((-(-blocks // 4) * 4, dim), np.uint8)
    steps[:blocks] = (np.log2(step[::32]) + 127).astype(np.uint8)
    got = raw[blocks * dim * 32:][:steps.size].reshape(-1, dim, 4)
    assert np.array_equal(got, steps.reshape(-1, 4, dim).transpose(0, 2, 1))


def test_act_pack_borders():
    """Peaks that just reach or just miss 127 steps, the smallest and largest steps, infinities and NaNs."""
    A = torch.zeros((1, 1, 64, 12), device=DEV)
    peaks = [127.0, 127.49999, 127.5, 127.50001, 128.0, 2.0 ** -126, 2.0 ** -140, 3.4e38, 2.0 ** 127, 1.0]
    A[0, 0, 5, :10] = torch.tensor(peaks)
    A[0, 0, 6, :10] = -A[0, 0, 5, :10] / 3
    A[0, 0, 40, 10], A[0, 0, 41, 11] = float("inf"), float("nan")
    packed = torch.zeros((1, 1, nb.act_bytes(64, 12)), dtype=torch.uint8, device=DEV)
    nb.act_pack(A, [[1]], packed)
    out = torch.zeros_like(A)
    nb.act_unpack(packed, [[1]], out)
    q, step = orc.act8(_np(A[0, 0]))
    assert np.array_equal(_np(out[0, 0]), q * step, equal_nan=True)
    assert torch.isnan(out[0, 0, 32:, 10:]).all() and (out[0, 0, :32, 10:] == 0).all()


@pytest.mark.parametrize("n,m,T,dim,out,gap,shift", [
    (1, 1, 1, 1, 1, 0, 0), (2, 2, 0, 5, 6, 0, 0), (2, 2, 77, 96, 50, 0, 0), (1, 2, 32, 16, 64, 0, 0),
    (2, 1, 33, 70, 33, 3, 1), (1, 1, 129, 300, 130, 0, 0), (1, 1, 500, 128, 256, 8, 0), (1, 1, 64, 257, 260, 0, 0),
    (1, 1, 100, 520, 300, 4, 4), (3, 2, 200, 64, 128, 0, 0), (1, 1, 9000, 40, 72, 0, 0), (1, 1, 4096, 256, 264, 0, 0),
    (1, 1, 130, 33, 1030, 1, 0),
])
def test_act_grad(n, m, T, dim, out, gap, shift):
    rng = np.random.default_rng(T + dim + out)
    _say(f"act_grad {n}x{m} T={T} dim={dim} out={out}")
    A, _ = _rows((n, m, T, dim), BF16, rng=rng)
    A *= torch.exp(torch.linspace(-3, 3, dim, device=DEV))
    dY, _ = _rows((n, m, T, out), BF16, gap, shift, rng=rng)
    mask = _mask(rng, n, m)
    packed = torch.full((n, m, nb.act_bytes(T, dim)), 255, dtype=torch.uint8, device=DEV)
    nb.act_pack(A, mask, packed)
    offset = 8
    G = torch.full((n, m, offset + (dim * out + 3) // 4 * 4 + 4), SENTINEL, device=DEV)
    nb.act_grad(packed, dY, mask, G, offset, dim, _ws(nb.act_workspace_bytes(n, m, T, dim, out)))
    for i in range(n):
        for j in range(m):
            if mask[i, j]:
                q, step = orc.act8(_np(A[i, j]))
                want, bound = orc.act_grad(q * step, _np(dY[i, j]))
                _close("G", G[i, j, offset:offset + dim * out].view(dim, out), want, bound)
            else:
                assert (G[i, j] == SENTINEL).all()
    assert (G[:, :, :offset] == SENTINEL).all() and (G[:, :, offset + dim * out:] == SENTINEL).all()


@pytest.mark.parametrize("T", [1, 63, 64, 65, 128, 129, 192, 193, 257, 321, 384, 500])
@pytest.mark.parametrize("n,m,dim,out", [(16, 16, 33, 70), (16, 16, 270, 12), (8, 8, 130, 260), (2, 8, 500, 1030),
                                         (16, 16, 200, 250), (8, 16, 255, 497)])
def test_act_grad_many(n, m, dim, out, T):
    """So many mini-batches or columns that the larger tiles are taken, with every number of stages and
    of tokens in the last one."""
    rng = np.random.default_rng(T + dim)
    _say(f"act_grad {n}x{m} T={T} dim={dim} out={out}")
    A, _ = _rows((n, m, T, dim), BF16, rng=rng)
    dY, _ = _rows((n, m, T, out), BF16, rng=rng)
    packed = torch.empty((n, m, nb.act_bytes(T, dim)), dtype=torch.uint8, device=DEV)
    mask = np.ones((n, m), np.uint8)
    nb.act_pack(A, mask, packed)
    values = torch.empty_like(A)
    nb.act_unpack(packed, mask, values)
    G = torch.full((n, m, (dim * out + 3) // 4 * 4), SENTINEL, device=DEV)
    nb.act_grad(packed, dY, mask, G, 0, dim, _ws(nb.act_workspace_bytes(n, m, T, dim, out)))
    for i in range(n):
        for j in {0, m // 2, m - 1} if i in (0, n // 2, n - 1) else {(i * 5) % m}:
            want, bound = orc.act_grad(_np(values[i, j]), _np(dY[i, j]))
            _close("G", G[i, j, :dim * out].view(dim, out), want, bound)


@pytest.mark.parametrize("out", [1, 2, 3, 5, 6, 7, 9])
@pytest.mark.parametrize("T", [64, 65, 67, 71, 128, 131])
def test_act_grad_narrow_rows(T, out):
    """Rows shorter than the 16 bytes of a load, whose last ones end with the buffer; what stands
    behind them, NaNs here, is in no result."""
    rng = np.random.default_rng(T + out)
    _say(f"act_grad T={T} out={out}")
    dim = 20
    A, _ = _rows((1, 1, T, dim), BF16, rng=rng)
    dY, whole = _rows((1, 1, T, out), BF16, rng=rng)
    whole[T * out:] = float("nan")
    packed = torch.zeros((1, 1, nb.act_bytes(T, dim)), dtype=torch.uint8, device=DEV)
    nb.act_pack(A, [[1]], packed)
    G = torch.empty((1, 1, dim * out), device=DEV)
    nb.act_grad(packed, dY, [[1]], G, 0, dim)
    q, step = orc.act8(_np(A[0, 0]))
    want, bound = orc.act_grad(q * step, _np(dY[0, 0]))
    _close("G", G[0, 0].view(dim, out), want, bound)


# ---------------------------------------------- far rows, states in place
def test_rows_beyond_32_bits():
    """Rows so far apart that byte offsets pass 2^32, and a table of more than 2^31 floats."""
    rng = np.random.default_rng(2)
    T, C, far = 520, 72, 1 << 22
    _say("scan, rows 2^22 apart")
    xg = torch.empty((1, 1, 1, T, far), dtype=BF16, device=DEV)
    dxg = torch.empty((1, 1, 1, T, far), dtype=BF16, device=DEV)
    near = _rows((2, T, C), BF16, rng=rng)[0].contiguous()
    x, g, dx, dg = (t[..., o:o + C] for t in (xg, dxg) for o in (0, far // 2))
    x.copy_(near[0]), g.copy_(near[1])
    h = torch.empty((1, 1, 1, T, C), dtype=BF16, device=DEV)
    dh = _rows(h.shape, BF16, rng=rng)[0].contiguous()
    st = torch.empty((1, 1, 1, 3, C), device=DEV)
    ws = _ws(nb.scan_workspace_bytes(1, 1, 1, T, C))
    nb.scan(x, g, [[1]], h, states=st, workspace=ws)
    nb.scan_grad(x, g, st, dh, [[1]], dx, dg, ws)
    v = _np(near)
    (ho, _, _), (eh, _, _) = orc.scan(v[0], v[1], np.zeros(C), np.zeros(C), T)
    (gx, gg, _, _), (ex, eg, _, _) = orc.scan_grad(v[0], v[1], np.zeros(C), np.zeros(C), T, _np(dh[0, 0, 0]), np.zeros(C))
    _close("h", h[0, 0, 0], ho, eh, BF16)
    _close("dx", dx[0, 0, 0], gx, ex, BF16)
    _close("dg", dg[0, 0, 0], gg, eg, BF16)
    del xg, dxg, x, g, dx, dg

    V, D = (1 << 20) + 5, 2100
    _say("embed, a table of 2.2e9 floats")
    X = torch.empty((1, V * D), device=DEV)
    tok = np.array([V - 1, 0, V - 3, V - 1, -1, V], np.int32)
    for t in (0, V - 3, V - 1):
        X[0, t * D:(t + 1) * D] = torch.from_numpy(rng.normal(size=D).astype(np.float32)).to(DEV)
    tokens = torch.from_numpy(tok).to(DEV).view(1, 1, 6)
    Y = torch.empty((1, 1, 6, D), device=DEV)
    nb.embed(X, 0, V, tokens, [[1]], Y)
    for k, t in enumerate(tok[:4]):
        assert torch.equal(Y[0, 0, k], X[0, int(t) * D:(int(t) + 1) * D])
    assert (Y[0, 0, 4:] == 0).all()
    for T in (6, 150):  # few tokens, and sorted ones
        X.fill_(SENTINEL)
        many = torch.full((1, 1, T), -1, dtype=torch.int32, device=DEV)
        many[0, 0, :6] = tokens[0, 0]
        dY = _rows((1, 1, T, D), F32, rng=rng)[0].contiguous()
        nb.embed_grad(dY, many, [[1]], X.view(1, 1, -1), 0, V, _ws(nb.embed_workspace_bytes(1, 1, T, V, D)))
        assert torch.equal(X[0, (V - 1) * D:], dY[0, 0, 0] + dY[0, 0, 3])
        assert torch.equal(X[0, :D], dY[0, 0, 1]) and torch.equal(X[0, (V - 3) * D:(V - 2) * D], dY[0, 0, 2])
        assert int(torch.count_nonzero(X)) == sum(int(torch.count_nonzero(t)) for t in (
            X[0, (V - 1) * D:], X[0, :D], X[0, (V - 3) * D:(V - 2) * D]))
    del X

    T, D, N = 300, 40, 24
    _say("act_grad, rows 2^22 apart")
    wide = torch.empty((1, 2, T, far), dtype=BF16, device=DEV)
    dY = wide[..., far - N:]
    dY.copy_(_rows((1, 2, T, N), BF16, rng=rng)[0])
    A = torch.empty((1, 2, T, far), dtype=BF16, device=DEV)[..., far - D:]
    A.copy_(_rows((1, 2, T, D), BF16, rng=rng)[0])
    packed = torch.empty((1, 2, nb.act_bytes(T, D)), dtype=torch.uint8, device=DEV)
    G = torch.empty((1, 2, D * N), device=DEV)
    nb.act_pack(A, [[1, 1]], packed)
    nb.act_grad(packed, dY, [[1, 1]], G, 0, D, _ws(nb.act_workspace_bytes(1, 2, T, D, N)))
    q, step = orc.act8(_np(A[0, 1]))
    want, bound = orc.act_grad(q * step, _np(dY[0, 1]))
    _close("G", G[0, 1].view(D, N), want, bound)
    A.fill_(SENTINEL)
    nb.act_unpack(packed, [[0, 1]], A)
    assert np.array_equal(_np(A[0, 1]), q * step) and (A[0, 0] == SENTINEL).all()


@pytest.mark.parametrize("T,C", [(16, 20), (200, 70), (700, 33), (3000, 130)])
def test_states_in_place(T, C):
    """h_last over h0 and dh0 over dh_last, in one tile and split over workgroups."""
    rng = np.random.default_rng(T)
    d = _scan_inputs(rng, 1, 2, 1, T, C, 0, "ragged", 1, 1, F32)
    mask = [[1, 1]]
    h, _, last, st = _scan_call(d, mask, 1, 2, 1, T, C, F32)
    state, h2 = d["h0"].clone(), torch.empty_like(h)
    ws = _ws(nb.scan_workspace_bytes(1, 2, 1, T, C))
    nb.scan(d["x"], d["g"], mask, h2, X=d["X"], offset=4, h0=state, h_last=state, lengths=d["lengths"], workspace=ws)
    assert torch.equal(h2, h) and torch.equal(state, last)
    dh = _rows(h.shape, F32, rng=rng)[0].contiguous()
    out = []
    for same in (False, True):
        dl = torch.linspace(-1, 1, 2 * C, device=DEV).view(1, 2, 1, C).contiguous()
        dx, _ = _rows(h.shape, F32, 3, 1)
        dg, _ = _rows(h.shape, F32, 3, 2)
        d0 = dl if same else torch.empty_like(dl)
        nb.scan_grad(d["x"], d["g"], st, dh, mask, dx, dg, ws, X=d["X"], offset=4, dh_last=dl, dh0=d0, lengths=d["lengths"])
        out.append((dx.clone(), dg.clone(), d0))
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_infinite_bias_and_empty_sequences():
    """A bias of -inf passes x through, one of +inf keeps the state; where a sequence has ended the state
    stays whatever the bias is."""
    T, C = 600, 3
    X = torch.tensor([[0.0, 0, 0, 0, -float("inf"), float("inf"), 0.0, 0]], device=DEV)
    x, g = torch.full((1, 1, 2, T, C), 3.0, device=DEV), torch.zeros((1, 1, 2, T, C), device=DEV)
    h0 = torch.full((1, 1, 2, C), 5.0, device=DEV)
    h, last = torch.empty_like(x), torch.empty_like(h0)
    lengths = torch.tensor([[[0, 300]]], dtype=torch.int32, device=DEV)
    nb.scan(x, g, [[1]], h, X=X, offset=4, h0=h0, h_last=last, lengths=lengths,
            workspace=_ws(nb.scan_workspace_bytes(1, 1, 2, T, C)))
    assert (last[0, 0, 0] == 5).all() and (h[0, 0, 0] == 0).all()
    assert last[0, 0, 1].tolist() == [3.0, 5.0, 3.0] and (h[0, 0, 1, 300:] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [9, 200, 600])
def test_lowest_biases(T, dtype):
    """Biases of the lowest finite values: the tokens before the length replace the state, the ones
    behind it leave it alone, backward too."""
    lowest = -3.4028234663852886e38
    X = torch.tensor([[0.0, 0, 0, 0, lowest, -3.39e38, -3.2e38, -float("inf"), 0.0, 0, 0, 0]], device=DEV)
    C, L = 4, T - 4
    x, g = torch.full((1, 1, 1, T, C), 3.0, dtype=dtype, device=DEV), torch.zeros((1, 1, 1, T, C), dtype=dtype, device=DEV)
    h0 = torch.full((1, 1, 1, C), 5.0, device=DEV)
    h, last = torch.empty_like(x), torch.empty_like(h0)
    st = torch.empty((1, 1, 1, -(-T // nb.SCAN_INTERVAL), C), device=DEV)
    lengths = torch.tensor([[[L]]], dtype=torch.int32, device=DEV)
    ws = _ws(nb.scan_workspace_bytes(1, 1, 1, T, C))
    nb.scan(x, g, [[1]], h, X=X, offset=4, h0=h0, h_last=last, lengths=lengths, states=st, workspace=ws)
    assert (last == 3).all() and (h[0, 0, 0, :L] == 3).all() and (h[0, 0, 0, L:] == 0).all()
    dx, dg, dl = torch.empty_like(x), torch.empty_like(x), torch.full_like(h0, 2.0)
    nb.scan_grad(x, g, st, torch.ones_like(x), [[1]], dx, dg, ws, X=X, offset=4, dh_last=dl, dh0=last, lengths=lengths)
    want = torch.ones(T, device=DEV)
    want[L - 1], want[L:] = 3, 0
    assert (dx[0, 0, 0].float() == want[:, None]).all() and (dg == 0).all() and (last == 0).all()


# ------------------------------------------------------------- all of them
def _one_pass(d, mask, sel=None):
    """Every call on the mini-batches of `mask`; the outputs by name.  `sel`: only mini-batch
    (i, j), in buffers of its own."""
    n, m, T, b, V, D, C = d["sizes"]
    pick = (lambda t: t) if sel is None else (lambda t: t[sel[0]:sel[0] + 1, sel[1]:sel[1] + 1].contiguous())
    X = d["X"] if sel is None else d["X"][sel[0]:sel[0] + 1].contiguous()
    if sel is not None:
        n, m, mask = 1, 1, np.ones((1, 1), np.uint8)
    tok, dY, x, g, dh, A = (pick(d[k]) for k in ("tokens", "dY", "x", "g", "dh", "A"))
    o = {k: torch.full(s, SENTINEL, dtype=t, device=DEV) for k, s, t in (
        ("Y", (n, m, T, D), BF16), ("G", (n, m, X.shape[1]), F32), ("h", x.shape, x.dtype), ("dx", x.shape, x.dtype),
        ("dg", x.shape, x.dtype), ("last", (n, m, b, C), F32), ("dh0", (n, m, b, C), F32),
        ("states", (n, m, b, -(-x.shape[3] // nb.SCAN_INTERVAL), C), F32),
        ("packed", (n, m, nb.act_bytes(T, D)), torch.uint8))}
    w = [_ws(nb.embed_workspace_bytes(n, m, T, V, D)), _ws(nb.scan_workspace_bytes(n, m, b, x.shape[3], C)),
         _ws(nb.act_workspace_bytes(n, m, T, D, D))]
    o["w"] = w

    def run():
        nb.embed(X, 0, V, tok, mask, o["Y"], scale=2.0)
        nb.scan(x, g, mask, o["h"], X=X, offset=V * D, h_last=o["last"], states=o["states"], workspace=w[1])
        nb.scan_grad(x, g, o["states"], dh, mask, o["dx"], o["dg"], w[1], X=X, G=o["G"], offset=V * D, dh0=o["dh0"])
        nb.act_pack(A, mask, o["packed"])
        nb.act_grad(o["packed"], dY, mask, o["G"], V * D + C, D, w[2])
        nb.embed_grad(dY, tok, mask, o["G"], 0, V, w[0], scale=2.0)

    return run, o


def _pass_inputs(seed, n=2, m=3, b=2, L=300, V=77, D=136, C=72):
    rng = np.random.default_rng(seed)
    T = b * L
    d = {"sizes": (n, m, T, b, V, D, C),
         "X": torch.from_numpy(rng.normal(0, 1, (n, V * D + C + D * D)).astype(np.float32)).to(DEV),
         "tokens": torch.from_numpy(_tokens(rng, "zipf", (n, m, T), V)).to(DEV)}
    for k, s in (("dY", (n, m, T, D)), ("A", (n, m, T, D)), ("x", (n, m, b, L, C)), ("g", (n, m, b, L, C)),
                 ("dh", (n, m, b, L, C))):
        d[k] = _rows(s, BF16, rng=rng)[0].contiguous()
    return d


OUT = ("Y", "G", "h", "dx", "dg", "last", "dh0", "states", "packed")


@pytest.mark.parametrize("L", [12, 300, 2100])
def test_results_of_a_mini_batch_are_its_own(L):
    """In a call of all, of some and of its own, bit for bit."""
    d = _pass_inputs(L, L=L)
    n, m = d["sizes"][:2]
    run, whole = _one_pass(d, np.ones((n, m), np.uint8))
    run()
    some_mask = np.array([[1, 0, 1], [0, 0, 1]], np.uint8)
    run, some = _one_pass(d, some_mask)
    run()
    for i in range(n):
        for j in range(m):
            run, one = _one_pass(d, None, (i, j))
            run()
            for k in OUT:
                assert torch.equal(one[k][0, 0], whole[k][i, j]), (k, i, j)
                if some_mask[i, j]:
                    assert torch.equal(some[k][i, j], whole[k][i, j]), (k, i, j)


def test_captured_and_replayed():
    """Captured once, replayed on new inputs with eager calls between, against the eager results."""
    d = _pass_inputs(1)
    mask = np.array([[1, 1, 0], [1, 0, 1]], np.uint8)
    run, o = _one_pass(d, mask)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(2, 6):
        new = _pass_inputs(seed)
        for k in ("X", "tokens", "dY", "A", "x", "g", "dh"):
            d[k].copy_(new[k])
        eager_run, want = _one_pass(new, mask)
        eager_run()
        for k in OUT:
            o[k].fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        done = torch.from_numpy(mask.astype(bool)).to(DEV)
        for k in OUT:
            assert torch.equal(o[k][done], want[k][done]), (k, seed)


def test_on_another_stream():
    d = _pass_inputs(7)
    mask = np.ones((2, 3), np.uint8)
    run, want = _one_pass(d, mask)
    run()
    run, o = _one_pass(d, mask)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    for k in OUT:
        assert torch.equal(o[k], want[k]), k


def test_two_streams_at_once():
    """Two callers with buffers of their own, taking turns at the launches."""
    mask = np.ones((2, 3), np.uint8)
    data = [_pass_inputs(seed, L=700) for seed in (8, 9)]
    want = []
    for d in data:
        run, o = _one_pass(d, mask)
        run()
        want.append(o)
    pairs = [_one_pass(d, mask) for d in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in data]
    for _ in range(4):
        for s, (run, _) in zip(streams, pairs):
            with torch.cuda.stream(s):
                run()
    torch.cuda.synchronize()
    for (_, o), w in zip(pairs, want):
        for k in OUT:
            assert torch.equal(o[k], w[k]), k


@pytest.mark.parametrize("n,m,T,dim,out", [(16, 16, 200, 200, 248), (8, 16, 321, 255, 500), (2, 8, 2100, 500, 1032)])
def test_act_grad_is_its_own_in_larger_tiles(n, m, T, dim, out):
    """One of many mini-batches, whose call takes larger tiles, against the same one alone."""
    rng = np.random.default_rng(T)
    A, dY = (_rows((n, m, T, w), BF16, rng=rng)[0].contiguous() for w in (dim, out))
    packed = torch.empty((n, m, nb.act_bytes(T, dim)), dtype=torch.uint8, device=DEV)
    mask = np.ones((n, m), np.uint8)
    nb.act_pack(A, mask, packed)
    G = torch.empty((n, m, dim * out), device=DEV)
    nb.act_grad(packed, dY, mask, G, 0, dim, _ws(nb.act_workspace_bytes(n, m, T, dim, out)))
    for i, j in ((0, 0), (n - 1, m - 1), (n // 2, 1)):
        one = torch.empty((1, 1, dim * out), device=DEV)
        nb.act_grad(packed[i:i + 1, j:j + 1].contiguous(), dY[i:i + 1, j:j + 1].contiguous(), [[1]], one, 0, dim,
                    _ws(nb.act_workspace_bytes(1, 1, T, dim, out)))
        assert torch.equal(one[0, 0], G[i, j]), (i, j)


def test_training_iteration():
    """Embeddings, a joint projection whose input is kept in 8 bits, the recurrence, a squared loss, and
    back: every gradient lands in its place of G and the fused step takes it.  Against the same model
    in float64 with autograd, with the activations' 8-bit values where the kernels use them."""
    n, m, b, L, V, D, C = 2, 2, 2, 70, 40, 48, 28
    T, scale = b * L, 3.0
    oW, oB = V * D, V * D + D * 2 * C
    P = oB + C
    rng = np.random.default_rng(11)
    X = torch.from_numpy(rng.normal(0, 0.2, (n, P)).astype(np.float32)).to(DEV)
    tok = torch.from_numpy(rng.integers(0, V, (n, m, T)).astype(np.int32)).to(DEV)
    target = torch.from_numpy(rng.normal(0, 1, (n, m, b, L, C)).astype(np.float32)).to(DEV)
    mask = np.array([[1, 1], [1, 0]], np.uint8)
    G = torch.zeros((n, m, P), device=DEV)
    E = torch.zeros((n, m, T, D), device=DEV)
    packed = torch.zeros((n, m, nb.act_bytes(T, D)), dtype=torch.uint8, device=DEV)
    nb.embed(X, 0, V, tok, mask, E, scale=scale)
    nb.act_pack(E, mask, packed)
    W = X[:, oW:oB].view(n, 1, D, 2 * C)
    xg = torch.matmul(E, W).view(n, m, b, L, 2 * C)
    h = torch.zeros((n, m, b, L, C), device=DEV)
    states = torch.zeros((n, m, b, 1, C), device=DEV)
    ws = _ws(nb.scan_workspace_bytes(n, m, b, L, C))
    nb.scan(xg[..., :C], xg[..., C:], mask, h, X=X, offset=oB, states=states, workspace=ws)
    dh = (h - target) / T
    dxg = torch.zeros_like(xg)
    nb.scan_grad(xg[..., :C], xg[..., C:], states, dh, mask, dxg[..., :C], dxg[..., C:], ws, X=X, G=G, offset=oB)
    d16 = dxg.view(n, m, T, 2 * C).to(BF16)
    nb.act_grad(packed, d16, mask, G, oW, D, _ws(nb.act_workspace_bytes(n, m, T, D, 2 * C)))
    dE = torch.matmul(dxg.view(n, m, T, 2 * C), W.transpose(-1, -2).contiguous())
    nb.embed_grad(dE, tok, mask, G, 0, V, _ws(nb.embed_workspace_bytes(n, m, T, V, D)), scale=scale)
    for i in range(n):
        p = X[i].double().cpu().requires_grad_(True)
        for j in range(m):
            if not mask[i, j]:
                assert (G[i, j] == 0).all()
                continue
            p.grad = None
            Eo = scale * p[:oW].view(V, D)[tok[i, j].long().cpu()]
            pre = (Eo @ p[oW:oB].view(D, 2 * C)).view(b, L, 2 * C)
            a, s, hs = torch.sigmoid(pre[..., C:] + p[oB:]), torch.zeros(b, C).double(), []
            for t in range(L):
                s = a[:, t] * s + (1 - a[:, t]) * pre[:, t, :C]
                hs.append(s)
            pre.retain_grad()
            (0.5 * (torch.stack(hs, 1) - target[i, j].double().cpu()).pow(2).sum() / T).backward()
            want, got = p.grad.numpy(), _np(G[i, j])
            # the projection's gradient from the input's 8-bit values and the bf16 gradient of its output
            q, st = orc.act8(_np(E[i, j]))
            dP = pre.grad.view(T, 2 * C).numpy()
            wW = (q * st).T @ dP
            # half a step of bf16 in dP; everything else is 32-bit arithmetic
            room = 2.0 ** -8 * (np.abs(q * st).T @ np.abs(dP)) * 1.01 + 1e-5 * np.abs(wW).max()
            assert (np.abs(got[oW:oB].reshape(D, 2 * C) - wW) <= room).all()
            for lo, hi in ((0, oW), (oB, P)):
                # 32-bit arithmetic through a recurrence of 70 steps and sums of 140 terms: a few
                # hundred roundings of 2^-24 of the block's largest entry
                assert np.abs(got[lo:hi] - want[lo:hi]).max() <= 1e-4 * np.abs(want[lo:hi]).max()
    X0, G0 = _np(X), _np(G)
    Vm = torch.zeros_like(X)
    Wm = nb.w_ring(n)
    nb.step(X, Vm, G, mask, Wm, 0.1, 0.9, nb.MIX_THEN_STEP)
    Xo, _ = ostep.step(X0, np.zeros((n, P)), G0, mask, Wm, np.float32(0.1), np.float32(0.9), ostep.MIX_THEN_STEP)
    assert np.abs(_np(X) - Xo).max() <= 1e-5
