"""Refusals of the token models' calls and their sizes, through the C ABI on the CPU: every
argument error is reported before anything would be launched."""

import ctypes

import numpy as np
import pytest

import paper_2211_00889_amd as nb
from paper_2211_00889_amd import _lib

MB = 1 << 20


class Arena:
    """Distinct made-up device addresses (never read: every call here is refused, or has no
    finished mini-batch)."""

    def __init__(self):
        self.next = 1 << 40

    def __call__(self, size=MB):
        p = self.next
        self.next += (size + 4095) // 4096 * 4096
        return p


def _mask(n, m, value=0):
    return np.full(n * m, value, np.uint8).tobytes()


def _defaults(call):
    a = Arena()
    n, m, b, T, dim, out, vocab = 2, 3, 2, 40, 24, 16, 50
    ws = {"workspace": a(64 * MB), "workspace_bytes": 64 * MB, "stream": None}
    common = {"n": n, "m": m, "T": T, "mask": _mask(n, m)}
    if call == "embed":
        return {"E": a(), "ld": 1200, "n": n, "m": m, "vocab": vocab, "dim": dim, "scale": 1.0, "tokens": a(),
                "T": T, "mask": common["mask"], "Y": a(), "ldy": dim, "dtype": 0, "stream": None}
    if call == "embed_grad":
        return {"dY": a(), "ldy": dim, "dtype": 0, "n": n, "m": m, "T": T, "tokens": a(), "vocab": vocab,
                "dim": dim, "scale": 1.0, "mask": common["mask"], "G": a(), "ld": 1200, **ws}
    if call == "scan":
        return {"x": a(), "g": a(), "ldx": dim, "dtype": 1, "n": n, "m": m, "batch": b, "T": T, "dim": dim,
                "bias": a(), "ld": 24, "lengths": a(), "mask": common["mask"], "h0": a(), "h": a(), "ldh": dim,
                "h_last": a(), "states": a(), **ws}
    if call == "scan_grad":
        return {"x": a(), "g": a(), "ldx": dim, "dtype": 1, "n": n, "m": m, "batch": b, "T": T, "dim": dim,
                "bias": a(), "ld": 24, "lengths": a(), "mask": common["mask"], "states": a(), "dh": a(),
                "lddh": dim, "dh_last": a(), "dx": a(), "dg": a(), "dh0": a(), "Gbias": a(), **ws}
    if call == "act_pack":
        return {"A": a(), "lda": dim, "dtype": 1, "n": n, "m": m, "T": T, "dim": dim, "mask": common["mask"],
                "packed": a(), "stream": None}
    if call == "act_unpack":
        return {"packed": a(), "n": n, "m": m, "T": T, "dim": dim, "mask": common["mask"], "A": a(), "lda": dim,
                "dtype": 1, "stream": None}
    return {"packed": a(), "dY": a(), "ldy": out, "n": n, "m": m, "T": T, "dim": dim, "out": out,
            "mask": common["mask"], "G": a(), "ld": 384, **ws}


def _call(name, **change):
    args = {**_defaults(name), **change}
    return getattr(_lib.load(), "nbsgd_" + name)(*args.values())


CALLS = ("embed", "embed_grad", "scan", "scan_grad", "act_pack", "act_unpack", "act_grad")


@pytest.mark.parametrize("name", CALLS)
def test_nothing_finished_is_valid(name):
    assert _call(name) == _lib.OK


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("change,status", [
    ({"n": 0}, _lib.E_SHAPE), ({"m": 0}, _lib.E_SHAPE), ({"n": 17}, _lib.E_UNSUPPORTED),
    ({"m": 65}, _lib.E_UNSUPPORTED), ({"T": -1}, _lib.E_SHAPE), ({"dim": 0}, _lib.E_SHAPE),
    ({"dim": 65537}, _lib.E_UNSUPPORTED), ({"T": (1 << 24) + 1}, _lib.E_UNSUPPORTED),
    ({"mask": None}, _lib.E_ARG)])
def test_sizes_and_mask(name, change, status):
    change = dict(change)
    if change.get("n", 0) > 16 or change.get("m", 0) > 64:
        change["mask"] = _mask(17, 65)
    assert _call(name, **change) == status
    assert _lib.load().nbsgd_last_error()


@pytest.mark.parametrize("name,arg,value,status", [
    ("embed", "dtype", 2, _lib.E_ARG), ("embed", "vocab", 0, _lib.E_SHAPE), ("embed", "ld", 1196, _lib.E_SHAPE),
    ("embed", "ld", 1201, _lib.E_SHAPE), ("embed", "ldy", 23, _lib.E_SHAPE), ("embed", "E", None, _lib.E_ARG),
    ("embed", "E", (1 << 40) + 4, _lib.E_ALIGN), ("embed", "tokens", None, _lib.E_ARG),
    ("embed", "tokens", (1 << 41) + 2, _lib.E_ALIGN), ("embed", "Y", (1 << 41) + 2, _lib.E_ALIGN),
    ("embed", "Y", None, _lib.E_ARG), ("embed", "T", 262145, _lib.E_UNSUPPORTED),
    ("embed", "vocab", (1 << 24) + 1, _lib.E_UNSUPPORTED),
    ("embed_grad", "dtype", -1, _lib.E_ARG), ("embed_grad", "G", None, _lib.E_ARG),
    ("embed_grad", "G", (1 << 41) + 8, _lib.E_ALIGN), ("embed_grad", "ld", 1198, _lib.E_SHAPE),
    ("embed_grad", "workspace", None, _lib.E_ARG), ("embed_grad", "workspace", (1 << 41) + 8, _lib.E_ALIGN),
    ("embed_grad", "workspace_bytes", 100, _lib.E_ARG), ("embed_grad", "dY", None, _lib.E_ARG),
    ("scan", "dtype", 7, _lib.E_ARG), ("scan", "batch", 0, _lib.E_SHAPE), ("scan", "ldx", 23, _lib.E_SHAPE),
    ("scan", "ldh", 0, _lib.E_SHAPE), ("scan", "x", None, _lib.E_ARG), ("scan", "g", (1 << 41) + 1, _lib.E_ALIGN),
    ("scan", "h", None, _lib.E_ARG), ("scan", "bias", (1 << 41) + 4, _lib.E_ALIGN), ("scan", "ld", 20, _lib.E_SHAPE),
    ("scan", "h0", (1 << 41) + 2, _lib.E_ALIGN), ("scan", "lengths", (1 << 41) + 1, _lib.E_ALIGN),
    ("scan_grad", "workspace", None, _lib.E_ARG), ("scan_grad", "ld", (1 << 41), _lib.E_SHAPE),
    ("scan", "batch", 1 << 21, _lib.E_UNSUPPORTED), ("scan", "ldx", (1 << 22) + 1, _lib.E_UNSUPPORTED),
    ("scan", "ldh", (1 << 22) + 1, _lib.E_UNSUPPORTED), ("scan_grad", "lddh", (1 << 22) + 1, _lib.E_UNSUPPORTED),
    ("scan_grad", "states", None, _lib.E_ARG), ("scan_grad", "dh", None, _lib.E_ARG),
    ("scan_grad", "dx", None, _lib.E_ARG), ("scan_grad", "dg", None, _lib.E_ARG),
    ("scan_grad", "lddh", 2, _lib.E_SHAPE), ("scan_grad", "Gbias", (1 << 41) + 4, _lib.E_ALIGN),
    ("scan_grad", "dh_last", (1 << 41) + 2, _lib.E_ALIGN), ("scan_grad", "workspace_bytes", 8, _lib.E_ARG),
    ("act_pack", "dtype", 3, _lib.E_ARG), ("act_pack", "A", None, _lib.E_ARG),
    ("act_pack", "packed", (1 << 41) + 8, _lib.E_ALIGN), ("act_pack", "packed", None, _lib.E_ARG),
    ("act_pack", "lda", 23, _lib.E_SHAPE), ("act_unpack", "lda", 23, _lib.E_SHAPE),
    ("act_unpack", "A", (1 << 41) + 1, _lib.E_ALIGN), ("act_unpack", "dtype", 3, _lib.E_ARG),
    ("act_grad", "out", 0, _lib.E_SHAPE), ("act_grad", "out", 65537, _lib.E_UNSUPPORTED),
    ("act_grad", "ld", 380, _lib.E_SHAPE), ("act_grad", "dY", (1 << 41) + 1, _lib.E_ALIGN),
    ("act_grad", "packed", None, _lib.E_ARG), ("act_grad", "G", None, _lib.E_ARG),
    ("act_grad", "T", 262145, _lib.E_UNSUPPORTED), ("act_grad", "ldy", (1 << 22) + 1, _lib.E_UNSUPPORTED),
])
def test_refusals(name, arg, value, status):
    change = {arg: value}
    if arg == "vocab" and value > 100:
        change["ld"] = 1 << 30
    assert _call(name, **change) == status, _lib.load().nbsgd_last_error()
    assert _lib.load().nbsgd_last_error()


@pytest.mark.parametrize("name,a,b", [
    ("embed", "Y", "E"), ("embed", "Y", "tokens"), ("embed_grad", "G", "dY"), ("embed_grad", "G", "workspace"),
    ("embed_grad", "workspace", "tokens"), ("scan", "h", "x"), ("scan", "h", "g"), ("scan", "h", "states"),
    ("scan", "states", "h0"), ("scan", "h_last", "states"), ("scan", "h_last", "lengths"),
    ("scan_grad", "dx", "x"), ("scan_grad", "dx", "dg"), ("scan_grad", "dg", "dh"), ("scan_grad", "Gbias", "bias"),
    ("scan_grad", "dh0", "states"), ("act_pack", "packed", "A"), ("act_unpack", "A", "packed"),
    ("act_grad", "G", "dY"), ("act_grad", "G", "packed")])
def test_overlap(name, a, b):
    d = _defaults(name)
    assert _call(name, **{a: d[b]}) == _lib.E_ARG
    assert b"overlap" in _lib.load().nbsgd_last_error()


def test_a_gradient_larger_than_the_memory():
    assert _call("act_grad", dim=65536, out=65536, ldy=65536, ld=1 << 32, n=5, m=4, mask=_mask(5, 4)) == \
        _lib.E_UNSUPPORTED


def test_the_forward_recurrence_of_one_tile_needs_no_workspace():
    assert _call("scan", T=256, workspace=None, workspace_bytes=0) == _lib.OK
    assert _call("scan", T=257, workspace=None, workspace_bytes=0) == _lib.E_ARG
    assert _call("scan", T=257, workspace_bytes=8) == _lib.E_ARG


def test_rows_side_by_side_do_not_overlap():
    p = 1 << 42
    assert _call("scan_grad", ldx=48, dx=p, dg=p + 48) == _lib.OK
    assert _call("scan_grad", ldx=48, dx=p + 48, dg=p) == _lib.OK
    assert _call("scan_grad", ldx=47, dx=p, dg=p + 48) == _lib.E_ARG  # the last element is the next row's first
    assert _call("scan_grad", ldx=48, dx=p, dg=p + 46) == _lib.E_ARG
    d = _defaults("scan")
    assert _call("scan", h_last=d["h0"]) == _lib.OK                   # the state in place
    d = _defaults("scan_grad")
    assert _call("scan_grad", dh0=d["dh_last"]) == _lib.OK


def test_empty_tokens_need_no_buffers():
    assert _call("embed", T=0, tokens=None, Y=None) == _lib.OK
    assert _call("act_pack", T=0, A=None, packed=None) == _lib.OK
    assert _call("scan", T=0, x=None, g=None, h=None, states=None, workspace=None, workspace_bytes=0) == _lib.OK


def test_sizes():
    assert nb.act_bytes(0, 5) == 0
    assert nb.act_bytes(1, 1) == 48          # 32 bytes of values, 4 of steps, whole sixteens
    assert nb.act_bytes(129, 10) == 5 * 10 * 32 + 2 * 10 * 4
    assert nb.act_bytes(262144, 65536) == 8192 * 65536 * 32 + 2048 * 65536 * 4
    assert nb.scan_workspace_bytes(1, 1, 1, 0, 8) == 0
    for call, args in ((nb.embed_workspace_bytes, (16, 64, 262144, 1 << 24, 65536)),
                       (nb.scan_workspace_bytes, (16, 64, 2, 1 << 24, 65536)),
                       (nb.act_workspace_bytes, (16, 64, 262144, 65536, 65536))):
        assert call(*args) >= 0
    for call, args in ((nb.act_bytes, (-1, 4)), (nb.embed_workspace_bytes, (1, 1, 1, 0, 4)),
                       (nb.scan_workspace_bytes, (1, 1, 0, 1, 4)), (nb.act_workspace_bytes, (1, 1, 1, 1, 0))):
        with pytest.raises(nb.NbsgdError) as e:
            call(*args)
        assert e.value.status == _lib.E_SHAPE
    assert _lib.load().nbsgd_act_bytes(4, 4, None) == _lib.E_ARG
    assert _lib.load().nbsgd_embed_workspace_bytes(1, 1, 1, 1, 1, None) == _lib.E_ARG
    assert ctypes.sizeof(ctypes.c_size_t) == 8


def test_binding_wants_device_tensors():
    torch = pytest.importorskip("torch")
    t = torch.zeros((1, 1, 4), dtype=torch.int32)
    with pytest.raises(TypeError):
        nb.embed(torch.zeros((1, 32)), 0, 4, t, np.ones((1, 1), np.uint8), torch.zeros((1, 1, 4, 8)))
    with pytest.raises(TypeError):
        nb.act_pack(torch.zeros((1, 1, 4, 8)), np.ones((1, 1), np.uint8), torch.zeros((1, 1, 48), dtype=torch.uint8))
