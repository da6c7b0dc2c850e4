"""The training-step operators' C ABI without a device: symbols, sizes, argument checks; and the profile's fit."""
import ctypes
import os
import re

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000  # a pointer that no refused call may follow


def _declared():
    text = open(os.path.join(ROOT, "include", "ones_train.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(ones_[a-z_0-9]+)\s*\(", text)))


def test_library_exports_and_binding_covers_every_declared_symbol():
    from paper_2108_03645_b200 import build, train
    lib = ctypes.CDLL(build.build())
    names = _declared()
    assert len(names) == 11
    for n in names:
        assert hasattr(lib, n), n
    assert sorted(train._SIGNATURES) == names


def _lib():
    from paper_2108_03645_b200 import train
    return train.lib()


def test_workspace_sizes():
    L = _lib()
    assert L.ones_layer_norm_workspace_bytes(-1, 8) == 0 and L.ones_layer_norm_workspace_bytes(8, 0) == 0
    assert L.ones_layer_norm_workspace_bytes(1, 8) >= 64
    # the sums over rows are kept per block, however many rows there are
    assert L.ones_layer_norm_workspace_bytes(1 << 30, 1024) == L.ones_layer_norm_workspace_bytes(1 << 20, 1024)
    assert L.ones_linear_ce_workspace_bytes(8, 0) == 0 and L.ones_linear_ce_workspace_bytes(-1, 8) == 0
    # far below the logits
    assert 0 < L.ones_linear_ce_workspace_bytes(8192, 128000) < 8192 * 128000 * 2 // 16
    assert L.ones_linear_ce_backward_workspace_bytes(8, 8, 8, 100) == 0
    whole = L.ones_linear_ce_backward_workspace_bytes(8192, 2048, 128000, 0)
    small = L.ones_linear_ce_backward_workspace_bytes(8192, 2048, 128000, 1024)
    assert 0 < small < whole < 8192 * 128000 * 2
    assert L.ones_orthogonalize_workspace_bytes(0, 8, 8) == 0 and L.ones_orthogonalize_workspace_bytes(1, 0, 8) == 0
    assert L.ones_orthogonalize_workspace_bytes(2, 200, 300) > 2 * 200 * 300 * 2
    assert 0 < L.ones_orthogonalize_workspace_bytes(1000, 128, 512) < 1024  # such matrices stay on the chip
    big = L.ones_orthogonalize_workspace_bytes(16, 65536, 4096)  # past 32 bits
    assert big > 2 * 16 * 65536 * 4096 * 2


NULL, PARAM, ALIGN, SPACE = -1, -3, -4, -5


@pytest.mark.parametrize("change, want", [
    ({"rows": -1}, PARAM), ({"cols": 0}, PARAM), ({"cols": 65537}, PARAM), ({"eps": 0.0}, PARAM), ({"eps": float("nan")}, PARAM),
    ({"type": 3}, PARAM), ({"type": 1, "wtype": 2}, PARAM), ({"ldx": 63}, PARAM), ({"ldy": 1}, PARAM), ({"x": None}, NULL),
    ({"y": None}, NULL), ({"x": P + 2}, ALIGN), ({"w": P + 1}, ALIGN)])
def test_layer_norm_refuses(change, want):
    a = dict(x=P, ldx=64, w=P, b=P, rows=4, cols=64, eps=1e-5, type=0, wtype=0, y=P, ldy=64, mean=P, rstd=P) | change
    assert _lib().ones_layer_norm(a["x"], a["ldx"], a["w"], a["b"], a["rows"], a["cols"], a["eps"], a["type"], a["wtype"], a["y"],
                                  a["ldy"], a["mean"], a["rstd"], None) == want


@pytest.mark.parametrize("change, want", [
    ({"rows": -1}, PARAM), ({"cols": 0}, PARAM), ({"type": -1}, PARAM), ({"lddy": 1}, PARAM), ({"lddx": 1}, PARAM), ({"dy": None}, NULL),
    ({"mean": None}, NULL), ({"dx": None}, NULL), ({"ws": None}, NULL), ({"dx": P + 2}, ALIGN), ({"dw": P + 2}, ALIGN),
    ({"ws": P + 16}, ALIGN), ({"size": 64}, SPACE)])
def test_layer_norm_backward_refuses(change, want):
    a = dict(dy=P, lddy=64, x=P, ldx=64, mean=P, rstd=P, w=P, rows=4, cols=64, type=0, wtype=0, dx=P, lddx=64, dw=P, db=P, ws=P,
             size=1 << 20) | change
    assert _lib().ones_layer_norm_backward(a["dy"], a["lddy"], a["x"], a["ldx"], a["mean"], a["rstd"], a["w"], a["rows"], a["cols"],
                                           a["type"], a["wtype"], a["dx"], a["lddx"], a["dw"], a["db"], a["ws"], a["size"],
                                           None) == want


@pytest.mark.parametrize("change, want", [
    ({"rows": -1}, PARAM), ({"cols": 0}, PARAM), ({"vocab": 0}, PARAM), ({"type": 0}, PARAM), ({"ldh": 63}, PARAM), ({"ldw": 8}, PARAM),
    ({"h": None}, NULL), ({"t": None}, NULL), ({"lse": None}, NULL), ({"ws": None}, NULL), ({"h": P + 8}, ALIGN), ({"ldw": 68}, ALIGN),
    ({"ws": P + 128}, ALIGN), ({"size": 16}, SPACE)])
def test_linear_ce_refuses(change, want):
    a = dict(h=P, ldh=64, w=P, ldw=64, t=P, rows=4, cols=64, vocab=100, type=1, loss=P, lse=P, ws=P, size=1 << 20) | change
    assert _lib().ones_linear_ce(a["h"], a["ldh"], a["w"], a["ldw"], a["t"], a["rows"], a["cols"], a["vocab"], a["type"], a["loss"],
                                 a["lse"], a["ws"], a["size"], None) == want


@pytest.mark.parametrize("change, want", [
    ({"rows": -1}, PARAM), ({"type": 0}, PARAM), ({"wtype": 2}, PARAM), ({"piece": 100}, PARAM), ({"piece": -256}, PARAM),
    ({"lddh": 1}, PARAM), ({"lddw": 1}, PARAM), ({"dw": None}, NULL), ({"g": None}, NULL), ({"dh": None}, NULL), ({"w": P + 8}, ALIGN),
    ({"ldw": 68}, ALIGN), ({"dh": P + 1}, ALIGN), ({"size": 1024}, SPACE)])
def test_linear_ce_backward_refuses(change, want):
    a = dict(g=P, h=P, ldh=64, w=P, ldw=64, t=P, lse=P, rows=4, cols=64, vocab=100, type=1, wtype=1, piece=0, dh=P, lddh=64, dw=P,
             lddw=64, ws=P, size=1 << 24) | change
    assert _lib().ones_linear_ce_backward(a["g"], a["h"], a["ldh"], a["w"], a["ldw"], a["t"], a["lse"], a["rows"], a["cols"], a["vocab"],
                                          a["type"], a["wtype"], a["piece"], a["dh"], a["lddh"], a["dw"], a["lddw"], a["ws"],
                                          a["size"], None) == want


@pytest.mark.parametrize("change, want", [
    ({"count": 0}, PARAM), ({"m": 0}, PARAM), ({"n": 1 << 21}, PARAM), ({"type": 5}, PARAM), ({"steps": 0}, PARAM), ({"eps": -1.0}, PARAM),
    ({"a": float("inf")}, PARAM), ({"ldg": 199}, PARAM), ({"stride": -1, "count": 2}, PARAM), ({"g": None}, NULL), ({"out": None}, NULL),
    ({"g": P + 2}, ALIGN), ({"out": P + 1}, ALIGN), ({"ws": P + 16}, ALIGN), ({"size": 1024}, SPACE)])
def test_orthogonalize_refuses(change, want):
    a = dict(g=P, ldg=200, stride=200 * 200, count=1, m=200, n=200, type=0, steps=5, a=3.4445, b=-4.775, c=2.0315, eps=1e-7, out=P, ws=P,
             size=1 << 24) | change
    assert _lib().ones_orthogonalize(a["g"], a["ldg"], a["stride"], a["count"], a["m"], a["n"], a["type"], a["steps"], a["a"], a["b"],
                                     a["c"], a["eps"], a["out"], a["ws"], a["size"], None) == want


def test_nothing_to_do_needs_no_device():
    L = _lib()
    assert L.ones_layer_norm(None, 8, None, None, 0, 8, 1e-5, 0, 0, None, 8, None, None, None) == 0
    assert L.ones_linear_ce(None, 8, None, 8, None, 0, 8, 8, 1, None, None, None, 0, None) == 0


def test_binding_refuses_cpu_tensors():
    torch = pytest.importorskip("torch")
    from paper_2108_03645_b200 import train
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        train.layer_norm(x)
    with pytest.raises(ValueError):
        train.linear_cross_entropy(x.bfloat16(), x.bfloat16(), torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        train.orthogonalize(x)


def test_profile_fit():
    from paper_2108_03645_b200 import profile_job as pj
    b = np.array([8, 16, 32, 64])
    a, c = pj.fit(b, 0.003 + 2e-4 * b)
    assert abs(a - 0.003) < 1e-12 and abs(c - 2e-4) < 1e-14
    a, c = pj.fit(b, 2e-4 * b - 1e-5)  # would need a < 0
    assert a == 0.0 and c > 0
    a, c = pj.fit(b, 0.01 - 1e-5 * b)  # would need c < 0
    assert c == 0.0 and a > 0
    assert pj.fit([8], [0.004]) == (0.0, 0.0005)
    for bad in ([0.0, 1, 1, 1], [np.nan, 1, 1, 1], [1, 1]):
        with pytest.raises(ValueError):
            pj.fit(b, bad)
    row = pj.job_row(8, 4, 64, 0.003, 2e-4, 0.01)
    assert row.dtype.itemsize == 48 and row["kmax"][0] == 4


@pytest.mark.parametrize("change, want", [
    ({"rows": -1}, PARAM), ({"cols": -1}, PARAM), ({"type": 0}, PARAM), ({"lds": 63}, PARAM), ({"ldd": 63}, PARAM), ({"src": None}, NULL),
    ({"dst": None}, NULL), ({"src": P + 1}, ALIGN), ({"dst": P + 8}, ALIGN), ({"ldd": 68}, ALIGN)])
def test_align_rows_refuses(change, want):
    a = {"src": P, "lds": 64, "rows": 4, "cols": 64, "type": 1, "dst": P, "ldd": 64, "stream": None}
    a.update(change)
    assert _lib().ones_align_rows(*a.values()) == want
