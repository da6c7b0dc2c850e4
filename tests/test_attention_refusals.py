"""The attention layer's operators without a device: symbols, sizes of workspaces, arguments that are refused before any launch."""
import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000  # a pointer that no refused call may follow
NULL, PARAM, ALIGN, SPACE = -1, -3, -4, -5


def _lib():
    from paper_2108_03645_b200 import train
    return train.lib()


def test_library_exports_and_binding_covers_every_declared_symbol():
    from paper_2108_03645_b200 import build, train
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ones_attention.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ones_[a-z_0-9]+)\s*\(", text)))
    assert len(names) == 10
    lib = C.CDLL(build.build())
    for n in names:
        assert hasattr(lib, n), n
    assert sorted(train._ATTENTION_SIGNATURES) == names


def test_workspace_sizes():
    L = _lib()
    assert L.ones_qk_norm_workspace_bytes(0) == 0 and L.ones_qk_norm_workspace_bytes(257) == 0 and L.ones_qk_norm_workspace_bytes(1) >= 8
    for bad in ((-1, 1, 2, 1), (8, -1, 2, 1), (8, 1, 0, 1), (8, 1, 3, 2), (8, 1, 129, 1), (8, 1, 2, 0), (1 << 30, 1, 2, 1), (8, (1 << 22) + 1, 2, 1),
                (8, 1, 2048, 1024)):
        assert L.ones_attention_workspace_bytes(*bad) == 0 and L.ones_attention_backward_workspace_bytes(*bad, 64) == 0
    assert L.ones_attention_backward_workspace_bytes(8, 1, 2, 1, 129) == 0
    # far below the scores; past 32 bits
    assert 0 < L.ones_attention_workspace_bytes(65536, 8, 32, 8) < 1 << 20
    assert L.ones_attention_backward_workspace_bytes((1 << 30) - 1, 1, 32, 8, 128) > 1 << 36
    assert L.ones_gradient_norm_workspace_bytes(-1) == 0 and L.ones_gradient_norm_workspace_bytes((1 << 20) + 1) == 0
    assert L.ones_gradient_norm_workspace_bytes(0) > 0


def _heads(p=P, token=512, head=64, heads=8):
    from paper_2108_03645_b200 import train
    return train.Heads(p, token, head, heads)


def _change(args, change):
    """Arguments with some replaced; "q.head" replaces a field."""
    args = dict(args)
    for key, value in change.items():
        if "." in key:
            name, field = key.split(".")
            h = args[name]
            args[name] = type(h)(h.data, h.token, h.head, h.heads)
            setattr(args[name], field, value)
        else:
            args[key] = value
    return [C.byref(v) if isinstance(v, C.Structure) else v for v in args.values()]


QK = [({"tokens": -1}, PARAM), ({"dim": 0}, PARAM), ({"dim": 257}, PARAM), ({"rotary": 63}, PARAM), ({"rotary": 66}, PARAM), ({"rotary": -2}, PARAM),
      ({"eps": -1.0}, PARAM), ({"eps": float("nan")}, PARAM), ({"type": 3}, PARAM), ({"type": 1, "wtype": 2}, PARAM), ({"q.head": 63}, PARAM),
      ({"k.token": -1}, PARAM), ({"q.heads": 7}, PARAM), ({"q.heads": 1025, "qo.heads": 1025}, PARAM), ({"q": None}, NULL), ({"ko": None}, NULL),
      ({"q.data": None}, NULL), ({"qo.data": None}, NULL), ({"pos": None}, NULL), ({"freq": None}, NULL), ({"q.data": P + 2}, ALIGN),
      ({"k.data": P + 1}, ALIGN), ({"pos": P + 4}, ALIGN), ({"freq": P + 4}, ALIGN), ({"qw": P + 2}, ALIGN)]


@pytest.mark.parametrize("change, want", QK)
def test_qk_norm_refuses(change, want):
    a = dict(q=_heads(), k=_heads(heads=2), pos=P, freq=P, qw=P, kw=P, tokens=4, dim=64, rotary=64, inter=0, eps=1e-6, type=0, wtype=0, qo=_heads(),
             ko=_heads(heads=2), stream=None)
    assert _lib().ones_qk_norm(*_change(a, change)) == want


@pytest.mark.parametrize("change, want", QK + [({"dq": None}, NULL), ({"dk.data": None}, NULL), ({"dk.heads": 3}, PARAM), ({"dq.head": 1}, PARAM),
                                               ({"ws": None}, NULL), ({"ws": P + 16}, ALIGN), ({"size": 64}, SPACE), ({"dkw": P + 1}, ALIGN)])
def test_qk_norm_backward_refuses(change, want):
    a = dict(dq=_heads(), dk=_heads(heads=2), q=_heads(), k=_heads(heads=2), pos=P, freq=P, qw=P, kw=P, tokens=4, dim=64, rotary=64, inter=0, eps=1e-6,
             type=0, wtype=0, qo=_heads(), ko=_heads(heads=2), dqw=P, dkw=P, ws=P, size=1 << 24, stream=None)
    assert _lib().ones_qk_norm_backward(*_change(a, change)) == want


ATTEND = [({"tokens": -1}, PARAM), ({"tokens": 1 << 30}, PARAM), ({"sequences": -1}, PARAM), ({"sequences": (1 << 22) + 1}, PARAM), ({"dim": 0}, PARAM),
          ({"dim": 129}, PARAM), ({"scale": 0.0}, PARAM), ({"scale": -1.0}, PARAM), ({"scale": float("nan")}, PARAM), ({"scale": float("inf")}, PARAM),
          ({"type": 0}, PARAM), ({"type": 3}, PARAM), ({"offsets": None, "sequences": 3}, PARAM), ({"offsets": None, "sequences": 0}, PARAM),
          ({"k.heads": 3}, PARAM), ({"k.heads": 0}, PARAM), ({"v.heads": 4}, PARAM), ({"q.heads": 12}, PARAM), ({"q.head": 56}, PARAM),
          ({"v.token": 0}, PARAM), ({"q": None}, NULL), ({"out": None}, NULL), ({"v.data": None}, NULL), ({"lse": None}, NULL), ({"ws": None}, NULL),
          ({"q.data": P + 8}, ALIGN), ({"k.data": P + 2}, ALIGN), ({"k.token": 516}, ALIGN), ({"q.head": 68}, ALIGN), ({"out.data": P + 1}, ALIGN),
          ({"lse": P + 2}, ALIGN), ({"offsets": P + 4}, ALIGN), ({"ws": P + 64}, ALIGN), ({"size": 256}, SPACE)]


@pytest.mark.parametrize("change, want", ATTEND)
def test_attention_refuses(change, want):
    a = dict(q=_heads(), k=_heads(heads=2), v=_heads(heads=2), offsets=P, tokens=200, sequences=2, dim=64, scale=0.125, type=1, out=_heads(), lse=P, ws=P,
             size=1 << 24, stream=None)
    assert _lib().ones_attention(*_change(a, change)) == want


@pytest.mark.parametrize("change, want", ATTEND + [({"dout": None}, NULL), ({"dq.data": None}, NULL), ({"dout.data": P + 8}, ALIGN),
                                                   ({"dk.heads": 8}, PARAM), ({"dv.data": P + 1}, ALIGN), ({"dq.token": 0}, PARAM)])
def test_attention_backward_refuses(change, want):
    a = dict(dout=_heads(), q=_heads(), k=_heads(heads=2), v=_heads(heads=2), out=_heads(), lse=P, offsets=P, tokens=200, sequences=2, dim=64, scale=0.125,
             type=1, dq=_heads(), dk=_heads(heads=2), dv=_heads(heads=2), ws=P, size=1 << 24, stream=None)
    assert _lib().ones_attention_backward(*_change(a, change)) == want


def test_attention_refuses_more_work_than_is_counted():
    """Tiles of tokens times heads of the keys are counted in 31 bits."""
    L = _lib()
    many, few = _heads(token=1024 * 64, heads=1024), _heads(token=1024 * 64, heads=512)
    n = (1 << 30) - 1
    for h in (many, few):
        a = [C.byref(h)] * 3
        assert L.ones_attention(*a, P, n, 1, 64, 0.125, 1, C.byref(h), P, P, 1 << 62, None) == PARAM
        assert L.ones_attention_backward(*a, C.byref(h), C.byref(h), P, P, n, 1, 64, 0.125, 1, *a, P, 1 << 62, None) == PARAM


def _list(values, kind):
    return (kind * max(len(values), 1))(*values)


@pytest.mark.parametrize("change, want", [
    ({"count": -1}, PARAM), ({"count": (1 << 20) + 1}, PARAM), ({"size": [5, -1]}, PARAM), ({"type": [0, 3]}, PARAM), ({"size": [1 << 43, 1]}, PARAM),
    ({"size": [1 << 42, 1 << 42]}, PARAM), ({"limit": -1.0}, PARAM), ({"limit": float("nan")}, PARAM), ({"limit": float("inf")}, PARAM),
    ({"eps": -1e-9}, PARAM), ({"eps": float("nan")}, PARAM), ({"g": [P, None]}, NULL), ({"out": [None, P]}, NULL), ({"g": None}, NULL), ({"out": None}, NULL),
    ({"norm": None}, NULL), ({"ws": None}, NULL), ({"g": [P + 2, P]}, ALIGN), ({"out": [P, P + 1]}, ALIGN), ({"norm": P + 1}, ALIGN), ({"ws": P + 8}, ALIGN),
    ({"bytes": 16}, SPACE)])
def test_clip_gradients_refuses(change, want):
    a = dict(g=[P, P], out=[P, P], size=[5, 7], type=[0, 1], count=2, limit=1.0, eps=1e-6, norm=P, ws=P, bytes=1 << 20) | change
    g, out = (None if a[x] is None else _list(a[x], C.c_void_p) for x in ("g", "out"))
    assert _lib().ones_clip_gradients(g, out, _list(a["size"], C.c_int64), _list(a["type"], C.c_int32), a["count"], a["limit"], a["eps"], a["norm"],
                                      a["ws"], a["bytes"], None) == want
    if not {"limit", "eps", "out"} & set(change):
        assert _lib().ones_gradient_norm(g, _list(a["size"], C.c_int64), _list(a["type"], C.c_int32), a["count"], a["norm"], a["ws"], a["bytes"],
                                         None) == want


def test_nothing_to_do_needs_no_device():
    L = _lib()
    none = _heads(p=None)
    kv = _heads(p=None, heads=2)
    assert L.ones_qk_norm(C.byref(none), C.byref(kv), None, None, None, None, 0, 64, 64, 0, 1e-6, 1, 0, C.byref(none), C.byref(kv), None) == 0
    assert L.ones_attention(C.byref(none), C.byref(kv), C.byref(kv), None, 0, 0, 64, 0.125, 1, C.byref(none), None, None, 0, None) == 0


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    from paper_2108_03645_b200 import train
    q, k = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, 1, 64, dtype=torch.bfloat16)
    pos, freq = torch.arange(4), train.rotary_frequencies(64, device="cpu")
    lse = torch.zeros(4, 2)
    for f in (lambda a: train.qk_norm(a, k, pos, freq), lambda a: train.attention(a, k, k), lambda a: train.gradient_norm([a]),
              lambda a: train.clip_gradients([a], 1.0), lambda a: train.qk_norm_backward(a, k, q, k, pos, freq),
              lambda a: train.attention_backward(q, a, k, k, q, lse)):
        with pytest.raises(ValueError, match="CUDA"):
            f(q)
        with pytest.raises(ValueError, match="no_grad"):
            f(q.clone().requires_grad_())
    with pytest.raises(ValueError, match="even"):
        train.rotary_frequencies(5, device="cpu")
    assert torch.equal(train.rotary_frequencies(4, 100.0, device="cpu"), torch.tensor([1.0, 0.1], dtype=torch.float64))
    assert train.rotary_frequencies(0, device="cpu").numel() == 0
