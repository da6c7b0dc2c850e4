"""The training-step operators against their definitions in 64 bits, on the GPU.

Bounds are derived from the arithmetic: u = the unit roundoff of the output's type (2^-24 for float32, 2^-8 for bfloat16,
2^-11 for float16), one rounding of the result, and what 32-bit sums and the 16-bit gradients of the logits can add, element
by element.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}   # round to nearest: half the spacing above 1
TINY = {F32: 0.0, BF16: 0.0, F16: 2.0 ** -25}             # half the spacing of float16's smallest numbers


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    yield
    from paper_2108_03645_b200 import train
    train.check()


def randn(*size, seed=0):
    return torch.randn(*size, generator=torch.Generator(device="cuda").manual_seed(seed + 1), device="cuda")


def close(got, want, bound):
    bad = (got.double() - want).abs() > bound
    assert not bool(bad.any()), float(((got.double() - want).abs() / bound.clamp(min=1e-300)).max())


def wide(t, pad):
    """t as a slice of a wider buffer whose other values are NaN."""
    w = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    w[:, :t.shape[1]] = t
    return w[:, :t.shape[1]]


# ---------------------------------------------------------------- layer norm

def norm_reference(x, w, b, eps, dy=None):
    x = x.double()
    w = torch.ones(x.shape[1], device="cuda").double() if w is None else w.double()
    b = torch.zeros(x.shape[1], device="cuda").double() if b is None else b.double()
    mean = x.mean(1)
    rstd = 1 / ((x - mean[:, None]).square().mean(1) + eps).sqrt()
    xh = (x - mean[:, None]) * rstd[:, None]
    out = [xh * w + b, mean, rstd, xh]
    if dy is not None:
        dy = dy.double()
        g = dy * w
        out += [rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)), (dy * xh).sum(0), dy.sum(0)]
    return out


def check_norm(x, w, b, dy, eps=1e-5):
    from paper_2108_03645_b200 import train
    y, mean, rstd = train.layer_norm(x, w, b, eps)
    dx, dw, db = train.layer_norm_backward(dy, x, mean, rstd, w)
    ry, rm, rr, xh, rdx, rdw, rdb = norm_reference(x, w, b, eps, dy)
    n, d = x.shape
    u = U[x.dtype]
    one = 2.0 ** -24
    # A sum of d values in 32 bits is a tree of chains of at most 64 additions: 2^6 * 2^-24 of the sum of magnitudes
    s = 2.0 ** -18
    big = x.double().abs().amax(1)
    assert bool(((mean.double() - rm).abs() <= s * big + one * rm.abs()).all())
    e_xh = (s * (big * rr) + 2 * s)[:, None] * (1 + xh.abs())          # of (x - mean) * rstd: mean, variance, roundings
    assert bool(((rstd.double() - rr).abs() <= rr * (2 * s + s * (big * rr) ** 2 * 0 + (s * big * rr) ** 2 + 4 * one)).all())
    wd = torch.ones(d, device="cuda").double() if w is None else w.double()
    close(y, ry, u * ry.abs() + e_xh * wd.abs() + 4 * one * (ry.abs() + 1) + TINY[x.dtype])
    g = dy.double() * wd
    ga = g.abs().mean(1, keepdim=True) + g.abs()
    gx = (g * xh).abs().mean(1, keepdim=True) + (g.abs() * e_xh).mean(1, keepdim=True)
    e_dx = rr[:, None] * (8 * s * (ga + (xh.abs() + 1) * gx) + e_xh * 2 * gx + (xh.abs() + 1) * (g.abs() * e_xh).mean(1, keepdim=True))
    close(dx, rdx, u * rdx.abs() + e_dx + TINY[x.dtype])
    uw = U[dw.dtype]
    a, p = (dy.double() * xh).abs().sum(0), dy.double().abs().sum(0)
    chain = (n + 64) * one  # the sum over rows, whatever its order
    close(dw, rdw, uw * rdw.abs() + (dy.double().abs() * e_xh).sum(0) + chain * a + TINY[dw.dtype] + 1e-30)
    close(db, rdb, uw * rdb.abs() + chain * p + TINY[dw.dtype] + 1e-30)
    return y, mean, rstd, dx, dw, db


SIZES = [(1, 1), (1, 8), (3, 7), (2, 64), (17, 255), (5, 256), (33, 264), (9, 512), (300, 520), (64, 1000), (40, 1023), (700, 1024),
         (7, 2048), (19, 2056), (5, 4095), (150, 4096), (3, 4100), (5, 8192), (4, 8200), (3, 16384), (2, 16390), (1, 65536), (2000, 48)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,d", SIZES)
def test_layer_norm(n, d, dtype):
    x = (randn(n, d, seed=n * d) * 2 + 1).to(dtype)
    dy = randn(n, d, seed=7).to(dtype)
    w, b = 1 + 0.3 * randn(d, seed=3), randn(d, seed=4)
    wt = F32 if (n + d) % 2 else dtype
    check_norm(x, w.to(wt), b.to(wt), dy)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("pad", [1, 3, 8, 24])
def test_layer_norm_strides(dtype, pad):
    x, dy = wide((randn(61, 136) + 2).to(dtype), pad), wide(randn(61, 136, seed=2).to(dtype), pad + 1)
    w, b = randn(136, seed=3).to(dtype), randn(136, seed=4).to(dtype)
    check_norm(x, w, b, dy)
    # a column slice: rows that start on no 16-byte boundary
    big = (randn(20, 200, seed=9)).to(dtype)
    check_norm(big[:, 1:101], w[:100].contiguous(), b[:100].contiguous(), big[:, 3:103])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layer_norm_parameters(dtype):
    from paper_2108_03645_b200 import train
    x, dy = randn(50, 96).to(dtype), randn(50, 96, seed=2).to(dtype)
    w, b = randn(96, seed=3), randn(96, seed=4)
    check_norm(x, None, None, dy)
    check_norm(x, w, None, dy)
    check_norm(x, None, b, dy)
    y, mean, rstd = train.layer_norm(x, w)
    dx, dw, db = train.layer_norm_backward(dy, x, mean, rstd, w, parameters=False)
    assert dw is None and db is None
    assert torch.equal(dx, train.layer_norm_backward(dy, x, mean, rstd, w)[0])


def test_layer_norm_large_offset_and_constant_rows():
    # a mean of 1000 standard deviations, and rows without any spread (variance 0: eps decides)
    x = torch.cat([randn(20, 640) + 1000.0, torch.full((3, 640), 5.0, device="cuda")])
    check_norm(x, randn(640, seed=3), randn(640, seed=4), randn(23, 640, seed=5))


def test_layer_norm_nan_and_infinity_stay_in_their_rows():
    from paper_2108_03645_b200 import train
    x = randn(9, 512)
    x[2, 5], x[7, 0] = float("nan"), float("inf")
    y, mean, rstd = train.layer_norm(x)
    ok = torch.tensor([i not in (2, 7) for i in range(9)], device="cuda")
    assert bool(torch.isfinite(y[ok]).all()) and bool(torch.isnan(y[~ok]).any(1).all())
    assert torch.equal(y[ok], train.layer_norm(x[ok])[0])


def test_layer_norm_empty_and_leading_dimensions():
    from paper_2108_03645_b200 import train
    x = torch.empty(0, 64, device="cuda")
    w = randn(64)
    y, mean, rstd = train.layer_norm(x, w, w)
    assert y.shape == (0, 64) and mean.shape == (0,)
    dx, dw, db = train.layer_norm_backward(x, x, mean, rstd, w)
    assert dx.shape == (0, 64) and not bool(dw.any()) and not bool(db.any())
    x = randn(3, 4, 64)
    y, mean, rstd = train.layer_norm(x, w, w)
    assert y.shape == x.shape and mean.shape == (3, 4)
    assert torch.equal(y.view(12, 64), train.layer_norm(x.view(12, 64), w, w)[0])
    # an expanded gradient, a transposed input, one vector
    dy = torch.ones(1, 1, 1, device="cuda").expand(3, 4, 64)
    dx, dw, db = train.layer_norm_backward(dy, x, mean, rstd, w)
    assert torch.allclose(db, torch.full_like(db, 12.0))
    xt = randn(64, 10).t()
    assert torch.equal(train.layer_norm(xt, w)[0], train.layer_norm(xt.contiguous(), w)[0])
    assert torch.equal(train.layer_norm(x[0, 0], w)[0], train.layer_norm(x[0], w)[0][0])


def test_layer_norm_rows_past_32_bits():
    # two rows 2^31 + 8 values apart
    from paper_2108_03645_b200 import train
    far = (1 << 31) + 8
    flat = torch.empty(far + 64, dtype=BF16, device="cuda")
    x = flat.as_strided((2, 64), (far, 1))
    x.copy_(randn(2, 64).bfloat16())
    y, mean, rstd = train.layer_norm(x)
    assert torch.equal(y, train.layer_norm(x.contiguous())[0])
    assert torch.equal(train.layer_norm_backward(x, x, mean, rstd)[0], train.layer_norm_backward(y * 0 + x, x.contiguous(), mean, rstd)[0])


@pytest.mark.parametrize("dtype,cols", [(F32, 96), (F32, 97), (BF16, 4096), (F16, 20000)])
def test_layer_norm_touches_nothing_else(dtype, cols):
    """Outputs and workspace between guard values, through the C ABI."""
    from paper_2108_03645_b200 import train
    L = train.lib()
    rows, size = 37, 4 if dtype == F32 else 2
    kind = {F32: 0, BF16: 1, F16: 2}[dtype]
    x, dy, w = randn(rows, cols).to(dtype), randn(rows, cols, seed=1).to(dtype), randn(cols, seed=2)
    nbytes = L.ones_layer_norm_workspace_bytes(rows, cols)

    def guarded(n):
        t = torch.full((n + 1024,), 0x5A, dtype=torch.uint8, device="cuda")
        return t, t.data_ptr() + 512
    y, yp = guarded(rows * cols * size)
    st, sp = guarded(rows * 8)
    dx, dxp = guarded(rows * cols * size)
    dwb, dwp = guarded(cols * 8)
    ws, wsp = guarded(nbytes)
    s = torch.cuda.current_stream().cuda_stream
    assert L.ones_layer_norm(x.data_ptr(), cols, w.data_ptr(), w.data_ptr(), rows, cols, 1e-5, kind, 0, yp, cols, sp, sp + 4 * rows, s) == 0
    assert L.ones_layer_norm_backward(dy.data_ptr(), cols, x.data_ptr(), cols, sp, sp + 4 * rows, w.data_ptr(), rows, cols, kind, 0, dxp,
                                      cols, dwp, dwp + 4 * cols, wsp, nbytes, s) == 0
    torch.cuda.synchronize()
    for t in (y, st, dx, dwb, ws):
        assert bool((t[:512] == 0x5A).all()) and bool((t[-512:] == 0x5A).all())


# ---------------------------------------------------------------- cross entropy

def ce_reference(h, w, t, dloss=None):
    h, w = h.double(), w.double()
    v = w.shape[0]
    live = (t >= 0) & (t < v)
    h = torch.where(live[:, None] | torch.isfinite(h).all(1, keepdim=True), h, torch.zeros_like(h))
    l = h @ w.t()
    lse = torch.logsumexp(l, 1)
    at = torch.where(live, t, torch.zeros_like(t))[:, None]
    loss = torch.where(live, lse - l.gather(1, at)[:, 0], torch.zeros_like(lse))
    out = {"lse": lse, "loss": loss, "l": l, "live": live, "mass": (h.abs() @ w.abs().t()).amax(1)}
    if dloss is not None:
        p = torch.softmax(l, 1).scatter_add(1, at, -torch.ones_like(at, dtype=torch.float64))
        p = p * torch.where(live, dloss.double(), torch.zeros_like(lse))[:, None]
        # rows that take part only: 0 * NaN is no contribution
        p[~live] = 0
        out |= {"p": p, "dh": p @ w, "dw": p.t() @ torch.where(live[:, None], h, torch.zeros_like(h)), "h": torch.where(live[:, None], h, torch.zeros_like(h)), "w": w}
    return out


def check_ce(h, w, t, dloss, piece=0, weight_gradient=None):
    from paper_2108_03645_b200 import train
    loss, lse = train.linear_cross_entropy(h, w, t)
    dh, dw = train.linear_cross_entropy_backward(dloss, h, w, t, lse, piece=piece, weight_gradient=weight_gradient)
    r = ce_reference(h, w, t, dloss)
    k = h.shape[1]
    # Products of 16-bit values are exact in 32 bits; each of about k / 8 partial sums loses at most one unit of 2^-23 of
    # the largest partial sum, which is at most the sum of magnitudes
    logit = (k / 8 + 4) * 2.0 ** -23 * r["mass"]
    fine = torch.isfinite(h).all(1)
    tol = logit + 2.0 ** -20 * (1 + r["lse"].abs())   # exponents, logarithm and their sums in 32 bits
    assert bool(((lse.double() - r["lse"]).abs() <= tol)[fine].all())
    assert bool(((loss.double() - r["loss"]).abs() <= 2 * tol)[fine].all())
    assert bool((loss[~r["live"]] == 0).all()) and bool((dh[~r["live"]] == 0).all())
    # dlogits: one rounding to 16 bits, and the relative error of exp(l - lse)
    g = torch.where(r["live"], dloss.double().abs(), torch.zeros_like(r["lse"]))
    soft = torch.softmax(r["l"], 1) * g[:, None]
    top = float(g.max()) if g.numel() else 0.0
    e = U[h.dtype] * r["p"].abs() + soft * (torch.expm1(2 * tol) + 2.0 ** -20)[:, None] + 2.0 ** -22 * g[:, None] * (r["p"] < 0) + TINY[h.dtype] * top
    e[~r["live"]] = 0
    n, v = r["p"].shape
    close(dh, r["dh"], U[dh.dtype] * r["dh"].abs() + 1.01 * (e @ r["w"].abs()) + (v / 8 + 8) * 2.0 ** -23 * (r["p"].abs() @ r["w"].abs()) + TINY[dh.dtype] + 1e-38)
    close(dw, r["dw"], U[dw.dtype] * r["dw"].abs() + 1.01 * (e.t() @ r["h"].abs()) + (n / 8 + 8) * 2.0 ** -23 * (r["p"].abs().t() @ r["h"].abs()) + TINY[dw.dtype] + 1e-38)
    return loss, lse, dh, dw


def ce_inputs(n, d, v, dtype, ignored, seed=0):
    w = (randn(v, d, seed=seed) * (2 / math.sqrt(d))).to(dtype)
    t = torch.randint(0, v, (n,), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    h = (randn(n, d, seed=seed + 5) + w[t].float() * 2).to(dtype)
    drop = torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(seed + 1), device="cuda") < ignored
    t[drop] = -100
    return h, w, t, (0.2 + randn(n, seed=seed + 2).abs())


CE = [(1, 1, 1, 0.0), (1, 8, 2, 0.0), (1, 64, 1000, 0.0), (2, 100, 129, 0.5), (5, 513, 4001, 0.0), (63, 64, 255, 0.2), (64, 96, 256, 0.2),
      (65, 72, 257, 0.2), (127, 33, 1024, 0.1), (129, 256, 300, 0.9), (255, 128, 5000, 0.1), (257, 130, 777, 0.3), (600, 1024, 2100, 0.1),
      (1030, 40, 3000, 0.0), (300, 2050, 500, 0.1), (2049, 8, 40, 0.4)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,d,v,ignored", CE)
def test_linear_cross_entropy(n, d, v, ignored, dtype):
    check_ce(*ce_inputs(n, d, v, dtype, ignored, seed=n + d + v))


@pytest.mark.parametrize("piece", [256, 512, 1024, 4096])
def test_linear_cross_entropy_pieces(piece):
    h, w, t, g = ce_inputs(200, 136, 3001, BF16, 0.2)
    check_ce(h, w, t, g, piece=piece)


def test_linear_cross_entropy_last_piece_of_one_entry():
    # few rows and a long piece: the product over the piece is cut into parts, and the last piece has less than they need
    h, w, t, g = ce_inputs(100, 64, 16385, F16, 0.2)
    check_ce(h, w, t, g, piece=16384)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_linear_cross_entropy_weight_gradient_in_32_bits(dtype):
    h, w, t, g = ce_inputs(100, 130, 600, dtype, 0.2)
    assert check_ce(h, w, t, g, weight_gradient=F32)[3].dtype == F32


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("scale", [1e-6, 1.0, 65536.0])
def test_linear_cross_entropy_loss_scales(dtype, scale):
    # the 16-bit gradients of the logits are scaled into range whatever the loss's scale (float16 outputs may overflow)
    h, w, t, g = ce_inputs(90, 64, 500, dtype, 0.2)
    if dtype == F16 and scale > 1:
        scale = 256.0
    check_ce(h, w, t, g * scale)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("pad", [1, 8, 13])
def test_linear_cross_entropy_strides(dtype, pad):
    h, w, t, g = ce_inputs(70, 72, 300, dtype, 0.2)
    check_ce(wide(h, pad), wide(w, pad), t, g)
    check_ce(wide(h, pad)[:, 1:60], wide(w, pad)[:, 1:60], t, g)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,d,v,piece", [(1, 64, 500, 0), (2, 1000, 3000, 512), (5, 1856, 4086, 0), (17, 72, 9000, 0), (64, 256, 2000, 256)])
def test_linear_cross_entropy_few_rows(n, d, v, piece, dtype):
    # no error is averaged over many products here: both terms of the gradients of the logits are kept, and only the
    # results' own roundings remain, 2^-8 (2^-11) / sqrt(3) of the norm in the mean at most
    from paper_2108_03645_b200 import train
    h, w, t, g = ce_inputs(n, d, v, dtype, 0.0, seed=n)
    loss, lse, dh, dw = check_ce(h, w, t, g, piece=piece)
    r = ce_reference(h, w, t, g)
    for got, want in ((dh, r["dh"]), (dw, r["dw"])):
        assert float((got.double() - want).norm() / want.norm()) <= 0.6 * U[dtype]


def test_linear_cross_entropy_no_row_takes_part():
    from paper_2108_03645_b200 import train
    h, w, t, g = ce_inputs(150, 64, 300, BF16, 0.0)
    t[:] = -1
    t[3], t[4], t[5] = 300, 1 << 40, -(1 << 50)
    loss, lse = train.linear_cross_entropy(h, w, t)
    dh, dw = train.linear_cross_entropy_backward(g, h, w, t, lse)
    assert not bool(loss.any()) and not bool(dh.any()) and not bool(dw.any()) and bool(torch.isfinite(lse).all())


def test_linear_cross_entropy_rows_that_take_no_part_do_not_matter():
    from paper_2108_03645_b200 import train
    h, w, t, g = ce_inputs(150, 64, 300, BF16, 0.3)
    h2, g2 = h.clone(), g.clone()
    h2[t < 0], g2[t < 0] = float("nan"), float("inf")
    a, b = (train.linear_cross_entropy(q, w, t) for q in (h, h2))
    assert torch.equal(a[0], b[0])
    for p, q in zip(train.linear_cross_entropy_backward(g, h, w, t, a[1]), train.linear_cross_entropy_backward(g2, h2, w, t, b[1])):
        assert torch.equal(p, q)


def test_linear_cross_entropy_extreme_logits():
    # a row that is certain of its target, one certain of another entry, logits of some hundreds, and one infinite entry
    from paper_2108_03645_b200 import train
    d, v = 64, 700
    w = torch.zeros(v, d, device="cuda")
    w[5, 0], w[9, 1] = 200.0, 200.0
    h = torch.zeros(4, d, device="cuda")
    h[0, 0] = h[1, 1] = 2.0
    h[2, 0] = -2.0
    t = torch.tensor([5, 5, 9, 9], device="cuda")
    h, w = h.bfloat16(), w.bfloat16()
    loss, lse, dh, dw = check_ce(h, w, t, torch.ones(4, device="cuda"))
    assert float(loss[0]) == 0.0 and float(loss[1]) == 400.0
    w[7, 3] = float("-inf")  # an entry that never comes: exp(-inf) = 0
    h[:, 3] = 1.0
    loss, lse = train.linear_cross_entropy(h, w, t)
    assert bool(torch.isfinite(loss).all())
    ref = torch.logsumexp(torch.cat([(h.double() @ w.double().t())[:, :7], (h.double() @ w.double().t())[:, 8:]], 1), 1)
    assert torch.allclose(lse.double(), ref, rtol=1e-5)


def test_linear_cross_entropy_empty_and_leading_dimensions():
    from paper_2108_03645_b200 import train
    h, w, t, g = ce_inputs(12, 64, 300, BF16, 0.0)
    loss, lse = train.linear_cross_entropy(h.view(3, 4, 64), w, t.view(3, 4))
    assert loss.shape == (3, 4) and torch.equal(loss.view(-1), train.linear_cross_entropy(h, w, t)[0])
    dh, dw = train.linear_cross_entropy_backward(g.view(3, 4), h.view(3, 4, 64), w, t.view(3, 4), lse)
    assert dh.shape == (3, 4, 64)
    loss, lse = train.linear_cross_entropy(h[:0], w, t[:0])
    dh, dw = train.linear_cross_entropy_backward(g[:0], h[:0], w, t[:0], lse)
    assert loss.shape == (0,) and dh.shape == (0, 64) and not bool(dw.any())


def test_linear_cross_entropy_weight_past_32_bits():
    # 2^31 + values in the weight: the last rows lie past a 32-bit offset
    from paper_2108_03645_b200 import train
    v, d = 140000, 16384
    w = torch.zeros(v, d, dtype=BF16, device="cuda")
    w[-300:] = (randn(300, d) * 0.01).bfloat16()
    h = randn(3, d, seed=2).bfloat16()
    t = torch.tensor([v - 1, v - 300, 0], device="cuda")
    loss, lse = train.linear_cross_entropy(h, w, t)
    l = torch.zeros(3, v, dtype=torch.float64, device="cuda")
    l[:, -300:] = h.double() @ w[-300:].double().t()
    ref = torch.logsumexp(l, 1)
    assert torch.allclose(lse.double(), ref, rtol=1e-5)
    assert torch.allclose(loss.double(), ref - l.gather(1, t[:, None])[:, 0], rtol=1e-4, atol=1e-4)


def test_linear_cross_entropy_gradient_against_differences():
    from paper_2108_03645_b200 import train
    h, w, t, g = ce_inputs(40, 48, 200, BF16, 0.2)
    _, lse = train.linear_cross_entropy(h, w, t)
    dh, dw = train.linear_cross_entropy_backward(g, h, w, t, lse, weight_gradient=F32)

    def total(hh, ww):
        l = hh @ ww.t()
        live = t >= 0
        at = torch.where(live, t, torch.zeros_like(t))[:, None]
        return float((torch.where(live, torch.logsumexp(l, 1) - l.gather(1, at)[:, 0], 0.0) * g.double()).sum())
    hd, wd = h.double(), w.double()
    for seed in range(4):
        a, b = randn(*h.shape, seed=seed + 50).double(), randn(*w.shape, seed=seed + 60).double()
        e = 1e-4
        num = (total(hd + e * a, wd) - total(hd - e * a, wd)) / (2 * e)
        # the roundings of dh and of dlogits, each below 2^-9 in root mean square, add up like a random walk over the values
        assert abs(num - float((dh.double() * a).sum())) <= 6 * 2 * 2.0 ** -9 * float((dh.double() * a).norm())
        num = (total(hd, wd + e * b) - total(hd, wd - e * b)) / (2 * e)
        assert abs(num - float((dw.double() * b).sum())) <= 6 * 2 * 2.0 ** -9 * float((dw.double() * b).norm())


def test_layer_norm_gradient_against_differences():
    from paper_2108_03645_b200 import train
    x, w, b, dy = randn(12, 40), 1 + 0.2 * randn(40, seed=1), randn(40, seed=2), randn(12, 40, seed=3)
    y, mean, rstd = train.layer_norm(x, w, b)
    dx, dw, db = train.layer_norm_backward(dy, x, mean, rstd, w)

    def total(xx, ww, bb):
        return float((torch.nn.functional.layer_norm(xx, (40,), ww, bb, 1e-5) * dy.double()).sum())
    xd, wd, bd = x.double(), w.double(), b.double()
    e = 1e-5
    for seed in range(3):
        p, q, r = randn(12, 40, seed=seed + 20).double(), randn(40, seed=seed + 30).double(), randn(40, seed=seed + 40).double()
        num = (total(xd + e * p, wd + e * q, bd + e * r) - total(xd - e * p, wd - e * q, bd - e * r)) / (2 * e)
        ana = float((dx.double() * p).sum() + (dw.double() * q).sum() + (db.double() * r).sum())
        assert abs(num - ana) <= 1e-4 * (1 + abs(num))


def test_autograd_functions():
    from paper_2108_03645_b200 import train
    x = randn(20, 64).requires_grad_()
    gain, shift = (1 + randn(64, seed=1) * 0.1).requires_grad_(), randn(64, seed=2).requires_grad_()
    head = (randn(300, 64, seed=3) * 0.1).bfloat16().requires_grad_()
    t = torch.arange(20, device="cuda") * 7
    loss = train.linear_cross_entropy_autograd(train.layer_norm_autograd(x, gain, shift).bfloat16(), head, t).mean()
    loss.backward()
    xr, gr, sr, hr = (p.detach().double().requires_grad_() for p in (x, gain, shift, head))
    ref = torch.nn.functional.cross_entropy(torch.nn.functional.layer_norm(xr, (64,), gr, sr) @ hr.t(), t)
    ref.backward()
    for a, b in ((x, xr), (gain, gr), (shift, sr), (head, hr)):
        assert float((a.grad.double() - b.grad).norm()) <= 0.02 * float(b.grad.norm())


# ---------------------------------------------------------------- orthogonalised update

def ns_reference(g, steps, coefficients, eps):
    a, b, c = coefficients
    x = g.double()
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        s = x @ x.mT
        x = a * x + (b * s + c * (s @ s)) @ x
    return x


def check_ns(g, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7):
    from paper_2108_03645_b200 import train
    o = train.orthogonalize(g, steps=steps, coefficients=coefficients, eps=eps)
    assert o.shape == g.shape and o.dtype == BF16
    r = ns_reference(g, steps, coefficients, eps)
    # bfloat16 result: a root mean square of 2^-8 / sqrt(3) at most, below 2^-9 over all mantissas; each step rounds three matrices to 11 bits, which the polynomial passes on with a slope of
    # about 1 where the values have arrived and which falls short of its gain on the values themselves before
    bound = 2.0 ** -9 + steps * 3 * 2.0 ** -11
    err = float((o.double() - r).norm() / r.norm().clamp(min=1e-30))
    assert err <= bound, (err, bound)
    return o


NS = [(1, 1), (1, 50), (50, 1), (7, 33), (64, 64), (100, 200), (200, 100), (128, 128), (128, 512), (512, 128), (129, 129), (128, 513),
      (130, 70), (513, 64), (255, 257), (500, 300), (256, 1024), (1000, 1368), (1111, 555), (32, 4096), (4100, 40), (247, 6276), (5000, 130), (71, 2063), (513, 8000), (128, 520), (600, 100), (77, 1025), (128, 4096), (8192, 128), (8000, 33), (20, 8191), (5, 8200), (9000, 128)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("m,n", NS)
def test_orthogonalize(m, n, dtype):
    check_ns((randn(m, n, seed=m + n) * 1e-2).to(dtype))


@pytest.mark.parametrize("count,m,n", [(2, 40, 30), (300, 16, 24), (3, 200, 333), (12, 90, 1188), (40, 2000, 64), (200, 30, 700), (7, 128, 1344), (12, 768, 768), (5, 300, 129), (160, 140, 130)])
def test_orthogonalize_many(count, m, n):
    g = randn(count, m, n).bfloat16()
    o = check_ns(g)
    from paper_2108_03645_b200 import train
    if count <= 12:
        for i in range(count):  # each as if it were alone (the same arithmetic in tiles of either size)
            assert torch.equal(o[i], train.orthogonalize(g[i]))


@pytest.mark.parametrize("m,n", [(96, 160), (300, 200)])
@pytest.mark.parametrize("steps,coefficients", [(1, (3.4445, -4.7750, 2.0315)), (2, (1.5, -0.5, 0.0)), (10, (1.5, -0.5, 0.0)), (3, (2.0, -1.5, 0.5))])
def test_orthogonalize_steps_and_coefficients(m, n, steps, coefficients):
    check_ns(randn(m, n), steps, coefficients)


@pytest.mark.parametrize("m,n", [(96, 160), (160, 96), (300, 520)])
def test_orthogonalize_singular_values(m, n):
    q = torch.linalg.svd(randn(m, n).double(), full_matrices=False)
    s = torch.linspace(0.05, 1.0, min(m, n), device="cuda").double()
    o = check_ns(((q.U * s) @ q.Vh).float())
    got = torch.linalg.svdvals(o.double())
    assert float(got.min()) > 0.6 and float(got.max()) < 1.25


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1.0, 1e12, 1e30])
def test_orthogonalize_any_scale(scale):
    for m, n in ((60, 90), (200, 300)):
        check_ns(randn(m, n) * scale, eps=1e-38 if scale < 1e-8 else 1e-7)


def test_orthogonalize_zero_and_nan():
    from paper_2108_03645_b200 import train
    for m, n in ((30, 50), (200, 150)):
        g = torch.zeros(3, m, n, device="cuda")
        g[2] = randn(m, n)
        g[1, 3, 4] = float("nan")
        o = train.orthogonalize(g)
        assert not bool(o[0].any()) and bool(torch.isnan(o[1]).any()) and bool(torch.isfinite(o[2]).all())
        assert torch.equal(o[2], train.orthogonalize(g[2]))


def test_orthogonalize_strides():
    from paper_2108_03645_b200 import train
    for dtype in (F32, BF16):
        for m, n in ((40, 70), (200, 144)):
            big = randn(3, m + 2, n + 5).to(dtype)
            view = big[:, 1:m + 1, 3:n + 3]
            assert torch.equal(train.orthogonalize(view), train.orthogonalize(view.contiguous()))
            t = big.mT
            assert torch.equal(train.orthogonalize(t), train.orthogonalize(t.contiguous()))
            one = big[:1, :m, :n].expand(2, m, n)
            assert torch.equal(train.orthogonalize(one), train.orthogonalize(one.contiguous()))


def test_orthogonalize_matrices_past_32_bits():
    from paper_2108_03645_b200 import train
    far = (1 << 31) + 16
    for m, n in ((32, 48), (140, 136)):
        flat = torch.empty(far + m * n, dtype=BF16, device="cuda")
        g = flat.as_strided((2, m, n), (far, n, 1))
        g.copy_(randn(2, m, n).bfloat16())
        assert torch.equal(train.orthogonalize(g), train.orthogonalize(g.contiguous()))


# ---------------------------------------------------------------- all of them

def test_same_inputs_give_the_same_bits():
    from paper_2108_03645_b200 import train
    x, dy, w = randn(3000, 1024).bfloat16(), randn(3000, 1024, seed=1).bfloat16(), randn(1024, seed=2)
    h, hw, t, g = ce_inputs(700, 512, 9000, BF16, 0.2)
    u = randn(4, 400, 600)
    first = None
    for _ in range(3):
        y, mean, rstd = train.layer_norm(x, w, w)
        loss, lse = train.linear_cross_entropy(h, hw, t)
        got = [y, mean, rstd, *train.layer_norm_backward(dy, x, mean, rstd, w), loss, lse,
               *train.linear_cross_entropy_backward(g, h, hw, t, lse), train.orthogonalize(u)]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_on_a_stream_of_the_callers_and_in_a_graph():
    from paper_2108_03645_b200 import train
    x, w = randn(64, 256).bfloat16(), randn(256, seed=1)
    h, hw, t, g = ce_inputs(100, 128, 900, BF16, 0.2)
    u, big = randn(2, 96, 128), randn(200, 300)

    def everything():
        y, mean, rstd = train.layer_norm(x, w, w)
        loss, lse = train.linear_cross_entropy(h, hw, t)
        return [y, *train.layer_norm_backward(y, x, mean, rstd, w), loss, *train.linear_cross_entropy_backward(g, h, hw, t, lse),
                train.orthogonalize(u), train.orthogonalize(big)]
    want = everything()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = everything()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_binding_refuses():
    from paper_2108_03645_b200 import binding, train
    x, w = randn(4, 64), randn(64)
    with pytest.raises(ValueError):
        train.layer_norm(x.double())
    with pytest.raises(ValueError):
        train.layer_norm(x, w[:32])
    with pytest.raises(ValueError):
        train.layer_norm(x, w, w.bfloat16())
    with pytest.raises(ValueError):
        train.layer_norm(x, w.half())
    with pytest.raises(binding.OnesError):
        train.layer_norm(x, w, eps=0.0)
    y, mean, rstd = train.layer_norm(x, w)
    with pytest.raises(ValueError):
        train.layer_norm_backward(y[:2], x, mean, rstd, w)
    with pytest.raises(ValueError):
        train.layer_norm_backward(y, x, mean.double(), rstd, w)
    h, hw, t, g = ce_inputs(8, 64, 100, BF16, 0.0)
    with pytest.raises(ValueError):
        train.linear_cross_entropy(h, hw.half(), t)
    with pytest.raises(ValueError):
        train.linear_cross_entropy(h, hw, t.int())
    with pytest.raises(ValueError):
        train.linear_cross_entropy(h[:4], hw, t)
    loss, lse = train.linear_cross_entropy(h, hw, t)
    with pytest.raises(ValueError):
        train.linear_cross_entropy_backward(g.double(), h, hw, t, lse)
    with pytest.raises(binding.OnesError):
        train.linear_cross_entropy_backward(g, h, hw, t, lse, piece=100)
    with pytest.raises(ValueError):
        train.orthogonalize(x[0])
    with pytest.raises(binding.OnesError):
        train.orthogonalize(x, steps=0)


def test_profiled_job_learns_and_is_scheduled():
    from paper_2108_03645_b200 import profile_job as pj
    job = pj.LanguageModelJob(pj.JobShape(width=128, inner=512, vocab=500, seq=32))
    token, target = job.batch(16, 0)
    losses = [float(job.step(token, target)) for _ in range(30)]
    assert all(math.isfinite(v) for v in losses) and losses[-1] < 0.7 * losses[0]
    # the step's gradients against automatic differentiation of the plain model in 32 bits
    loss, grads = job.gradients(token, target)
    p = [q.detach().float().requires_grad_() for q in (job.w1, job.w2, job.head, job.gain, job.shift)]
    x = job.embedding[token].float()
    z = x + torch.nn.functional.gelu(x @ p[0]) @ p[1]
    ref = torch.nn.functional.cross_entropy(torch.nn.functional.layer_norm(z, (128,), p[3], p[4]) @ p[2].t(), target, ignore_index=-100)
    ref.backward()
    assert abs(float(loss) - float(ref.detach())) <= 0.02 * float(ref.detach()) + 1e-3
    for got, want in zip(grads, p):
        assert float((got.float() - want.grad).norm()) <= 0.05 * float(want.grad.norm())
    out = pj.main(["--b0", "4", "--kmax", "2", "--width", "128", "--vocab", "1000", "--seq", "32", "--generations", "10"])
    assert len(out["seconds"]) == 3 and out["a"] >= 0 and out["c"] >= 0 and out["a"] + out["c"] > 0
    assert out["scheduled_batch"] in (0, 4, 8, 16) and out["cluster_gpus"] <= 64
