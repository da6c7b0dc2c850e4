"""Training-step operators at the edges of what they accept, on the GPU: weights of the loss that differ by orders of
magnitude, matrices that are small beside eps, infinities, second derivatives, waits that run out, row counts near 2^31; and
the precision that the kernels claim. References are the definitions in 64 bits."""
import ctypes as C
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_train_ops import (BF16, F16, F32, TINY, U, _device, ce_inputs, ce_reference, check_ns, close, ns_reference,  # noqa: E402,F401
                            randn)


# ---------------------------------------------------------------- uneven weights of the loss

@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n", [48, 300])
@pytest.mark.parametrize("least", [1.0, 1e-2, 1e-3, 1e-5])
def test_linear_cross_entropy_uneven_weights(n, least, dtype):
    """Rows that weigh little beside others keep their gradients: what a 16-bit gradient of a logit is off by is one rounding of
    it, or of float16's smallest numbers with the largest |dloss| at 2^15: 2^-25 * 2^-15 of that."""
    from paper_2108_03645_b200 import train
    h, w, t, _ = ce_inputs(n, 96, 32001, dtype, 0.1, seed=n)
    w = (w.float() + 0.1).to(dtype)                # a mean: what is lost does not average out
    g = torch.full((n,), 1024.0, device="cuda")    # float16 training scales its loss
    g[1::2] *= least
    _, lse = train.linear_cross_entropy(h, w, t)
    dh, dw = train.linear_cross_entropy_backward(g, h, w, t, lse)
    r = ce_reference(h, w, t, g)
    k, v = h.shape[1], w.shape[0]
    tol = (k / 8 + 4) * 2.0 ** -23 * r["mass"] + 2.0 ** -20 * (1 + r["lse"].abs())   # of a logit, as in check_ce
    live = r["live"].double() * g.double()
    soft = torch.softmax(r["l"], 1) * live[:, None]
    e = U[dtype] * r["p"].abs() + soft * (torch.expm1(2 * tol) + 2.0 ** -20)[:, None] + 2.0 ** -22 * live[:, None] * (r["p"] < 0)
    e += TINY[dtype] * 2.0 ** -15 * float(g.max()) * r["live"][:, None]
    close(dh, r["dh"], U[dtype] * r["dh"].abs() + 1.01 * (e @ r["w"].abs()) + (v / 8 + 8) * 2.0 ** -23 * (r["p"].abs() @ r["w"].abs()) + TINY[dtype])
    close(dw, r["dw"], U[dtype] * r["dw"].abs() + 1.01 * (e.t() @ r["h"].abs()) + (n / 8 + 8) * 2.0 ** -23 * (r["p"].abs().t() @ r["h"].abs()) + TINY[dtype])


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("scale", [2.0 ** -120, 2.0 ** -100, 2.0 ** -60, 2.0 ** 110])
def test_linear_cross_entropy_weights_of_any_scale(scale, dtype):
    """Far beyond float16's range: dweight in 32 bits."""
    from paper_2108_03645_b200 import train
    h, w, t, g = ce_inputs(100, 64, 500, dtype, 0.2)
    g = (g * scale).float()
    _, lse = train.linear_cross_entropy(h, w, t)
    dw = train.linear_cross_entropy_backward(g, h, w, t, lse, weight_gradient=F32)[1]
    want = ce_reference(h, w, t, g)["dw"]
    # root mean square of the roundings below 2^-8; a result below 2^-126 is a multiple of 2^-149
    assert float((dw.double() - want).norm()) <= 2.0 ** -8 * float(want.norm()) + 2.0 ** -148 * want.numel() ** 0.5


# ---------------------------------------------------------------- matrices that are small beside eps

FORMS = [(30, 50), (40, 3000), (200, 150), (300, 2000), (150, 6000)]  # one block, a cluster, one launch of all blocks, cut along K


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n", FORMS)
def test_orthogonalize_zero_at_any_eps(m, n, dtype):
    from paper_2108_03645_b200 import train
    for eps in (1e-38, 1e-30, 1e-20, 1e-7, 1.0):
        g = torch.zeros(2, m, n, dtype=dtype, device="cuda")
        g[1] = randn(m, n).to(dtype)
        o = train.orthogonalize(g, eps=eps)
        assert not bool(o[0].any()) and bool(torch.isfinite(o[1]).all()) and bool(o[1].any())
        assert not bool(train.orthogonalize(g[0], eps=eps).any())


@pytest.mark.parametrize("m,n", FORMS)
@pytest.mark.parametrize("ratio", [1e-3, 1e-5, 5e-7, 1e-9, 1e-12])
def test_orthogonalize_small_beside_eps(m, n, ratio):
    g = randn(m, n)
    check_ns(g * (ratio * 1e-7 / g.norm()))
    check_ns(g * (ratio / g.norm()), steps=2, eps=1.0)
    check_ns(g * (ratio / g.norm()), steps=10, coefficients=(1.5, -0.5, 0.0), eps=1.0)


def test_orthogonalize_each_matrix_has_its_own_scale():
    from paper_2108_03645_b200 import train
    for m, n in FORMS:
        g = torch.stack([randn(m, n, seed=k) for k in range(4)])
        g *= torch.tensor([1.0, 1e-11, 0.0, 1e-14], device="cuda")[:, None, None]
        o = train.orthogonalize(g)
        assert not bool(o[2].any())
        for a, b in zip(g[[0, 1, 3]], o[[0, 1, 3]]):
            want = ns_reference(a, 5, (3.4445, -4.7750, 2.0315), 1e-7)
            assert float((b.double() - want).norm()) <= (2.0 ** -9 + 15 * 2.0 ** -11) * float(want.norm())


def test_orthogonalize_many_steps():
    """As many as are taken, and none beyond: the small coefficients make X decay, the second set holds it at 1."""
    from paper_2108_03645_b200 import binding, train
    for m, n in FORMS:
        check_ns(randn(m, n), steps=60, coefficients=(0.9, 0.0, 0.0))
        s = torch.linalg.svdvals(train.orthogonalize(randn(m, n), steps=1024, coefficients=(1.5, -0.5, 0.0)).double())
        assert float(s.max()) < 1.02
        with pytest.raises(binding.OnesError):
            train.orthogonalize(randn(m, n), steps=1025)


# ---------------------------------------------------------------- waits that run out

@pytest.mark.parametrize("which", [0, 1, 2])
def test_a_wait_that_runs_out_is_reported_once_and_waited_for_once(which):
    """A kernel of each file that waits a thousand times for what nobody sends: it spends one limit, not a thousand, the
    status says so once, and what comes after it is as before."""
    import time
    from paper_2108_03645_b200 import binding, train
    L = train.lib()
    x, h = randn(300, 512), ce_inputs(40, 64, 300, BF16, 0.2)
    everything = lambda: (*train.layer_norm(x), *train.linear_cross_entropy(*h[:3]), train.orthogonalize(x))  # noqa: E731
    want = everything()
    train.check()
    assert L.ones_train_wait_limit(C.c_ulonglong(20_000_000)) == 0
    try:
        begin = time.monotonic()
        assert L.ones_train_wait_for_nothing(which, 1000, C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
        torch.cuda.synchronize()
        assert 0.02 <= time.monotonic() - begin < 2.0
    finally:
        assert L.ones_train_wait_limit(C.c_ulonglong(0)) == 0
    with pytest.raises(binding.OnesError) as e:
        train.check()
    assert e.value.code == -9
    train.check()
    assert all(torch.equal(a, b) for a, b in zip(want, everything()))
    train.check()


# ---------------------------------------------------------------- automatic differentiation

def test_second_derivatives_are_refused():
    """The gradients are not differentiable themselves: a penalty on them is an error, not a constant."""
    from paper_2108_03645_b200 import train
    x, w = randn(6, 64).requires_grad_(), randn(64, seed=1).requires_grad_()
    loss = train.layer_norm_autograd(x, w).pow(3).sum()
    gx, gw = torch.autograd.grad(loss, (x, w), create_graph=True)
    with pytest.raises(RuntimeError):
        (loss + gx.pow(2).sum() + gw.pow(2).sum()).backward()
    h, hw, t, _ = ce_inputs(10, 64, 50, BF16, 0.0)
    h.requires_grad_(), hw.requires_grad_()
    loss = train.linear_cross_entropy_autograd(h, hw, t).pow(2).sum()
    gh, gw = torch.autograd.grad(loss, (h, hw), create_graph=True)
    with pytest.raises(RuntimeError):
        (loss + gh.float().pow(2).sum() + gw.float().pow(2).sum()).backward()


def test_functions_outside_the_graph_refuse_what_asks_for_a_gradient():
    from paper_2108_03645_b200 import train
    x, w = randn(6, 64), randn(64, seed=1)
    h, hw, t, g = ce_inputs(10, 64, 50, BF16, 0.0)
    y, mean, rstd = train.layer_norm(x, w, w)
    loss, lse = train.linear_cross_entropy(h, hw, t)
    ask = lambda v: v.clone().requires_grad_()  # noqa: E731
    # (orthogonalize is what an optimiser does with a gradient, under no_grad as a rule)
    calls = [(train.layer_norm, (x, w, w), 3), (train.layer_norm_backward, (y, x, mean, rstd, w), 5), (train.linear_cross_entropy, (h, hw, t), 2),
             (train.linear_cross_entropy_backward, (g, h, hw, t, lse), 3), (train.orthogonalize, (x,), 1)]
    for f, args, n in calls:
        for i in range(n):
            mine = [ask(v) if j == i else v for j, v in enumerate(args)]
            with pytest.raises(ValueError):
                f(*mine)
            with torch.no_grad():
                f(*mine)
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(x, torch.ones_like(x))
        with pytest.raises(ValueError):
            train.layer_norm(dual, w)
        with pytest.raises((ValueError, RuntimeError, NotImplementedError)):
            train.layer_norm_autograd(dual, w)


# ---------------------------------------------------------------- as many rows as are taken

def test_layer_norm_of_the_most_rows():
    """2^31 - 2^16 rows of one value, through the C ABI: the last ones are reached, and nothing behind them."""
    from paper_2108_03645_b200 import train
    L = train.lib()
    n = (1 << 31) - (1 << 16)
    free = torch.cuda.mem_get_info()[0]
    if free < 48 << 30:
        pytest.skip("needs 48 GB")
    x = torch.zeros(n + 64, dtype=BF16, device="cuda")
    dy = torch.zeros(n + 64, dtype=BF16, device="cuda")
    out = torch.full((n + 64,), 77.0, dtype=BF16, device="cuda")
    x[n - 5:], dy[n - 5:n], dy[n:] = 3.0, 2.0, 1000.0
    stat = torch.full((2, n + 64), 7.0, device="cuda")
    shift, sums = torch.full((1,), 0.5, dtype=BF16, device="cuda"), torch.empty(2, device="cuda")
    nbytes = L.ones_layer_norm_workspace_bytes(n, 1)
    space = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    assert L.ones_layer_norm(x.data_ptr(), 1, None, shift.data_ptr(), n, 1, 1e-5, 1, 1, out.data_ptr(), 1, stat.data_ptr(), stat[1].data_ptr(), s) == 0
    assert float(out[:n].min()) == float(out[:n].max()) == 0.5 and bool((out[n:] == 77.0).all())
    assert bool((stat[0, n - 5:n] == 3.0).all()) and bool((stat[:, n:] == 7.0).all()) and float(stat[0, :n - 5].abs().max()) == 0.0
    assert L.ones_layer_norm_backward(dy.data_ptr(), 1, x.data_ptr(), 1, stat.data_ptr(), stat[1].data_ptr(), None, n, 1, 1, 0, out.data_ptr(), 1,
                                      sums.data_ptr(), sums[1:].data_ptr(), space.data_ptr(), nbytes, s) == 0
    assert float(out[:n].abs().max()) == 0.0 and bool((out[n:] == 77.0).all())
    assert sums.tolist() == [0.0, 10.0]


# ---------------------------------------------------------------- infinities in the weight

@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n", [1, 40, 63, 64, 100, 300])
def test_linear_cross_entropy_entry_that_never_comes(n, dtype):
    """An entry whose logit is -inf in every row has probability 0: its row of dweight is 0, whatever the number of rows, and the
    others are as if it were not there. Some rows take no part."""
    from paper_2108_03645_b200 import train
    h, w, t, g = ce_inputs(n, 64, 300, dtype, 0.3)
    h[:, 3] = 1.0
    t[t == 7] = 8
    w[7, 3] = float("-inf")
    loss, lse = train.linear_cross_entropy(h, w, t)
    dw = train.linear_cross_entropy_backward(g, h, w, t, lse, weight_gradient=F32)[1]
    keep = torch.arange(300, device="cuda") != 7
    _, lse2 = train.linear_cross_entropy(h, w[keep].contiguous(), t - (t > 7).long())
    want = train.linear_cross_entropy_backward(g, h, w[keep].contiguous(), t - (t > 7).long(), lse2, weight_gradient=F32)[1]
    assert not bool(dw[7].any())
    # lse of the same logits joined in another order: a few roundings of 2^-24, which can move a 16-bit rounding
    assert float((dw[keep] - want).norm()) <= 2 * U[dtype] * float(want.norm())


# ---------------------------------------------------------------- precision

@pytest.mark.parametrize("d", [64, 1024, 4096, 16384])
def test_linear_cross_entropy_logits_of_one_product(d):
    """What is given back for the cut-off of evenly growing sums is at most 2^-30 * 4096 of a logit that had lost nothing."""
    from paper_2108_03645_b200 import train
    w = torch.zeros(300, d, dtype=BF16, device="cuda")
    h = torch.zeros(3, d, dtype=BF16, device="cuda")
    w[5, 0], w[9, d - 1] = 200.0, 200.0
    h[0, 0], h[1, d - 1], h[2, 0] = 2.0, 2.0, 2.0
    t = torch.tensor([7, 5, 5], device="cuda")
    loss, lse = train.linear_cross_entropy(h, w, t)
    bound = 400.0 * (4096 * 2.0 ** -30 + 2 * 2.0 ** -23)
    assert bool(((lse.double() - 400.0).abs() <= bound).all())
    assert bool(((loss[:2].double() - 400.0).abs() <= bound).all()) and float(loss[2]) == 0.0


@pytest.mark.parametrize("d,bound", [(2048, 7.5e-7), (4096, 1.2e-6)])
def test_linear_cross_entropy_precision(d, bound):
    """Dense rows: losses and log-sums near their exact values. Logits that are cut off by 2^-30 of themselves per column, as in
    the tensor cores, move both by 1.0e-6 of their norm at 2048 columns and by twice that at 4096, if it is not given back."""
    from paper_2108_03645_b200 import train
    n, v = 512, 32000
    w = (randn(v, d) * (2 / math.sqrt(d))).bfloat16()
    t = torch.randint(0, v, (n,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    h = (randn(n, d, seed=1) + w[t].float() * (4 * torch.rand(n, 1, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda"))).bfloat16()
    loss, lse = train.linear_cross_entropy(h, w, t)
    r = ce_reference(h, w, t)
    assert float((loss.double() - r["loss"]).norm()) <= bound * float(r["loss"].norm())
    assert float((lse.double() - r["lse"]).norm()) <= bound * float(r["lse"].norm())


def momentum(m, n, dtype):
    """A part of low rank, and noise."""
    r = max(1, min(m, n) // 4)
    return ((randn(m, r) @ randn(r, n, seed=1) / math.sqrt(r) + 0.5 * randn(m, n, seed=2)) * 1e-3).to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n", [(768, 768), (1999, 1001), (128, 4096), (71, 2063), (128, 256), (32, 8192)])
def test_orthogonalize_precision(m, n, dtype):
    """Within 2.2e-3 of the norm, of which the rounding of the result is 1.66e-3."""
    from paper_2108_03645_b200 import train
    g = momentum(m, n, dtype)
    want = ns_reference(g, 5, (3.4445, -4.7750, 2.0315), 1e-7)
    assert float((train.orthogonalize(g).double() - want).norm()) <= 2.2e-3 * float(want.norm())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,bound", [(32, 512, 3e-4), (71, 2063, 5e-4), (32, 8192, 2.5e-4), (200, 2500, 2e-4), (300, 4000, 2e-4)])
def test_orthogonalize_rows_have_their_length(m, n, bound, dtype):
    """The roundings of the result average out over a long row; what is left is the row's factor. A model of the arithmetic in 64
    bits has it off (root mean square over the rows, at most over six inputs) by 2.0e-4, 3.2e-4, 1.5e-4, 1.2e-4 and 0.9e-4 for
    these sizes, and by at least 4.1e-4, 7.0e-4, 3.6e-4, 2.8e-4 and 3.5e-4 without the Gram matrix's diagonal in 32 bits or
    without the factors that give back the rounding of the polynomial's."""
    from paper_2108_03645_b200 import train
    g = momentum(m, n, dtype)
    for flip in (False, True):
        o = train.orthogonalize(g.mT if flip else g).double()
        o = o.mT if flip else o
        want = ns_reference(g, 5, (3.4445, -4.7750, 2.0315), 1e-7)
        off = (o * want).sum(1) / want.square().sum(1) - 1
        assert float(off.square().mean().sqrt()) <= bound
