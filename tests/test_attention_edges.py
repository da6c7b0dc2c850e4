"""Attention and norm at the edges of their ranges, on the GPU: scores and squares that 32 bits do not hold, tensors whose parts are
of very different size, calls that outlast the limit of a wait.

Bounds are those of the operators' other tests (u = the unit roundoff of the type), but for the gradients of the scores: what they take
over from the rounding of `out` is given back, so that only products of two roundings are left of it.
"""
import math

import pytest

torch = pytest.importorskip("torch")
from test_attention_ops import BF16, F16, F32, TINY, U, attend64, close, randn  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    yield
    from paper_2108_03645_b200 import train
    train.check()


def hidden(n, first, dim, dtype, low, level, mark=1.0):
    """q, k, v of one head: value 0 of the first `first` keys is `low`, of every query `mark`; the others score level * 8 more or less."""
    q, k, v = (randn(n, 1, dim, seed=i) * 0.5 for i in range(3))
    q[..., 0], k[..., 0] = mark, 0.0
    q[..., 1], k[..., 1] = 1.0, level * 8
    k[:first, :, 0] = low
    return [t.to(dtype) for t in (q, k, v)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("first, level", [(128, -20), (128, -50), (200, -100), (256, -300), (300, 3), (1, -20), (130, -100)])
def test_attention_first_keys_score_minus_infinity(first, level, dim, dtype):
    """Rows see what is left; those that see nothing have lse = -infinity and NaN, as the definition has it."""
    from paper_2108_03645_b200 import train
    n = 500
    q, k, v = hidden(n, first, dim, dtype, -math.inf, level)
    out, lse = train.attention(q, k, v, scale=0.125)
    assert bool(out[:first].isnan().all()) and bool((lse[:first] == -math.inf).all())
    want, want_e, wlse, wlse_e, _, _ = attend64(q[first:], k[first:], v[first:], [n - first], 0.125)
    close(lse[first:], wlse, wlse_e)
    close(out[first:], want, want_e)


@pytest.mark.parametrize("scale, mark", [(0.125, 1.0), (0.125, 4.0), (1.0, 1.0), (1.0, 4.0)])
@pytest.mark.parametrize("first", [128, 150])
def test_attention_first_keys_hold_the_lowest_value(first, scale, mark):
    """The type's lowest value in a column that only hides: a finite score, or one that 32 bits do not hold."""
    from paper_2108_03645_b200 import train
    q, k, v = hidden(400, first, 64, BF16, torch.finfo(BF16).min, -100, mark)
    out, lse = train.attention(q, k, v, scale=scale)
    want, want_e, wlse, wlse_e, _, _ = attend64(q[first:], k[first:], v[first:], [400 - first], scale)
    close(lse[first:], wlse, wlse_e)
    close(out[first:], want, want_e)
    if scale * mark < 0.5:  # all scores alike: the mean of what the row sees
        mean = v[:first].double().cumsum(0) / torch.arange(1, first + 1, device="cuda").view(-1, 1, 1)
        size = v[:first].double().abs().cumsum(0) / torch.arange(1, first + 1, device="cuda").view(-1, 1, 1)
        close(out[:first], mean, 2.0 ** -8 * mean.abs() + (2.0 ** -8 + first * 2.0 ** -24) * size)


@pytest.mark.parametrize("heads, kv, dim", [(1, 1, 64), (1, 1, 128), (3, 1, 64)])
def test_attention_calls_outlast_the_limit_of_a_wait(heads, kv, dim):
    """A long sequence whose tiles are all whole, then a short one whose last tile is not: the warps that have to do with the short one only
    wait as long as the others are at work, whatever that takes."""
    import ctypes as C
    from paper_2108_03645_b200 import train
    n = 1 << 16
    q, k, v, dout = (randn(n + 100, h, dim, seed=h + i).bfloat16() for i, h in enumerate((heads, kv, kv, heads)))
    offsets = torch.tensor([0, n, n + 100], device="cuda")
    out, lse = train.attention(q, k, v, offsets)
    want = [out, lse, *train.attention_backward(dout, q, k, v, out, lse, offsets)]
    train.check()
    L = train.lib()
    assert L.ones_train_wait_limit(C.c_ulonglong(200_000)) == 0  # a fraction of each pass
    try:
        out, lse = train.attention(q, k, v, offsets)
        got = [out, lse, *train.attention_backward(dout, q, k, v, out, lse, offsets)]
        train.check()
    finally:
        assert L.ones_train_wait_limit(C.c_ulonglong(0)) == 0
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def gradients64(q, k, v, dout, scale):
    """Gradients of one sequence and bounds of their errors: {name: (value, bound)}."""
    u, f16 = U[q.dtype], q.dtype == F16
    n, h, d = q.shape
    kv = k.shape[1]
    x = {"dq": q, "dk": k, "dv": v}
    g, ge = ({name: torch.zeros_like(t, dtype=torch.float64) for name, t in x.items()} for _ in range(2))
    mask = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    # float16: ds is held times a power of two that takes 2 dim |dout| |v| to 2^15 at most and 2^13 at least (two powers of two, rounded up),
    # dim <= 128, in steps of 2^-24: off by 2^-25 2^8 / 2^13 = 2^-30 of the largest |dout| |v|, of the row for dq and of all for dk
    step = 2.0 ** -30 if f16 else 0.0
    for head in range(h):
        kh = head // (h // kv)
        a, b, c, do = (t.double() for t in (q[:, head], k[:, kh], v[:, kh], dout[:, head]))
        s = (a @ b.T * scale).masked_fill(~mask, -math.inf)
        # a score: sums of up to 128 products cut off at every 16 (2^-23 each), its factor and the argument of the exponential
        se = ((a.abs() @ b.abs().T * scale) * 2.0 ** -19 + 2.0 ** -20).masked_fill(~mask, 0).amax(1, keepdim=True)
        p = (s - torch.logsumexp(s, 1)[:, None]).exp()
        o = p @ c
        dp = do @ c.T
        off = dp - (do * o).sum(1, keepdim=True)
        ds = p * off
        g["dv"][:, kh] += p.T @ do
        g["dq"][:, head] = scale * ds @ b
        g["dk"][:, kh] += scale * ds.T @ a
        ge["dv"][:, kh] += (p * (u + 4 * se + n * 2.0 ** -22)).T @ do.abs()
        # out is off by two roundings of u (its own and the probabilities'), and so is dout . out; dp by its 32-bit sums
        de = (2 * u + 4 * se + n * 2.0 ** -24) * (do.abs() * (p @ c.abs())).sum(1, keepdim=True)
        dpe = 2.0 ** -19 * ((do.abs() * o.abs()).sum(1, keepdim=True) + do.abs() @ c.abs().T)
        # ds: its rounding, that of p, and dp's. Its sum over the row, which is 0, is known to n 2^-22 of its terms. What it is off by is taken off all of
        # them by their p. Of de, ds + p de is rounded (u p de), what all of these roundings add up to is in the sum (u de), and so is de, to be
        # met by the rounding of p (u p de): sum_j (1 + x_j) (ds_j + p_j e) k_j - (e + sum_j x_j (ds_j + p_j e)) sum_j (1 + y_j) p_j k_j, |x|, |y| <= u
        own = ds.abs() * (u + 4 * se + n * 2.0 ** -22) + p * dpe
        common = p * (own.sum(1, keepdim=True) * (u + 4 * se) + ds.abs().sum(1, keepdim=True) * (n * 2.0 ** -22) + de * (3 * u + 4 * se) +
                      (p * dpe).sum(1, keepdim=True))
        most = do.abs().amax(1, keepdim=True) * c.abs().max()
        ge["dq"][:, head] += scale * (own + common + mask * most * step) @ b.abs()
        ge["dk"][:, kh] += scale * (own + common + mask * most.max() * step).T @ a.abs()
        if f16:
            ge["dv"][:, kh] += 2.0 ** -37 * mask.double().T @ do.abs() + TINY[F16]
            ge["dq"][:, head] += TINY[F16]
            ge["dk"][:, kh] += TINY[F16]
    return {name: (g[name], ge[name] + u * g[name].abs() + 2.0 ** -130) for name in x}


def check_gradients(q, k, v, dout, lengths, scale=None):
    """Every sequence by itself."""
    from paper_2108_03645_b200 import train
    offsets = torch.tensor([0] + lengths).cumsum(0).cuda()
    out, lse = train.attention(q, k, v, offsets, scale=scale)
    got = dict(zip(("dq", "dk", "dv"), train.attention_backward(dout, q, k, v, out, lse, offsets, scale=scale)))
    for i in range(len(lengths)):
        rows = slice(int(offsets[i]), int(offsets[i + 1]))
        if not lengths[i]:
            continue
        for name, (want, bound) in gradients64(q[rows], k[rows], v[rows], dout[rows], scale or q.shape[-1] ** -0.5).items():
            close(got[name][rows], want, bound)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads, kv, dim", [(1, 1, 64), (2, 1, 128), (3, 1, 77)])
@pytest.mark.parametrize("mean, recent, large", [(4, False, False), (4, True, False), (4, False, True), (4, True, True), (0, True, True)])
def test_attention_gradients_of_inputs_with_structure(mean, recent, large, heads, kv, dim, dtype):
    """Values with a common mean, scores that favour the latest keys, and first keys that are large where no query looks: the rounding of
    `out` does not show in the gradients, wherever a row's probabilities lie."""
    n = 1000
    q, k, v, dout = (randn(n, h, dim, seed=h + i) * f for i, (h, f) in enumerate(((heads, 1.0), (kv, 0.5), (kv, 1.0), (heads, 1.0))))
    v += mean * (1 + 0.25 * randn(1, 1, dim, seed=9))
    q[..., 0], k[..., 0] = 2.0, 0.0
    if recent:
        k[..., 0] = torch.arange(n, device="cuda").view(-1, 1) * 0.1
    q[..., 3] = 0.0
    if large:
        k[:128, :, 3] = 60 * randn(128, kv, seed=7).sign()
        k[:128, :, 0] -= 40.0
    check_gradients(*(t.to(dtype) for t in (q, k, v, dout)), [n], scale=0.25)


@pytest.mark.parametrize("first, mark", [(100, 1.0), (128, 1.0), (150, 1.0), (128, 4.0)])
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_gradients_beside_the_lowest_value(dim, first, mark):
    """Keys that a column with the type's lowest value hides take nothing from the others' precision, and get nothing."""
    from paper_2108_03645_b200 import train
    n = 400
    q, k, v = hidden(n, first, dim, BF16, torch.finfo(BF16).min, -3, mark)
    dout = randn(n, 1, dim, seed=5).bfloat16()
    dout[:first] = 0
    out, lse = train.attention(q, k, v, scale=0.125)
    got = dict(zip(("dq", "dk", "dv"), train.attention_backward(dout, q, k, v, out, lse, scale=0.125)))
    for name, (want, bound) in gradients64(q[first:], k[first:], v[first:], dout[first:], 0.125).items():
        close(got[name][first:], want, bound)
        if mark == 1.0:  # (where the hidden rows' own scores are -infinity, they are NaN)
            assert not bool(got[name][:first].any())


@pytest.mark.parametrize("which", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("size", [2.0 ** -13, 2.0 ** -40])
def test_attention_bfloat16_gradients_beside_larger_sequences(which, size):
    """A sequence whose tensor is far smaller than its neighbour's has gradients as exact as by itself."""
    lengths = [300, 200, 70]
    x = {name: randn(570, h, 64, seed=h + i) for i, (name, h) in enumerate((("q", 4), ("k", 2), ("v", 2), ("dout", 4)))}
    x[which][300:500] *= size
    check_gradients(*(t.bfloat16() for t in x.values()), lengths)


@pytest.mark.parametrize("which", ["v", "dout"])
def test_attention_bfloat16_gradients_of_small_tokens(which):
    """The same between tokens of one sequence."""
    x = {name: randn(600, h, 128, seed=h + i) for i, (name, h) in enumerate((("q", 2), ("k", 1), ("v", 1), ("dout", 2)))}
    x[which][:100] *= 2.0 ** 14
    check_gradients(*(t.bfloat16() for t in x.values()), [600])


@pytest.mark.parametrize("heads, kv, dim", [(4, 2, 64), (3, 3, 128), (5, 1, 77)])
@pytest.mark.parametrize("which", ["v", "dout", "both"])
def test_attention_float16_gradients_beside_larger_sequences(which, heads, kv, dim):
    """A sequence whose dout or v is far smaller than its neighbours' has gradients as exact as by itself."""
    lengths = [300, 1, 200, 0, 129, 70]
    n = sum(lengths)
    q, k, v, dout = (randn(n, h, dim, seed=h + i) for i, h in enumerate((heads, kv, kv, heads)))
    small = slice(301, 501)
    if which != "dout":
        v *= 2.0 ** 7
        v[small] *= 2.0 ** -14
    if which != "v":
        dout *= 2.0 ** 6
        dout[small] *= 2.0 ** -12
    check_gradients(*(t.half() for t in (q, k, v, dout)), lengths)


@pytest.mark.parametrize("heads, kv", [(2, 1), (3, 3)])
def test_attention_float16_dq_of_small_rows(heads, kv):
    """dq of each row is as exact as its own dout allows."""
    q, k, v, dout = (randn(600, h, 64, seed=h + i) for i, h in enumerate((heads, kv, kv, heads)))
    dout *= 2.0 ** 8
    dout[50:] *= 2.0 ** -13
    dout[300:, -1] *= 2.0 ** -2
    check_gradients(*(t.half() for t in (q, k, v, dout)), [600])


@pytest.mark.parametrize("gap", [17.0, 17.5, 18.5])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attention_many_small_probabilities(gap, dtype):
    """One key far above 131071 others that together have a share of the row: float16 keeps them in steps of 2^-31 of the largest."""
    from paper_2108_03645_b200 import train
    n = 1 << 17
    q, k, v = torch.zeros(n, 1, 64, device="cuda"), torch.zeros(n, 1, 64, device="cuda"), torch.ones(n, 1, 64, device="cuda")
    q[..., 0], k[0, 0, 0], v[0] = 1.0, gap, 0.0
    out, lse = train.attention(*(t.to(dtype) for t in (q, k, v)), scale=1.0)
    rest = torch.arange(n, device="cuda", dtype=torch.float64) * math.exp(-gap)
    want, u = rest / (1 + rest), U[dtype]
    # 32-bit sums: 64 probabilities of a tile one after the other, then n / 128 tiles; products with v in n / 16 steps, cut off
    sums = (64 + n / 128) * 2.0 ** -24
    close(lse[:, 0], gap + torch.log1p(rest), torch.full_like(rest, 2.0 ** -20 + 2.0 ** -22 * gap + sums))
    bound = want * (2 * u + sums + n / 16 * 2.0 ** -23) + (2.0 ** -32 * n if dtype == F16 else 0.0) + TINY[dtype]
    close(out[:, 0], want[:, None].expand(n, 64), bound[:, None].expand(n, 64))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim, rotary, interleaved", [(64, 64, False), (128, 64, True), (81, 40, False)])
@pytest.mark.parametrize("size, eps", [(1e20, 1e-6), (1e30, 0.0), (3e37, 1e-6), (1e-25, 0.0), (1e-30, 1e-36)])
def test_qk_norm_squares_that_32_bits_do_not_hold(size, eps, dim, rotary, interleaved, dtype):
    """Vectors whose squares overflow or vanish, beside ordinary ones."""
    from test_attention_ops import check_qk_norm
    from paper_2108_03645_b200 import train
    q, k = randn(21, 3, dim), randn(21, 2, dim, seed=1)
    q[::2] *= size
    k[1::2, 1] *= size
    w = 1 + 0.2 * randn(dim, seed=3)
    f = 1e-3 / max(1.0, 1 / size)  # what is divided by the vectors' size stays in range
    dq, dk = f * randn(21, 3, dim, seed=5), f * randn(21, 2, dim, seed=6)
    check_qk_norm(*(t.to(dtype) for t in (q, k)), torch.arange(21, device="cuda") * 3, train.rotary_frequencies(rotary), w, w, dq.to(dtype), dk.to(dtype),
                  eps=eps, interleaved=interleaved)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attention_gradients_do_not_depend_on_other_sequences(dtype):
    """The bits of a sequence's results, whatever its neighbours hold: large values, small ones, infinities, NaN."""
    from paper_2108_03645_b200 import train
    lengths = [70, 5, 200, 131]
    offsets = torch.tensor([0] + lengths).cumsum(0).cuda()
    for heads, kv, dim in ((4, 2, 128), (3, 1, 64), (5, 1, 77)):
        plain = [randn(sum(lengths), h, dim, seed=i).to(dtype) for i, h in enumerate((heads, kv, kv, heads))]

        def step(q, k, v, dout):
            out, lse = train.attention(q, k, v, offsets)
            return [out, lse, *train.attention_backward(dout, q, k, v, out, lse, offsets)]
        want = step(*plain)
        for factor in (100.0, 1e-3, math.inf, math.nan):
            args = [t.clone() for t in plain]
            for t in args:
                t[75:275] *= factor
            keep = torch.ones(sum(lengths), dtype=torch.bool, device="cuda")
            keep[75:275] = False
            for a, b in zip(step(*args), want):
                assert torch.equal(a[keep], b[keep]), factor


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attention_many_empty_sequences(dtype):
    """Far more sequences than tokens: the same bits as without those that are empty."""
    from paper_2108_03645_b200 import train
    q, k, v, dout = (randn(450, h, 64, seed=i).to(dtype) for i, h in enumerate((4, 2, 2, 4)))
    few = torch.tensor([0, 1, 300, 430], device="cuda")
    many = few.repeat_interleave(2000)
    results = []
    for offsets in (few, many):
        out, lse = train.attention(q, k, v, offsets)
        results.append([out, lse, *train.attention_backward(dout, q, k, v, out, lse, offsets)])
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("limit", [1e-4, 1.0, 1e20])
def test_clip_factors_that_32_bits_do_not_hold(limit, dtype):
    """Gradients near the end of their range, scaled to a small norm."""
    from paper_2108_03645_b200 import train
    g = (randn(5000) * 5e37).to(dtype)
    want = g.double() * (limit / (float(g.double().norm()) + 1e-6))
    train.clip_gradients([g], limit)
    close(g, want, (U[dtype] + 2.0 ** -21) * want.abs() + TINY[dtype])
