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
