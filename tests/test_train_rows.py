"""Training-step operators on rows of odd lengths, starts and distances, on the GPU: the definitions in 64 bits, as in
test_train_ops, at the sizes where another kernel or another end of a row begins."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_train_ops import BF16, F16, F32, _device, ce_inputs, check_ce, check_norm, randn  # noqa: E402,F401


def placed(t, ld, start):
    """t's values in rows `ld` apart that begin `start` values into a buffer of NaN."""
    n, d = t.shape
    buf = torch.full((start + n * ld + 8,), float("nan"), dtype=t.dtype, device="cuda")
    out = buf.as_strided((n, d), (ld, 1), start)
    out.copy_(t)
    return out


# lengths around whole warps' shares (512 columns), around the steps between kernels, and few and many rows of each
ROWS = [(4800, 257), (4800, 505), (6000, 511), (1200, 131), (2500, 257), (1200, 511), (300, 1025), (1184, 1535), (700, 1537), (1300, 2047),
        (298, 2049), (1200, 2561), (297, 4095), (1190, 4001), (310, 4097), (1184, 8191), (150, 8193), (299, 16383), (3, 12345)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,d", ROWS)
def test_layer_norm_odd_rows(n, d, dtype):
    x, dy = (randn(n, d, seed=n + d) * 2 + 1).to(dtype), randn(n, d, seed=7).to(dtype)
    w, b = 1 + 0.3 * randn(d, seed=3), randn(d, seed=4)
    check_norm(x, w, b, dy)                                            # starts change from row to row
    check_norm(placed(x, d + 3, 1), w.to(dtype), b.to(dtype), placed(dy, d + 2, 5))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("start", range(8))
def test_layer_norm_first_and_last_block(dtype, start):
    """The blocks that reach over a tensor's ends: few columns to a row, every start, and a tensor within its own block."""
    for n, d, ld in ((300, 1501, 1501), (1200, 1030, 1031)):
        x, dy = placed((randn(n, d, seed=start) + 1).to(dtype), ld, start), placed(randn(n, d, seed=5).to(dtype), d, 7 - start)
        check_norm(x, randn(d, seed=3), randn(d, seed=4), dy)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,d", [(301, 1501), (1200, 1537), (4801, 505)])
def test_layer_norm_odd_rows_keep_nan_to_themselves(n, d, dtype):
    from paper_2108_03645_b200 import train
    x = randn(n, d).to(dtype)
    want = train.layer_norm(x)[0]
    x[7, d - 1], x[n - 1, 0], x[0, 3] = float("nan"), float("inf"), float("nan")
    got = train.layer_norm(x)[0]
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[[0, 7, n - 1]] = False
    assert torch.equal(got[keep], want[keep]) and not bool(got[~keep].isfinite().any())


@pytest.mark.parametrize("dtype,n,d", [(F32, 300, 1501), (F32, 1200, 1501), (BF16, 300, 1501), (F16, 299, 8195), (BF16, 4800, 505)])
def test_layer_norm_odd_rows_touch_nothing_else(dtype, n, d):
    from paper_2108_03645_b200 import train
    L = train.lib()
    kind = {F32: 0, BF16: 1, F16: 2}[dtype]
    x, dy, w = randn(n, d).to(dtype), randn(n, d, seed=1).to(dtype), randn(d, seed=2)
    stat = torch.empty(2, n, device="cuda")
    nbytes = L.ones_layer_norm_workspace_bytes(n, d)
    space, dwb = torch.empty(nbytes, dtype=torch.uint8, device="cuda"), torch.empty(2, d, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    ld, start = d + 3, 5                                               # what lies between the rows stays as it is
    for call in ("forward", "backward"):
        out = torch.full((start + n * ld + 8,), 77.0, dtype=dtype, device="cuda")
        p = out.data_ptr() + start * out.element_size()
        if call == "forward":
            rc = L.ones_layer_norm(x.data_ptr(), d, w.data_ptr(), w.data_ptr(), n, d, 1e-5, kind, 0, p, ld, stat.data_ptr(),
                                   stat[1].data_ptr(), s)
        else:
            rc = L.ones_layer_norm_backward(dy.data_ptr(), d, x.data_ptr(), d, stat.data_ptr(), stat[1].data_ptr(), w.data_ptr(), n, d,
                                            kind, 0, p, ld, dwb.data_ptr(), dwb[1].data_ptr(), space.data_ptr(), nbytes, s)
        assert rc == 0
        inside = torch.zeros_like(out, dtype=torch.bool)
        inside.as_strided((n, d), (ld, 1), start).fill_(True)
        assert bool((out[~inside] == 77.0).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,d,ld,start", [(1, 1, 1, 0), (1, 5, 5, 3), (7, 9, 9, 1), (40, 8, 11, 2), (301, 505, 505, 7), (33, 2048, 2051, 4),
                                          (3000, 71, 72, 1), (5, 10001, 10001, 6)])
def test_align_rows(n, d, ld, start, dtype):
    from paper_2108_03645_b200 import train
    src = placed(randn(n, d, seed=n).to(dtype), ld, start)
    ldd = (d + 7) // 8 * 8 + 8
    dst = torch.full((n, ldd), 77.0, dtype=dtype, device="cuda")
    assert train.lib().ones_align_rows(src.data_ptr(), ld, n, d, 1 if dtype == BF16 else 2, dst.data_ptr(), ldd,
                                       torch.cuda.current_stream().cuda_stream) == 0
    up = (d + 7) // 8 * 8
    assert torch.equal(dst[:, :d], src) and bool((dst[:, d:up] == 0).all()) and bool((dst[:, up:] == 77.0).all())


def test_align_rows_past_32_bits():
    from paper_2108_03645_b200 import train
    n, d, ld = 70001, 33, 33001                                        # 2.3e9 values from first to last
    src = torch.zeros(n * ld + 1, dtype=BF16, device="cuda").as_strided((n, d), (ld, 1), 1)
    src.copy_(randn(n, d))
    dst = torch.empty(n, 40, dtype=BF16, device="cuda")
    assert train.lib().ones_align_rows(src.data_ptr(), ld, n, d, 1, dst.data_ptr(), 40, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(dst[:, :d], src)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,d,v", [(3, 65, 300), (200, 501, 1000), (64, 174, 40001), (600, 72, 100)])
def test_linear_cross_entropy_odd_rows(n, d, v, dtype):
    h, w, t, g = ce_inputs(n, d, v, dtype, 0.1)
    check_ce(placed(h, d + 1, 3), placed(w, d + 3, 1), t, g)


# many rows and a small weight: the rows are what is cut into parts, and how many of them take part is known late
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,d,v,ignored,piece", [(3000, 72, 300, 0.1, 0), (5000, 65, 111, 0.0, 0), (2000, 520, 260, 0.97, 0),
                                                 (2500, 130, 1000, 0.3, 256), (9000, 96, 50, 0.999, 0), (4097, 8, 2, 0.5, 0)])
def test_linear_cross_entropy_small_weight(n, d, v, ignored, piece, dtype):
    h, w, t, g = ce_inputs(n, d, v, dtype, ignored)
    check_ce(h, w, t, g, piece=piece)
    check_ce(h, w, t, g, piece=piece, weight_gradient=F32)


def test_linear_cross_entropy_small_weight_no_row_takes_part():
    from paper_2108_03645_b200 import train
    h, w, t, g = ce_inputs(3000, 72, 300, BF16, 0.0)
    t[:] = -1
    loss, lse = train.linear_cross_entropy(h, w, t)
    dh, dw = train.linear_cross_entropy_backward(g, h, w, t, lse)
    assert not bool(loss.any()) and not bool(dh.any()) and not bool(dw.any())


@pytest.mark.parametrize("n", [1, 31, 33, 8191, 8192, 8193, 20000])
def test_linear_cross_entropy_finds_the_rows_that_take_part(n):
    """Whatever their number and place: their order shows in the gradients."""
    h, w, t, g = ce_inputs(n, 64, 40, BF16, 0.4, seed=n)
    check_ce(h, w, t, g)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [1, 9, 15, 17, 33, 113, 130, 207, 255, 257, 271, 513, 777])
def test_linear_cross_entropy_weight_gradient_rows_of_any_length(d, dtype):
    """Whatever the lengths, starts and distances of its rows, and nothing beside them."""
    from paper_2108_03645_b200 import train
    L = train.lib()
    n, v = 70, 700
    h, w, t, g = ce_inputs(n, d, v, dtype, 0.1)
    lse = train.linear_cross_entropy(h, w, t)[1]
    dh, want = train.linear_cross_entropy_backward(g, h, w, t, lse, weight_gradient=F32)
    check_ce(h, w, t, g)
    kind, up = (1 if dtype == BF16 else 2), (d + 7) // 8 * 8
    wa, ha = torch.zeros(v, up, dtype=dtype, device="cuda"), h.contiguous()
    wa[:, :d] = w
    nbytes = L.ones_linear_ce_backward_workspace_bytes(n, d, v, 0)
    space = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    for ld, start in ((d, 0), (d, 1), (d + 1, 3), (d + 2, 6), (up + 8, 2)):
        buf = torch.full((start + v * ld + 16,), 77.0, dtype=dtype, device="cuda")
        assert L.ones_linear_ce_backward(g.data_ptr(), ha.data_ptr(), d, wa.data_ptr(), up, t.data_ptr(), lse.data_ptr(), n, d, v, kind, kind,
                                         0, dh.data_ptr(), d, buf.data_ptr() + 2 * start, ld, space.data_ptr(), nbytes, s) == 0
        got = buf.as_strided((v, d), (ld, 1), start)
        assert torch.equal(got, want.to(dtype))                        # the same sums, rounded once
        inside = torch.zeros_like(buf, dtype=torch.bool)
        inside.as_strided((v, d), (ld, 1), start).fill_(True)
        assert bool((buf[~inside] == 77.0).all())
