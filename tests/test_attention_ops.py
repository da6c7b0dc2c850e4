"""Norm and rotation of queries and keys, causal attention over packed sequences and clipping of gradients against their
definitions in 64 bits, on the GPU.

Bounds are derived from the arithmetic: u = the unit roundoff of the type (2^-24 for float32, 2^-8 for bfloat16, 2^-11 for
float16): one rounding of the result, one of the probabilities and one of the scores' gradients for their products, and what
32-bit sums add, element by element.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -25}  # half the spacing of the smallest numbers (or all of it)


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    yield
    from paper_2108_03645_b200 import train
    train.check()


def randn(*size, seed=0):
    return torch.randn(size, generator=torch.Generator(device="cuda").manual_seed(seed + 1), device="cuda")


def close(got, want, bound):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bool(bad.any()), (int(bad.sum()), float(((got.double() - want).abs() / bound.clamp(min=1e-300)).nan_to_num(1e300).max()))


def packed(parts, gap=0):
    """Tensors [tokens][heads][dim] as slices of one buffer whose other values are NaN."""
    h = [p.shape[1] for p in parts]
    buf = torch.full((parts[0].shape[0], sum(h) + gap, parts[0].shape[2]), float("nan"), dtype=parts[0].dtype, device="cuda")
    out, at = [], 0
    for p in parts:
        buf[:, at:at + p.shape[1]] = p
        out.append(buf[:, at:at + p.shape[1]])
        at += p.shape[1]
    return out


# ---------------------------------------------------------------- norm and rotation

def turn64(x, cos, sin, interleaved):
    half = cos.shape[-1]
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    y = x.clone()
    p, q = a * cos - b * sin, a * sin + b * cos
    if interleaved:
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = p, q
    else:
        y[..., :half], y[..., half:2 * half] = p, q
    return y


def pair_size(x, half, interleaved):
    """|a| + |b| of the pair that a value turns with, |x| where it does not turn."""
    one = torch.ones(half, dtype=torch.float64, device="cuda")
    return turn64(x.abs(), one, one, interleaved).abs() + turn64(x.abs(), one, -one, interleaved).abs()


def check_qk_norm(q, k, pos, freq, qw, kw, dq, dk, eps=1e-6, interleaved=False):
    from paper_2108_03645_b200 import train
    got = train.qk_norm(q, k, pos, freq, qw, kw, eps=eps, interleaved=interleaved)
    grads = train.qk_norm_backward(dq, dk, q, k, pos, freq, qw, kw, eps=eps, interleaved=interleaved)
    u, e = U[q.dtype], 2.0 ** -19  # e: sums of up to 256 squares in chains of 16 and a tree, r, sine and cosine (2^-22), products
    angle = pos.double()[..., None] * freq
    cos, sin = angle.cos()[..., None, :], angle.sin()[..., None, :]
    for x, w, dy, y, dx, dw in ((q, qw, dq, got[0], grads[0], grads[2]), (k, kw, dk, got[1], grads[1], grads[3])):
        x64, w64 = x.double(), torch.ones(x.shape[-1], device="cuda").double() if w is None else w.double()
        r = 1 / (x64.square().mean(-1, keepdim=True) + eps).sqrt()
        n = x64 * r * w64
        want = turn64(n, cos, sin, interleaved)
        close(y, want, u * want.abs() + e * pair_size(n, freq.numel(), interleaved) + TINY[x.dtype])
        g = turn64(dy.double(), cos, -sin, interleaved)
        ge = e * pair_size(dy.double(), freq.numel(), interleaved)
        gw, m = g * w64, (g.abs() + ge / e) * w64.abs()
        c = (gw * x64).mean(-1, keepdim=True)
        want = r * (gw - x64 * r * r * c)
        size = r * (m + x64.abs() * r * r * (m * x64.abs()).mean(-1, keepdim=True))
        close(dx, want, u * want.abs() + 2 * e * size + TINY[x.dtype])
        want = (g * x64 * r).flatten(0, -2).sum(0)
        close(dw, want, U[dw.dtype] * want.abs() + 2.0 ** -15 * ((g.abs() + ge / e) * x64.abs() * r).flatten(0, -2).sum(0) + TINY[dw.dtype])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("tokens, heads, kv, dim, rotary, interleaved, wtype", [
    (1, 1, 1, 64, 64, False, None), (5, 8, 2, 64, 64, False, F32), (33, 16, 4, 128, 128, False, "x"), (7, 3, 3, 128, 64, True, F32),
    (129, 5, 1, 80, 80, False, "x"), (40, 6, 2, 96, 32, False, F32), (17, 2, 1, 81, 40, True, F32), (9, 4, 2, 33, 32, False, "x"),
    (3, 2, 2, 1, 0, False, F32), (11, 3, 1, 2, 2, True, "x"), (257, 1, 1, 256, 256, False, F32), (6, 1, 1, 255, 254, True, F32),
    (1000, 12, 3, 128, 128, True, "x"), (3, 100, 7, 24, 8, False, F32)])
def test_qk_norm(dtype, tokens, heads, kv, dim, rotary, interleaved, wtype):
    from paper_2108_03645_b200 import train
    scale = 0.3 + 2 * randn(1, heads + kv, 1, seed=9).abs()
    x = (randn(tokens, heads + kv, dim) * scale).to(dtype)
    q, k = packed([x[:, :heads], x[:, heads:]], gap=1)
    wt = dtype if wtype == "x" else wtype
    qw, kw = (None, None) if wt is None else ((1 + 0.2 * randn(dim, seed=3)).to(wt), (1 + 0.2 * randn(dim, seed=4)).to(wt))
    pos = torch.arange(tokens, device="cuda") * 3 + 5
    dq, dk = randn(tokens, heads, dim, seed=5).to(dtype) * 0.1, randn(tokens, kv, dim, seed=6).to(dtype) * 0.1
    check_qk_norm(q, k, pos, train.rotary_frequencies(rotary), qw, kw, dq, dk, interleaved=interleaved)


@pytest.mark.parametrize("dtype, heads, kv, dim, rotary", [(BF16, 1, 1, 256, 256), (BF16, 2, 2, 192, 192), (F32, 1, 0, 256, 256), (F16, 2, 1, 255, 254)])
def test_qk_norm_many_tokens_of_few_heads(dtype, heads, kv, dim, rotary):
    """Blocks take as many tokens at a time as the room for their angles allows."""
    from paper_2108_03645_b200 import train
    n = 50000
    q, k = randn(n, heads, dim).to(dtype), randn(n, kv, dim, seed=1).to(dtype)
    freq, w = train.rotary_frequencies(rotary), 1 + 0.2 * randn(dim, seed=3)
    check_qk_norm(q, k, torch.arange(n, device="cuda"), freq, w, w, randn(n, heads, dim, seed=5).to(dtype), randn(n, kv, dim, seed=6).to(dtype))


def test_qk_norm_at_far_positions_and_back():
    """Angles of 2^40 radians keep what 64 bits hold of them; negative positions turn the other way."""
    from paper_2108_03645_b200 import train
    q, k = randn(64, 2, 64), randn(64, 1, 64, seed=1)
    freq = train.rotary_frequencies(64)
    e = randn(64, 2, 64, seed=2), randn(64, 1, 64, seed=3)
    check_qk_norm(q, k, torch.arange(64, device="cuda") + 4_000_000, freq, None, None, *e)
    check_qk_norm(q, k, -torch.arange(64, device="cuda") * 977, freq, None, None, *e, interleaved=True)
    far = train.qk_norm(q, k, torch.full((64,), 1 << 31, device="cuda"), freq[:1])[0].double()
    a = torch.tensor(float(1 << 31), dtype=torch.float64)
    r = 1 / (q.double().square().mean(-1) + 1e-6).sqrt()
    want = (q[..., 0].double() * a.cos().item() - q[..., 1].double() * a.sin().item()) * r
    assert float((far[..., 0] - want).abs().max()) < 1e-5


def test_qk_norm_shapes_zeros_and_no_tokens():
    from paper_2108_03645_b200 import train
    freq = train.rotary_frequencies(32)
    q, k = randn(2, 3, 4, 32).bfloat16(), randn(2, 3, 2, 32, seed=1).bfloat16()
    pos = torch.arange(3, device="cuda").expand(2, 3)
    a = train.qk_norm(q, k, pos, freq)
    b = train.qk_norm(q.view(6, 4, 32), k.view(6, 2, 32), pos.reshape(6), freq)
    assert torch.equal(a[0].view(6, 4, 32), b[0]) and torch.equal(a[1].view(6, 2, 32), b[1])
    t = q.transpose(-1, -2).contiguous().transpose(-1, -2)  # values of a head are apart
    assert torch.equal(train.qk_norm(t, k, pos, freq)[0], a[0])
    z = torch.zeros(5, 2, 32, device="cuda")
    y = train.qk_norm(z, z, torch.arange(5, device="cuda"), freq)
    assert torch.equal(y[0], z)
    none = train.qk_norm(q[:, :0], k[:, :0], pos[:, :0], freq)
    assert none[0].shape == (2, 0, 4, 32)
    w = torch.ones(32, device="cuda")
    _, _, dw, _ = train.qk_norm_backward(q[:, :0], k[:, :0], q[:, :0], k[:, :0], pos[:, :0], freq, w, w)
    assert not bool(dw.any())


def test_qk_norm_one_head_or_none():
    """A single head's distance to the next does not matter, and one side may have no heads."""
    from paper_2108_03645_b200 import train
    freq, pos = train.rotary_frequencies(32), torch.arange(10, device="cuda").view(2, 5)
    q, k = randn(2, 5, 1, 32), randn(2, 5, 3, 32, seed=1)
    want = train.qk_norm(q, k, pos, freq)
    odd = q.as_strided((2, 5, 1, 32), (160, 32, 1, 1))
    assert torch.equal(train.qk_norm(odd, k, pos, freq)[0], want[0])
    for x in train.qk_norm_backward(odd, k, odd, k, pos, freq), train.qk_norm_backward(q, k, q, k, pos, freq):
        assert torch.equal(x[0], train.qk_norm_backward(q, k, q, k, pos, freq)[0])
    none = train.qk_norm(q[:, :, :0], k, pos, freq)
    assert none[0].shape == (2, 5, 0, 32) and torch.equal(none[1], want[1])
    assert torch.equal(train.qk_norm(q, k[:, :, :0], pos, freq)[0], want[0])


def test_qk_norm_keeps_what_is_not_finite_in_its_vector():
    from paper_2108_03645_b200 import train
    q, k = randn(9, 4, 64).half(), randn(9, 2, 64, seed=1).half()
    pos, freq = torch.arange(9, device="cuda"), train.rotary_frequencies(64)
    want = train.qk_norm(q, k, pos, freq)[0]
    q[3, 1, 5], q[6, 0, 63] = float("nan"), float("inf")
    got = train.qk_norm(q, k, pos, freq)[0]
    keep = torch.ones(9, 4, dtype=torch.bool, device="cuda")
    keep[3, 1] = keep[6, 0] = False
    assert torch.equal(got[keep], want[keep]) and bool(got[3, 1].isnan().all())


def test_qk_norm_gradients_against_differences():
    from paper_2108_03645_b200 import train
    pos, freq = torch.arange(3, device="cuda"), train.rotary_frequencies(16)
    q, k, w = randn(3, 2, 16), randn(3, 1, 16, seed=1), 1 + 0.1 * randn(16, seed=2)
    cq, ck = randn(3, 2, 16, seed=3).double(), randn(3, 1, 16, seed=4).double()

    def f(q, k, w):
        a, b = train.qk_norm(q, k, pos, freq, w, w)
        return float((a.double() * cq).sum() + (b.double() * ck).sum())
    dq, dk, dqw, dkw = train.qk_norm_backward(cq.float(), ck.float(), q, k, pos, freq, w, w)
    for x, g, at in ((q, dq, 0), (k, dk, 1), (w, dqw + dkw, 2)):
        for i in (0, 7, x.numel() - 1):
            args = [q, k, w]
            side = []
            for s in (1, -1):
                y = x.clone()
                y.view(-1)[i] += s * 2.0 ** -7
                args[at] = y
                side.append(f(*args))
            # the third derivative is of order 10, the values have 2^-22 of about 10
            assert abs((side[0] - side[1]) * 2 ** 6 - float(g.reshape(-1)[i])) < 10 * 2.0 ** -14 * 4 + 2.0 ** 6 * 1e-5


# ---------------------------------------------------------------- attention

def attend64(q, k, v, lengths, scale, dout=None):
    """out, lse, bounds of their errors; with dout also gradients and theirs."""
    u = U[q.dtype]
    n, h, d = q.shape
    kv = k.shape[1]
    q64, k64, v64 = (t.double() for t in (q, k, v))
    z = lambda t: torch.zeros_like(t, dtype=torch.float64)
    out, out_e, lse, lse_e = z(q), z(q), z(q[..., 0]), z(q[..., 0])
    g = {x: z(t) for x, t in (("dq", q), ("dk", k), ("dv", v))}
    ge = {x: z(t) for x, t in g.items()}
    at = 0
    f16 = q.dtype == F16
    for length in lengths:
        rows = slice(at, at + length)
        at += length
        if not length:
            continue
        mask = torch.ones(length, length, dtype=torch.bool, device="cuda").tril()
        for head in range(h):
            kh = head // (h // kv)
            a, b, c = q64[rows, head], k64[rows, kh], v64[rows, kh]
            s = (a @ b.T * scale).masked_fill(~mask, -math.inf)
            # a score: sums of up to 128 products cut off at every 16 (2^-23 each), its factor and the argument of the exponential
            se = ((a.abs() @ b.abs().T * scale) * 2.0 ** -19 + 2.0 ** -20).masked_fill(~mask, 0).amax(1, keepdim=True)
            l = torch.logsumexp(s, 1)
            p = (s - l[:, None]).exp()
            o = p @ c
            out[rows, head], lse[rows, head] = o, l
            out_e[rows, head] = u * o.abs() + (u + 4 * se + length * 2.0 ** -24) * (p @ c.abs())
            if f16:  # what is below 2^-14 of the row's maximum is rounded to steps of 2^-24
                out_e[rows, head] += 2.0 ** -25 * mask.double() @ c.abs() + TINY[F16]
            lse_e[rows, head] = se[:, 0] + 2.0 ** -20 + l.abs() * 2.0 ** -22
            if dout is None:
                continue
            do = dout[rows, head].double()
            dp = do @ c.T
            delta = (do * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            g["dv"][rows, kh] += p.T @ do
            g["dq"][rows, head] = scale * ds @ b
            g["dk"][rows, kh] += scale * ds.T @ a
            pe = p * (u + 4 * se)
            ge["dv"][rows, kh] += pe.T @ do.abs() + p.T @ do.abs() * length * 2.0 ** -22
            # delta comes from out as it was rounded; dp and delta are sums of 128 products in 32 bits
            de = (do.abs() * out_e[rows, head]).sum(1, keepdim=True) + 2.0 ** -19 * ((do.abs() * o.abs()).sum(1, keepdim=True) + do.abs() @ c.abs().T)
            dse = p * de + ds.abs() * (u + 4 * se) + p * (dp - delta).abs() * length * 2.0 ** -22
            # ds is held as float16 times 2^sigma with sigma = 15 - 8 - e - f, where max |dout| >= 2^(e - 1), max |v| >= 2^(f - 1): its
            # steps are 2^-24 at least, so it is off by 2^-25 2^-sigma = 2^-32 2^(e + f) <= 2^-30 max |dout| max |v|
            most = dout[:sum(lengths)].double().abs().max() * v64[:sum(lengths)].abs().max()
            dse = dse + mask * most * 2.0 ** -30
            if f16:
                ge["dv"][rows, kh] += 2.0 ** -37 * mask.double().T @ do.abs() + TINY[F16]
                ge["dq"][rows, head] += TINY[F16]
                ge["dk"][rows, kh] += TINY[F16]
            ge["dq"][rows, head] += scale * dse @ b.abs()
            ge["dk"][rows, kh] += scale * dse.T @ a.abs()
    for x in g:
        ge[x] += u * g[x].abs() + 2.0 ** -130
    return out, out_e + 2.0 ** -130, lse, lse_e, g, ge


def check_attention(q, k, v, lengths, dout=None, scale=None, tail=0, dense=False):
    from paper_2108_03645_b200 import train
    offsets = None if dense else torch.tensor([0] + lengths).cumsum(0).cuda()
    out, lse = train.attention(q, k, v, offsets, scale=scale)
    r_out, r_out_e, r_lse, r_lse_e, g, ge = attend64(q, k, v, lengths, scale or q.shape[-1] ** -0.5, dout)
    n = sum(lengths)
    assert not bool(out[n:].any()) and not bool(lse[n:].any()) and out.shape == q.shape and lse.shape == q.shape[:-1]
    close(lse[:n], r_lse[:n], r_lse_e[:n])
    close(out[:n], r_out[:n], r_out_e[:n])
    if dout is not None:
        for name, got in zip(("dq", "dk", "dv"), train.attention_backward(dout, q, k, v, out, lse, offsets, scale=scale)):
            assert not bool(got[n:].any())
            close(got[:n], g[name][:n], ge[name][:n])


def qkv(lengths, heads, kv, dim, dtype, tail=0, pack=True, seed=0):
    n = sum(lengths) + tail
    parts = [randn(n, h, dim, seed=seed + i).to(dtype) for i, h in enumerate((heads, kv, kv))]
    parts[0] += randn(1, heads, dim, seed=seed + 7).to(dtype)
    parts[1] += randn(1, kv, dim, seed=seed + 8).to(dtype)
    for p in parts:
        p[n - tail:] = float("nan")
    return packed(parts, gap=1) if pack else parts


SHAPES = [
    ([1], 1, 1, 64), ([2], 2, 1, 64), ([128], 1, 1, 128), ([129], 1, 1, 128), ([127, 1, 130], 2, 2, 64), ([300], 4, 1, 128),
    ([1, 40, 7, 3, 1, 22], 8, 2, 64), ([513, 255, 257], 4, 2, 96), ([700], 6, 2, 80), ([65, 0, 66, 0, 0, 1], 3, 1, 128), ([400], 7, 1, 64),
    ([333], 16, 1, 128), ([50, 60], 128, 1, 32), ([1100], 2, 1, 128), ([100], 1, 1, 1), ([90], 2, 1, 7), ([211], 15, 3, 77), ([140], 5, 1, 121),
    ([20] * 60, 4, 4, 64), ([2000, 10], 1, 1, 64), ([130], 100, 1, 64)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("lengths, heads, kv, dim", SHAPES)
def test_attention_forward(lengths, heads, kv, dim, dtype):
    check_attention(*qkv(lengths, heads, kv, dim, dtype), lengths)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("lengths, heads, kv, dim", SHAPES)
def test_attention_backward(lengths, heads, kv, dim, dtype):
    check_attention(*qkv(lengths, heads, kv, dim, dtype), lengths, randn(sum(lengths), heads, dim, seed=11).to(dtype) * 1e-3)


@pytest.mark.parametrize("dim", [64, 128, 77])
@pytest.mark.parametrize("tail", [1, 129, 700])
def test_attention_tokens_of_no_sequence(dim, tail):
    """Whatever lies behind the last sequence, NaN here, reaches nothing, and its own rows are zeros."""
    lengths = [3, 190, 64]
    q, k, v = qkv(lengths, 4, 2, dim, BF16, tail=tail)
    dout = randn(sum(lengths) + tail, 4, dim, seed=5).bfloat16()
    dout[sum(lengths):] = float("nan")
    check_attention(q, k, v, lengths, dout, tail=tail)


def test_attention_sequences_do_not_reach_each_other():
    """NaN and infinities in one sequence leave the bits of the others as they are."""
    from paper_2108_03645_b200 import train
    lengths = [70, 5, 200, 131]
    offsets = torch.tensor([0] + lengths).cumsum(0).cuda()
    for heads, kv, dim in ((4, 2, 128), (3, 1, 64), (2, 2, 50)):
        q, k, v = qkv(lengths, heads, kv, dim, BF16, pack=False)
        dout = randn(sum(lengths), heads, dim, seed=3).bfloat16()
        out, lse = train.attention(q, k, v, offsets)
        want = [out, lse, *train.attention_backward(dout, q, k, v, out, lse, offsets)]
        for value in (float("nan"), float("inf")):
            for sequence in (1, 2):
                rows = slice(int(offsets[sequence]), int(offsets[sequence + 1]))
                args = [t.clone() for t in (q, k, v, dout)]
                for t in args:
                    t[rows] = value
                out, lse = train.attention(*args[:3], offsets)
                got = [out, lse, *train.attention_backward(args[3], *args[:3], out, lse, offsets)]
                keep = torch.ones(sum(lengths), dtype=torch.bool, device="cuda")
                keep[rows] = False
                for a, b in zip(got, want):
                    assert torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("heads, kv, dim", [(3, 1, 64), (4, 2, 128), (5, 1, 128), (7, 1, 64), (15, 3, 77)])
def test_attention_rows_that_are_not_there_have_no_say(heads, kv, dim):
    """Sequences whose rows share a tile with rows of the next one, which is NaN or large, or with none: the output's bits are theirs alone."""
    from paper_2108_03645_b200 import train
    lengths = [70, 300, 5, 331, 129]
    offsets = torch.tensor([0] + lengths).cumsum(0).cuda()
    q, k, v = (3 * t for t in qkv(lengths, heads, kv, dim, BF16, pack=False))
    want = train.attention(q, k, v, offsets)
    for value in (float("nan"), 1e4, -1e4):
        for sequence in range(5):
            rows = slice(int(offsets[sequence]), int(offsets[sequence + 1]))
            args = [t.clone() for t in (q, k, v)]
            for t in args:
                t[rows] = value
            keep = torch.ones(sum(lengths), dtype=torch.bool, device="cuda")
            keep[rows] = False
            for a, b in zip(train.attention(*args, offsets), want):
                assert torch.equal(a[keep], b[keep])


def test_attention_dense_batches_and_offsets_agree():
    from paper_2108_03645_b200 import train
    q, k, v = (randn(3, 150, h, 64, seed=h).bfloat16() for h in (4, 2, 2))
    dout = randn(3, 150, 4, 64, seed=9).bfloat16()
    out, lse = train.attention(q, k, v)
    offsets = torch.arange(4, device="cuda") * 150
    flat = [t.flatten(0, 1) for t in (q, k, v)]
    out2, lse2 = train.attention(*flat, offsets)
    assert torch.equal(out.flatten(0, 1), out2) and torch.equal(lse.flatten(0, 1), lse2)
    a = train.attention_backward(dout, q, k, v, out, lse)
    b = train.attention_backward(dout.flatten(0, 1), *flat, out2, lse2, offsets)
    for x, y in zip(a, b):
        assert torch.equal(x.flatten(0, 1), y)


def test_attention_layouts():
    """Heads before tokens, values apart, broadcast heads: the same results as of plain tensors."""
    from paper_2108_03645_b200 import train
    q, k, v = (randn(200, h, 64, seed=h).bfloat16() for h in (4, 2, 2))
    out, lse = train.attention(q, k, v)
    for f in (lambda t: t.transpose(0, 1).contiguous().transpose(0, 1), lambda t: t.transpose(1, 2).contiguous().transpose(1, 2),
              lambda t: torch.cat([t[:, :, :1], t], 2)[:, :, 1:]):
        assert torch.equal(train.attention(f(q), f(k), f(v))[0], out)
    one = k[:, :1].expand(200, 4, 64)
    assert torch.equal(train.attention(q, one, one)[0], train.attention(q, one.contiguous(), one.contiguous())[0])


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim", [77, 50, 121])
def test_attention_what_lies_between_heads_does_not_matter(dtype, dim):
    """Heads on 16-byte boundaries that end off them: NaN or zeros behind each, and nothing behind the last."""
    from paper_2108_03645_b200 import train
    n, wide = 150, (dim + 7) // 8 * 8
    plain = [randn(n, h, dim, seed=h).to(dtype) for h in (4, 2, 3, 5)]
    plain = [plain[0], plain[1], plain[1] * 0.5, plain[0] * 0.1]
    results = []
    for value in (0.0, float("nan")):
        args = []
        for x in plain:
            buf = torch.full((n * x.shape[1] * wide,), value, dtype=dtype, device="cuda")
            y = buf.as_strided(x.shape, (x.shape[1] * wide, wide, 1))
            y.copy_(x)
            args.append(buf[:buf.numel() - wide + dim].as_strided(x.shape, (x.shape[1] * wide, wide, 1)))
        q, k, v, dout = args
        out, lse = train.attention(q, k, v)
        gap = torch.full((n, 4, wide), value, dtype=dtype, device="cuda")[..., :dim]
        gap.copy_(out)
        results.append([out, lse, *train.attention_backward(dout, q, k, v, gap, lse)])
    for a, b in zip(*results):
        assert torch.equal(a, b)
    check_attention(*plain[:3], [n], plain[3])


def test_attention_offsets_out_of_order_stay_inside():
    """Offsets count as their running maximum within [0, tokens]; what they cover no more is zeros."""
    from paper_2108_03645_b200 import train
    q, k, v = (randn(300, h, 64, seed=h).bfloat16() for h in (2, 1, 1))
    dout = randn(300, 2, 64, seed=4).bfloat16()
    for bad, good in (([-5, 100, 50, 170, 9999], [0, 100, 100, 170, 300]), ([40, 90, 200], [40, 90, 200]), ([7], [7]), ([300, 0], [300, 300]),
                      ([1 << 40, 3], [300, 300]), ([-(1 << 40), 20, 20, 19], [0, 20, 20, 20])):
        a, b = torch.tensor(bad).cuda(), torch.tensor(good).cuda()
        out, lse = train.attention(q, k, v, a)
        out2, lse2 = train.attention(q, k, v, b)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
        cover = torch.zeros(300, dtype=torch.bool, device="cuda")
        cover[good[0]:good[-1]] = True
        assert not bool(out[~cover].any()) and bool((out[cover] != 0).any(2).all())
        for x, y in zip(train.attention_backward(dout, q, k, v, out, lse, a), train.attention_backward(dout, q, k, v, out2, lse2, b)):
            assert torch.equal(x, y) and not bool(x[~cover].any())


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attention_scores_of_all_sizes(dtype):
    """Rows whose maximum climbs from tile to tile, falls, or is met once far away: the output is rescaled, or not."""
    n, d = 900, 64
    q = torch.zeros(n, 1, d, device="cuda")
    q[:, 0, 0] = 8
    k = 0.01 * randn(n, 1, d)
    ramp = torch.linspace(0, 60, n, device="cuda")
    for climb in (ramp, -ramp, torch.where(torch.arange(n, device="cuda") == 400, 50.0, -20.0), 3 * torch.sin(ramp)):
        k[:, 0, 0] = climb
        check_attention(q.to(dtype), k.to(dtype), randn(n, 1, d, seed=1).to(dtype), [n], randn(n, 1, d, seed=2).to(dtype) * 1e-2, scale=0.125)


def test_attention_repeats_its_bits():
    from paper_2108_03645_b200 import train
    lengths = [1500, 30, 700, 1, 257]
    q, k, v = qkv(lengths, 8, 2, 128, BF16)
    dout = randn(sum(lengths), 8, 128, seed=4).bfloat16()
    offsets = torch.tensor([0] + lengths).cumsum(0).cuda()
    first = None
    for _ in range(5):
        out, lse = train.attention(q, k, v, offsets)
        got = [out, lse, *train.attention_backward(dout, q, k, v, out, lse, offsets)]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_attention_gradients_against_differences():
    from paper_2108_03645_b200 import train
    q, k, v = (randn(40, h, 32, seed=h).half() for h in (2, 1, 1))
    c = randn(40, 2, 32, seed=9).half()

    def f(q, k, v):  # the definition, whose differences are those of the formula
        return float((attend64(q, k, v, [40], 32 ** -0.5)[0] * c.double()).sum())
    out, lse = train.attention(q, k, v)
    for at, g in enumerate(train.attention_backward(c, q, k, v, out, lse)):
        for i in (0, 333, 1279):
            side = []
            for s in (1, -1):
                args = [t.clone().double() for t in (q, k, v)]
                args[at].reshape(-1)[i] += s * 1e-4
                side.append(sum(float(x) for x in [_f64(*args, c)]))
            want = (side[0] - side[1]) / 2e-4
            assert abs(want - float(g.reshape(-1)[i])) < 0.01 * (1 + abs(want)), (at, i)


def _f64(q, k, v, c):
    s = torch.einsum("ihd,jkd->hij", q, k) * 32 ** -0.5
    s = s.masked_fill(~torch.ones(40, 40, dtype=torch.bool, device="cuda").tril(), -math.inf)
    return (torch.einsum("hij,jkd->ihd", s.softmax(-1), v) * c.double()).sum()


# ---------------------------------------------------------------- norm and clipping of gradients

def tensors(shapes, seed=0, scale=1e-2):
    return [(randn(*s, seed=seed + i) * scale).to(t) for i, (s, t) in enumerate(shapes)]


MIXED = [((3, 5), F32), ((1000,), BF16), ((0,), F32), ((257, 129), F16), ((), F32), ((40000,), F32), ((7, 0, 2), BF16), ((70001,), BF16)]


def check_clip(gs, limit, out=None, eps=1e-6):
    from paper_2108_03645_b200 import train
    total = math.sqrt(sum(float(g.double().square().sum()) for g in gs))
    assert abs(float(train.gradient_norm(gs)) - total) <= 2.0 ** -22 * total
    keep = [g.clone() for g in gs]
    norm = train.clip_gradients(gs, limit, out=out, eps=eps)
    assert abs(float(norm) - total) <= 2.0 ** -22 * total  # 32 squares in 32 bits, and its own rounding
    f = min(1.0, limit / (total + eps))
    for g, got in zip(keep, out or gs):
        want = g.double() * f
        close(got, want, (U[g.dtype] + 2.0 ** -21) * want.abs() + TINY[g.dtype])
    if out is not None:
        assert all(torch.equal(a, b) for a, b in zip(keep, gs))
    return norm


@pytest.mark.parametrize("limit", [0.0, 0.5, 1e9])
@pytest.mark.parametrize("apart", [False, True])
def test_clip(limit, apart):
    gs = tensors(MIXED)
    check_clip(gs, limit, [torch.full_like(g, float("nan")) for g in gs] if apart else None)


@pytest.mark.parametrize("count", [1, 31, 32, 33, 999, 1000, 1001, 2503])
def test_clip_counts(count):
    gs = [randn(1 + i % 300, seed=i).to((F32, BF16, F16)[i % 3]) for i in range(count)]
    check_clip(gs, 0.25)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_clip_leaves_what_lies_around(dtype):
    """Tensors that start and end on any boundary, side by side; in place, and into tensors on other boundaries."""
    sizes = [1, 2, 3, 5, 8, 15, 16, 17, 100, 4095, 4097, 20000]
    whole = randn(sum(sizes) + 3 * len(sizes), seed=3).to(dtype)
    other = torch.full((whole.numel() + 1,), 7.0, dtype=dtype, device="cuda")
    spans, at = [], 1
    for s in sizes:
        spans.append((at, at + s))
        at += s + 2
    inside = torch.zeros(whole.numel(), dtype=torch.bool, device="cuda")
    for a, b in spans:
        inside[a:b] = True
    keep = whole.clone()
    check_clip([whole[a:b] for a, b in spans], 1.0, [other[a + 1:b + 1] for a, b in spans])
    assert bool((other[1:][~inside] == 7.0).all())
    check_clip([whole[a:b] for a, b in spans], 1.0)
    assert torch.equal(whole[~inside], keep[~inside])


@pytest.mark.parametrize("scale", [1e-30, 1e-23, 1e-19, 1.0, 1e17, 1e25, 3e36])
def test_norm_of_all_sizes(scale):
    """Squares that 32 bits do not hold, beside others and beside zeros."""
    gs = [randn(5000, seed=1) * scale, (randn(333, seed=2) * scale).bfloat16(), torch.zeros(100000, device="cuda")]
    from paper_2108_03645_b200 import train
    total = math.sqrt(sum(float(g.double().square().sum()) for g in gs))
    assert abs(float(train.gradient_norm(gs)) - total) <= 2.0 ** -22 * total
    one = torch.zeros(64, device="cuda")
    one[5], one[40] = 1.0, 1e-30
    assert float(train.gradient_norm([one])) == 1.0


def test_clip_what_is_not_finite():
    from paper_2108_03645_b200 import train
    gs = tensors(MIXED)
    gs[5][17] = float("inf")
    norm = train.clip_gradients(gs, 1.0)
    assert math.isinf(float(norm))
    assert not bool(gs[1].any()) and bool(gs[5][17].isnan()) and int(gs[5].isnan().sum()) == 1  # times 0
    gs = tensors(MIXED)
    gs[1][3] = float("nan")
    assert math.isnan(float(train.clip_gradients(gs, 1.0))) and all(bool(g.isnan().all()) for g in gs)
    z = [torch.zeros(10, device="cuda"), torch.zeros(0, device="cuda")]
    assert float(train.clip_gradients(z, 1.0, eps=0.0)) == 0.0 and not bool(z[0].any())
    assert float(train.gradient_norm([])) == 0.0 and float(train.clip_gradients([], 1.0)) == 0.0


def test_clip_layouts_versions_and_refusals():
    from paper_2108_03645_b200 import train
    g = randn(30, 50).t()
    want = g.clone()
    version = g._version
    norm = train.clip_gradients([g], 1.0)
    assert g._version > version
    close(g, want.double() / (float(norm) + 1e-6), 2.0 ** -21 * want.double().abs())
    a = randn(100)
    for bad in ([a, a], [a[:60], a[50:]], [a, a[3:4]]):
        with pytest.raises(ValueError, match="share"):
            train.clip_gradients(bad, 1.0)
    assert abs(float(train.gradient_norm([a, a])) - math.sqrt(2) * float(a.double().norm())) < 1e-4
    with pytest.raises(ValueError):
        train.clip_gradients([a], 1.0, out=[randn(99)])
    with pytest.raises(ValueError):
        train.clip_gradients([randn(10, 10)[:, :5]], 1.0)
    with pytest.raises(ValueError):
        train.gradient_norm([a, torch.zeros(3)])
    from paper_2108_03645_b200.binding import OnesError
    for limit, eps in ((-1.0, 1e-6), (float("nan"), 1e-6), (1.0, -1.0), (float("inf"), 1e-6)):
        with pytest.raises(OnesError):
            train.clip_gradients([a], limit, eps=eps)
