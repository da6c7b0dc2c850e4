"""The attention layer's operators as they are used together: in the profiled job's step, in captured graphs, on streams of the
caller's, in many small sequences, and with gradients through automatic differentiation."""
import ctypes as C
import json
import math

import pytest

torch = pytest.importorskip("torch")


def test_job_shapes_are_checked():
    from paper_2108_03645_b200 import profile_job as pj
    assert pj.JobShape(heads=16, kv_heads=4).kv_heads == 4
    for bad in (dict(heads=3), dict(heads=16, kv_heads=5), dict(heads=-1), dict(heads=4), dict(clip=-1.0), dict(clip=float("nan")), dict(heads=8, kv_heads=-2)):
        with pytest.raises(ValueError):
            pj.JobShape(**bad)


def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.fixture
def checked():
    _gpu()
    yield
    from paper_2108_03645_b200 import train
    train.check()


def randn(*size, seed=0):
    return torch.randn(size, generator=torch.Generator(device="cuda").manual_seed(seed + 1), device="cuda")


def _rms(x, w, eps=1e-6):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * w


@pytest.mark.gpu
@pytest.mark.parametrize("heads, kv", [(4, 0), (8, 2), (2, 1)])
def test_job_with_attention(heads, kv, checked):
    """The step's gradients against automatic differentiation of the plain model in 32 bits; two steps run, the second from other
    weights; clipping scales the gradients and nothing else."""
    from paper_2108_03645_b200 import profile_job as pj
    shape = pj.JobShape(width=128, inner=512, vocab=500, seq=48, heads=heads, kv_heads=kv)
    job = pj.LanguageModelJob(shape)
    token, target = job.batch(6, 0)
    loss, grads = job.gradients(token, target)
    names = ("w1", "w2", "head", "gain", "shift", "wqkv", "wo", "q_gain", "k_gain")
    p = {n: getattr(job, n).detach().float().requires_grad_() for n in names}
    d, kvh, n = job.head_dim, job.kv_heads, token.numel()
    x = job.embedding[token].float()
    q, k, v = (x @ p["wqkv"]).view(6, 48, heads + 2 * kvh, d).split([heads, kvh, kvh], 2)
    a = (torch.arange(48, device="cuda").double()[:, None] * job.frequencies).float()
    cos, sin = a.cos()[:, None], a.sin()[:, None]

    def turn(t):
        l, r = t[..., :d // 2], t[..., d // 2:]
        return torch.cat([l * cos - r * sin, r * cos + l * sin], -1)
    q, k = turn(_rms(q, p["q_gain"])), turn(_rms(k, p["k_gain"]))
    s = torch.einsum("bihd,bjhd->bhij", q, k.repeat_interleave(heads // kvh, 2)) * d ** -0.5
    s = s.masked_fill(~torch.ones(48, 48, dtype=torch.bool, device="cuda").tril(), -math.inf).softmax(-1)
    y = x + torch.einsum("bhij,bjhd->bihd", s, v.repeat_interleave(heads // kvh, 2)).reshape(n, -1) @ p["wo"]
    z = y + torch.nn.functional.gelu(y @ p["w1"]) @ p["w2"]
    ref = torch.nn.functional.cross_entropy(torch.nn.functional.layer_norm(z, (128,), p["gain"], p["shift"]) @ p["head"].t(), target, ignore_index=-100)
    ref.backward()
    assert abs(float(loss) - float(ref.detach())) <= 0.02 * float(ref.detach())
    for name, got in zip(names, grads):
        # a chain of at most ten roundings to bfloat16, each off by 2^-9 of the norm in the mean and 2^-8 at most
        assert float((got.float() - p[name].grad).norm()) <= 0.05 * float(p[name].grad.norm()), name
    for _ in range(2):
        assert math.isfinite(float(job.step(token, target)))
    plain, clipped = pj.LanguageModelJob(shape), pj.LanguageModelJob(pj.JobShape(**{**shape.__dict__, "clip": 1e-3}))
    total = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    assert total > 2e-3
    plain.step(token, target), clipped.step(token, target)
    for a, b in zip(plain.momentum, clipped.momentum):
        assert float((b - a * (1e-3 / total)).norm()) <= 2.0 ** -7 * float(b.norm())


@pytest.mark.gpu
def test_job_without_attention_is_as_it_was(checked):
    from paper_2108_03645_b200 import profile_job as pj
    job = pj.LanguageModelJob(pj.JobShape(width=128, inner=512, vocab=500, seq=32))
    assert len(job.gradients(*job.batch(4, 0))[1]) == 5 and len(job.matrices) == 2


@pytest.mark.gpu
def test_profile_command_with_attention(checked, capsys):
    from paper_2108_03645_b200 import profile_job as pj
    out = pj.main(["--b0", "4", "--kmax", "2", "--width", "128", "--vocab", "1000", "--seq", "40", "--generations", "5", "--heads", "4", "--kv-heads",
                   "2", "--clip", "1.0"])
    assert len(out["seconds"]) == 3 and all(t > 0 for t in out["seconds"])
    assert json.loads(capsys.readouterr().out)["batches"] == [4, 8, 16]


@pytest.mark.gpu
def test_automatic_differentiation(checked):
    """The two functions with a graph against those without, through a shared leaf, and what they refuse."""
    from paper_2108_03645_b200 import train
    x = randn(90, 6, 64).bfloat16().requires_grad_()
    w = (1 + 0.1 * randn(64, seed=1)).requires_grad_()
    pos, freq = torch.arange(90, device="cuda"), train.rotary_frequencies(64)
    offsets = torch.tensor([0, 50, 90], device="cuda")
    c = randn(90, 4, 64, seed=2).bfloat16()

    def run():
        q, k = train.qk_norm_autograd(x[:, :4], x[:, 4:5], pos, freq, w, w)
        return train.attention_autograd(q, k, x[:, 5:], offsets)
    out = run()
    out.backward(c)
    with torch.no_grad():
        q, k = train.qk_norm(x[:, :4], x[:, 4:5], pos, freq, w, w)
        o, lse = train.attention(q, k, x[:, 5:], offsets)
        assert torch.equal(o, out)
        dq, dk, dv = train.attention_backward(c, q, k, x[:, 5:], o, lse, offsets)
        dq, dk, a, b = train.qk_norm_backward(dq, dk, x[:, :4], x[:, 4:5], pos, freq, w, w)
    assert torch.equal(x.grad, torch.cat([dq, dk, dv], 1)) and torch.equal(w.grad, a + b)
    only_q = train.qk_norm_autograd(x[:, :4], x[:, 4:5], pos, freq)[0]  # the other result has no gradient
    (g,) = torch.autograd.grad(only_q, x, torch.ones_like(only_q))
    assert not bool(g[:, 4:].any()) and bool(g[:, :4].any())
    with pytest.raises(RuntimeError):
        out = run()
        (g,) = torch.autograd.grad(out, x, c, create_graph=True)
        g.sum().backward()


@pytest.mark.gpu
def test_captured_steps_follow_their_inputs(checked):
    """Two graphs with the operators' forward and backward passes and the clipping, replayed in turn with other values and other bounds of
    the sequences, beside eager calls between them."""
    from paper_2108_03645_b200 import train
    n = 300
    pos, freq = torch.arange(n, device="cuda"), train.rotary_frequencies(64)

    def inputs(seed):
        return [randn(n, h, 64, seed=seed + h).bfloat16() for h in (4, 2, 3, 5)]  # q, k, v (two of three heads), dout (four of five)

    def step(q, k, v, dout, offsets):
        qn, kn = train.qk_norm(q, k, pos, freq)
        out, lse = train.attention(qn, kn, v[:, :2], offsets)
        dq, dk, dv = train.attention_backward(dout[:, :4], qn, kn, v[:, :2], out, lse, offsets)
        dq, dk, _, _ = train.qk_norm_backward(dq, dk, q, k, pos, freq)
        grads = [dq, dk, dv]
        norm = train.clip_gradients(grads, 0.5)
        return [out, lse, *grads, norm]

    bounds = [torch.tensor(b, device="cuda") for b in ([0, 100, 300], [0, 1, 250], [30, 30, 299], [0, 300, 300])]
    states, graphs = [], []
    side = torch.cuda.Stream()
    for i in range(2):
        state = [*inputs(i), bounds[i].clone()]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(*state)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(*state)
        states.append((state, out))
        graphs.append(graph)
    for turn in range(4):
        want = []
        for i in range(2):
            fresh = [*inputs(10 * turn + i), bounds[(turn + i) % 4]]
            for to, x in zip(states[i][0], fresh):
                to.copy_(x)
            want.append(fresh)
        graphs[1].replay()
        graphs[0].replay()
        for i in (0, 1):
            for a, b in zip(states[i][1], step(*want[i])):
                assert torch.equal(a, b)


@pytest.mark.gpu
def test_two_streams_at_once(checked):
    from paper_2108_03645_b200 import train
    offsets = torch.tensor([0, 700, 900, 1500], device="cuda")
    data = [[randn(1500, h, 128, seed=7 * s + h).bfloat16() for h in (4, 2, 2, 4)] for s in range(2)]

    def step(q, k, v, dout):
        out, lse = train.attention(q, k, v, offsets)
        return [out, lse, *train.attention_backward(dout, q, k, v, out, lse, offsets)]
    want = [step(*d) for d in data]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(step(*data[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[i]))


@pytest.mark.gpu
@pytest.mark.parametrize("dim, heads, kv", [(64, 16, 16), (128, 8, 8), (64, 2, 1)])
def test_many_short_sequences(dim, heads, kv, checked):
    """More items for a block than it lists at once; against the definition in 64 bits, by norms: each of three roundings to bfloat16 is off
    by at most 2^-8 of its value."""
    from paper_2108_03645_b200 import train
    b, n = 6000, 3
    q, k, v, dout = (randn(b, n, h, dim, seed=h + i).bfloat16() for i, h in enumerate((heads, kv, kv, heads)))
    out, lse = train.attention(q, k, v)
    grads = train.attention_backward(dout, q, k, v, out, lse)
    t = heads // kv
    x = [a.double().requires_grad_() for a in (q, k, v)]
    s = torch.einsum("bihd,bjhd->bhij", x[0], x[1].repeat_interleave(t, 2)) * dim ** -0.5
    s = s.masked_fill(~torch.ones(n, n, dtype=torch.bool, device="cuda").tril(), -math.inf)
    o = torch.einsum("bhij,bjhd->bihd", s.softmax(-1), x[2].repeat_interleave(t, 2))
    want = torch.autograd.grad(o, x, dout.double())
    assert float((lse.double() - s.detach().logsumexp(-1).transpose(1, 2)).abs().max()) < 1e-5
    for a, c in zip((out, *grads), (o.detach(), *want)):
        assert float((a.double() - c).norm()) <= 3 * 2.0 ** -8 * float(c.norm())


@pytest.mark.gpu
@pytest.mark.parametrize("first", ["zero", "small", "large"])
def test_first_token_says_nothing_of_the_others(first, checked):
    """Queries and keys of the first token are zeros, or a millionth or a million of the others': the gradients are as exact."""
    from paper_2108_03645_b200 import train
    n, f = 400, {"zero": 0.0, "small": 1e-6, "large": 1e6}[first]
    q, k, v, dout = (randn(n, h, 64, seed=h + i) for i, h in enumerate((4, 2, 2, 4)))
    q[0] *= f
    k[0] *= f if f < 1 else 1.0
    q, k, v, dout = (t.bfloat16() for t in (q, k, v, dout))
    offsets = torch.tensor([0, 1, n], device="cuda")  # a sequence of its own
    out, lse = train.attention(q, k, v, offsets)
    got = train.attention_backward(dout, q, k, v, out, lse, offsets)
    x = [t[1:].double().requires_grad_() for t in (q, k, v)]
    s = torch.einsum("ihd,jhd->hij", x[0], x[1].repeat_interleave(2, 1)) * 0.125
    s = s.masked_fill(~torch.ones(n - 1, n - 1, dtype=torch.bool, device="cuda").tril(), -math.inf).softmax(-1)
    want = torch.autograd.grad(torch.einsum("hij,jhd->ihd", s, x[2].repeat_interleave(2, 1)), x, dout[1:].double())
    for a, c in zip(got, want):
        assert float((a[1:].double() - c).norm()) <= 2 * 2.0 ** -8 * float(c.norm())


@pytest.mark.gpu
def test_waits_of_the_attention_end():
    """A kernel of each of its files that waits for what nobody sends gives up, and the next status says so, once."""
    _gpu()
    from paper_2108_03645_b200 import train
    from paper_2108_03645_b200.binding import OnesError
    L = train.lib()
    assert L.ones_train_wait_limit(C.c_ulonglong(20_000_000)) == 0
    try:
        for which in (3, 4):
            assert L.ones_train_wait_for_nothing(which, 100, C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
            with pytest.raises(OnesError):
                train.check()
            train.check()
        assert L.ones_train_wait_for_nothing(5, 1, None) == -3
    finally:
        assert L.ones_train_wait_limit(C.c_ulonglong(0)) == 0
