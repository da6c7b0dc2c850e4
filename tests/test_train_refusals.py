"""Arguments that the training-step operators refuse, without a device: each is turned into an error before any launch."""
import pytest

from test_train_abi import ALIGN, P, PARAM, _lib  # noqa: F401


@pytest.mark.parametrize("m,n", [(200, 200), (64, 64), (64, 4000)])
@pytest.mark.parametrize("steps", [1025, 1 << 29, (1 << 31) - 1])
def test_orthogonalize_refuses_steps_without_end(m, n, steps):
    assert _lib().ones_orthogonalize(P, n, m * n, 1, m, n, 0, steps, 3.4445, -4.775, 2.0315, 1e-7, P, P, 1 << 24, None) == PARAM


def test_functions_outside_the_graph_refuse_what_asks_for_a_gradient():
    torch = pytest.importorskip("torch")
    from paper_2108_03645_b200 import train
    x = torch.zeros(4, 8)
    for f, args in ((train.layer_norm, (x,)), (train.linear_cross_entropy, (x.bfloat16(), x.bfloat16(), torch.zeros(4, dtype=torch.int64))),
                    (train.orthogonalize, (x,))):
        with pytest.raises(ValueError, match="CUDA"):
            f(*args)
        with pytest.raises(ValueError, match="no_grad"):
            f(args[0].clone().requires_grad_(), *args[1:])
        with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):
            f(args[0].clone().requires_grad_(), *args[1:])


@pytest.mark.parametrize("rows", [(1 << 31) - (1 << 16) + 1, (1 << 31) - 1])
@pytest.mark.parametrize("cols", [1, 8, 300])
def test_layer_norm_refuses_more_rows_than_it_counts(rows, cols):
    L = _lib()
    assert L.ones_layer_norm(P, cols, None, None, rows, cols, 1e-5, 1, 1, P, cols, P, P, None) == PARAM
    assert L.ones_layer_norm_workspace_bytes(rows, cols) == 0
    assert L.ones_layer_norm_backward(P, cols, P, cols, P, P, None, rows, cols, 1, 0, P, cols, P, P, P, 1 << 30, None) == PARAM


@pytest.mark.parametrize("change", [{"t": P + 4}, {"loss": P + 2}, {"lse": P + 1}])
def test_linear_ce_refuses_elements_off_their_alignment(change):
    a = dict(h=P, ldh=64, w=P, ldw=64, t=P, loss=P, lse=P) | change
    assert _lib().ones_linear_ce(a["h"], a["ldh"], a["w"], a["ldw"], a["t"], 4, 64, 100, 1, a["loss"], a["lse"], P, 1 << 20, None) == ALIGN


@pytest.mark.parametrize("change", [{"g": P + 2}, {"t": P + 4}, {"lse": P + 2}])
def test_linear_ce_backward_refuses_elements_off_their_alignment(change):
    a = dict(g=P, t=P, lse=P) | change
    assert _lib().ones_linear_ce_backward(a["g"], P, 64, P, 64, a["t"], a["lse"], 4, 64, 100, 1, 1, 0, P, 64, P, 64, P, 1 << 24, None) == ALIGN


@pytest.mark.parametrize("change", [{"mean": P + 2}, {"rstd": P + 3}])
def test_layer_norm_refuses_statistics_off_their_alignment(change):
    a = dict(mean=P, rstd=P) | change
    L = _lib()
    assert L.ones_layer_norm(P, 64, P, P, 4, 64, 1e-5, 0, 0, P, 64, a["mean"], a["rstd"], None) == ALIGN
    assert L.ones_layer_norm_backward(P, 64, P, 64, a["mean"], a["rstd"], P, 4, 64, 0, 0, P, 64, P, P, P, 1 << 20, None) == ALIGN


def test_profile_runs_and_checks_on_the_jobs_device(monkeypatch):
    """Events and the status of the waits are of the current device: the job's, whichever is current at the call."""
    torch = pytest.importorskip("torch")
    from paper_2108_03645_b200 import profile_job, train
    current, seen = [0], []

    class Device:
        def __init__(self, device):
            self.index = device if device is None or isinstance(device, int) else torch.device(device).index

        def __enter__(self):
            self.before = current[0]
            current[0] = self.before if self.index is None else self.index

        def __exit__(self, *a):
            current[0] = self.before

    class Event:
        def __init__(self, enable_timing):
            pass

        def record(self):
            seen.append(("record", current[0]))

        def synchronize(self):
            pass

        def elapsed_time(self, other):
            return 1.0

    class Status:
        def ones_train_status(self, stream):
            seen.append(("status", current[0]))
            return 0

    class Job:
        device = torch.device("cuda:1")

        def batch(self, samples, seed):
            return ()

        def step(self):
            seen.append(("step", current[0]))

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: type("S", (), {"cuda_stream": 0})())
    monkeypatch.setattr(train, "lib", Status)
    assert profile_job.profile(Job(), [8], steps=2, warmup=1) == [0.0005]
    assert {name for name, _ in seen} == {"record", "status", "step"} and {index for _, index in seen} == {1}
    seen.clear()
    train.check("cuda:2"), train.check()
    assert seen == [("status", 2), ("status", 0)]
