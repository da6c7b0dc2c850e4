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
