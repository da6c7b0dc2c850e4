"""What the attention layer's operators do at the ends of their range, without a device: index arithmetic, gradients that there are none of."""
import pytest


@pytest.mark.parametrize("group", [1, 2, 3, 77, 128])
def test_rows_that_see_a_key_far_away(group):
    """Tokens times heads of a group pass 32 bits in long sequences: a key far before a tile's queries is seen by all of them."""
    from paper_2108_03645_b200 import train
    first_row = train.lib().ones_attention_first_row
    far = [-(1 << 30) + 1, -(1 << 31) // group - 40, -(1 << 24) - 3, -(1 << 20)]
    for behind in [*(b for b in far if b > -(1 << 30)), *range(-300, 260)]:
        for lane in (0, 1, 31):  # keys of a warp, one behind the other
            got, exact = first_row(behind, group) + lane * group, (behind + lane) * group
            for row in (0, 1, 31, 32, 63, 64, 96, 127):
                assert (row >= got) == (row >= exact), (behind, lane, row)


def test_gradients_of_frequencies_are_refused():
    """There are none, and whoever asks is told so, before any launch."""
    torch = pytest.importorskip("torch")
    from paper_2108_03645_b200 import train
    q, k = torch.zeros(4, 2, 64), torch.zeros(4, 1, 64)
    freq = train.rotary_frequencies(64, device="cpu").requires_grad_()
    for x in (q, q.clone().requires_grad_()):
        with pytest.raises(ValueError, match="frequencies"):
            train.qk_norm_autograd(x, k, torch.arange(4), freq)
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):
        train.qk_norm_autograd(q, k, torch.arange(4), freq)


def test_job_shapes_that_no_step_takes_are_refused():
    """What the operators refuse is no shape of a job: it fails when it is made, not at its first step."""
    from paper_2108_03645_b200 import profile_job as pj
    for bad in (dict(clip=float("inf")), dict(width=4096, heads=256, kv_heads=1), dict(width=4096, heads=2048)):
        with pytest.raises(ValueError):
            pj.JobShape(**bad)
    assert pj.JobShape(width=4096, heads=128, kv_heads=1, clip=1e30).heads == 128


def test_backward_workspace_holds_no_copy_of_the_inputs():
    """A few bytes for each row of each head, whatever the type, however long the vectors are."""
    from paper_2108_03645_b200 import train
    need = train.lib().ones_attention_backward_workspace_bytes
    tokens, heads = 65536, 32
    assert 4 * tokens * heads < need(tokens, 8, heads, heads, 128) < 9 * tokens * heads
