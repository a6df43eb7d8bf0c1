"""What RefreshLoop refuses of a policy before anything runs (no GPU is needed)."""
import pytest
import torch

from paper_2607_27600_amd.refresh import Model, RefreshLoop, run_stream


def _model():
    return Model(mode="last_layer", n_layers=1, n_heads_q=4, n_heads_kv=2, head_dim=64, hidden=64, vocab=8,
                 w_lm=torch.zeros(8, 64, dtype=torch.bfloat16), w_o=torch.zeros(64, 256, dtype=torch.bfloat16))


@pytest.mark.parametrize("J,recent", [(4, 5), (4, 8), (1, 2)])
def test_more_recent_entries_than_are_kept(J, recent):
    """All of them would score alike and the oldest of them stay."""
    with pytest.raises(ValueError, match="n_recent"):
        RefreshLoop(_model(), J, 4, device="cpu", policy="weight", n_recent=recent)
    assert RefreshLoop(_model(), J, 4, device="cpu", policy="weight", n_recent=J).n_recent == J


def test_a_stream_without_queries():
    """Without attention every weight is 0, and a refresh would keep the first entries whatever came."""
    loop, calls = RefreshLoop(_model(), 4, 4, device="cpu", policy="weight"), []
    for chunked in (True, False):
        with pytest.raises(ValueError, match="policy weight"):
            run_stream(loop, lambda t0, t1: calls.append((t0, t1)), 3, 5, chunked=chunked)
    assert not calls and loop.n == 0
