"""The operators with axes and with sinks without a GPU: where a session's text goes on."""
import pytest


@pytest.mark.parametrize("n", [1, 90, 100, 101, 102, 150, 195, 196, 197, 690])
def test_text_goes_on_behind_a_picture(n):
    """At the position that a longer prompt gives its text behind the whole picture, or before that where the picture ends early; on one
    axis at the number of tokens."""
    import torch

    from paper_2609_35065_gb300 import prefix_step
    cfg = prefix_step.session()
    at = prefix_step.prompt_positions(cfg, n)
    p = prefix_step.next_position(at)
    assert p.shape == (3, 1) and p.dtype == torch.int32 and p.is_contiguous()
    assert (p == at.max() + 1).all()
    longer = prefix_step.prompt_positions(cfg, n + 1)[:, n]
    if n % 196 == 0 or n % 196 < 100:
        assert (p[:, 0] == longer).all()                # more text, or text behind a whole picture
    flat = prefix_step.prompt_positions(prefix_step.Config(), n)
    assert prefix_step.next_position(flat).tolist() == [n]
