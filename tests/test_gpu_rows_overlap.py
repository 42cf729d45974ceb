"""A projection added to its own rows in place is refused; beside them, and over another residual, it is not."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 30, 1100])
def test_in_place_over_x(tvg, rows):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows)
    r = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    x, w = r(2 * rows, 1024), r(1024, 1024) * 1024 ** -0.5
    first, second = x[:rows], x[rows:]
    with pytest.raises(tvg.TvgError):
        tvg.linear_lora_fused(first, w, None, None, None, residual=first, out=first)
    want = tvg.linear_lora_fused(first, w, None, None, None, residual=first)
    # the rows right behind x, a residual right behind x
    assert torch.equal(tvg.linear_lora_fused(first, w, None, None, None, residual=first, out=second), want)
    second.copy_(first)
    assert torch.equal(tvg.linear_lora_fused(first, w, None, None, None, residual=second, out=second), want)
