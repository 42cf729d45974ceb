"""A projection whose output lies over its rows is refused on the host, before any launch."""
import pytest

import paper_1802_04799_amd as tvg


@pytest.mark.parametrize("dtype,size", [(tvg.TVG_BF16, 2), (tvg.TVG_F32, 4)])
def test_y_over_x_is_refused(dtype, size):
    d = tvg.LinearLoraDesc(8, 64, 96, 4, 16, dtype, 0, 0)
    need = tvg.tvg_linear_lora_workspace_size(d)
    x, w, a, b, other, ws = 0x100000, 0x200000, 0x300000, 0x400000, 0x500000, 0x600000
    # all of it, its last element, from before it into its first; with x as the residual, with another, without one
    for y in (x, x + (8 * 64 - 1) * size, x - (8 * 96 - 1) * size):
        for residual in (x, other, None):
            assert tvg.tvg_linear_lora_fused(d, x, w, a, b, other, None, None, residual, y, ws, need, 0) == 3
    # without adapters too
    d = tvg.LinearLoraDesc(8, 64, 64, 0, 1, dtype, 0, 0)
    need = tvg.tvg_linear_lora_workspace_size(d)
    assert tvg.tvg_linear_lora_fused(d, x, w, None, None, None, None, None, x, x, ws, need, 0) == 3
