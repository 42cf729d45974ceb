"""Projections with adapters: infinities in rows and scales, middle vectors at the end of a type's range."""
import pytest

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
INF = float("inf")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rank", [1, 4, 8, 12, 16, 20, 40])
@pytest.mark.parametrize("rows,k,shifted", [(1, 64, False), (20, 64, False), (60, 260, False), (1100, 1100, False), (2100, 2060, False),
                                            (4100, 2600, False), (20, 64, True), (1100, 1100, True)])
def test_an_infinity_in_a_row(tvg, rows, k, shifted, rank, dtype):
    """Positive adapters and weights: a row with an infinity comes out infinite, the others as they were, whatever the rank.  So
    do rows of an adapter whose scale is infinite."""
    import torch
    to = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(rows + rank)
    u = lambda *s: (torch.rand(s, generator=g, device="cuda") + 0.5).to(to)
    x, w, a, b = u(rows, 128), u(k, 128), u(3, rank, 128), u(3, k, rank)
    if shifted:
        room = torch.zeros(x.numel() + 8, dtype=to, device="cuda")
        x = room[1:1 + x.numel()].view(rows, 128).copy_(x)
    index = torch.randint(0, 3, (rows,), generator=g, device="cuda", dtype=torch.int32)
    clean = tvg.linear_lora_fused(x, w, a, b, index)
    assert bool(torch.isfinite(clean).all())
    at = rows * 2 // 3
    x[at, 77] = INF
    y = tvg.linear_lora_fused(x, w, a, b, index)
    keep = torch.arange(rows, device="cuda") != at
    assert bool((y[at] == INF).all()) and torch.equal(y[keep], clean[keep])
    scale = torch.ones(3, device="cuda")
    scale[int(index[at])] = INF
    y = tvg.linear_lora_fused(x, w, a, b, index, scale)
    keep = index != index[at]
    assert bool((y[~keep] == INF).all()) and torch.equal(y[keep], clean[keep])
