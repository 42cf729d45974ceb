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


@pytest.mark.parametrize("rows,k", [(1, 64), (60, 260), (1100, 1100)])
def test_a_middle_vector_between_the_largest_numbers_of_bf16_and_of_fp32(tvg, rows, k):
    """h = 1.003 times bf16's largest number, which fp32 holds and bf16 rounds to infinity; y = h / 2^20.  The sum of both parts is
    within 2^-17 of h, y rounds once."""
    import torch
    x = torch.zeros((rows, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((k, 64), dtype=torch.bfloat16, device="cuda")
    x[:, 5] = torch.finfo(torch.bfloat16).max
    a, b = torch.zeros((2, 16, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, k, 16), dtype=torch.bfloat16, device="cuda")
    a[1, 3, 5], b[1, :, 3] = 1, 2.0 ** -20
    for sign in (1.0, -1.0):
        scale = torch.tensor([1.0, sign * 1.003], device="cuda")
        y = tvg.linear_lora_fused(x, w, a, b, torch.ones(rows, dtype=torch.int32, device="cuda"), scale)
        want = float(scale[1]) * torch.finfo(torch.bfloat16).max * 2.0 ** -20
        assert bool(((y.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -17 + 4 * H) * abs(want)).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k,shifted", [(1, 64, False), (20, 64, False), (60, 260, False), (1100, 1100, False), (2100, 2060, False),
                                            (4100, 2600, False), (1100, 1100, True)])
def test_an_infinity_in_b(tvg, rows, k, shifted, dtype):
    """One channel of one adapter: infinite in its rows in fp32, infinite or not a number in bf16, and nothing else changes."""
    import torch
    to = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(rows)
    u = lambda *s: (torch.rand(s, generator=g, device="cuda") + 0.5).to(to)
    x, w, a, b = u(rows, 128), u(k, 128), u(3, 12, 128), u(3, k, 12)
    if shifted:
        room = torch.zeros(b.numel() + 8, dtype=to, device="cuda")
        b = room[1:1 + b.numel()].view(b.shape).copy_(b)
        room = torch.zeros(x.numel() + 8, dtype=to, device="cuda")
        x = room[1:1 + x.numel()].view(x.shape).copy_(x)
    index = torch.randint(0, 3, (rows,), generator=g, device="cuda", dtype=torch.int32)
    clean = tvg.linear_lora_fused(x, w, a, b, index)
    b[int(index[0]), k // 2, 7] = INF
    y = tvg.linear_lora_fused(x, w, a, b, index)
    hit = torch.zeros(y.shape, dtype=torch.bool, device="cuda")
    hit[index == index[0], k // 2] = True
    assert bool((y[hit] == INF).all()) if dtype == "f32" else not bool(torch.isfinite(y[hit]).any())
    assert torch.equal(y[~hit], clean[~hit])
