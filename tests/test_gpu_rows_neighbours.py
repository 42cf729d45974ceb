"""A row of a projection with adapters keeps its bits whatever adapters the other rows of the call have: which, how many and in
what order.  (What the adapters of the others hold is tested beside the projection.)"""
import pytest

pytestmark = pytest.mark.gpu


def others(rows, keep, own, adapters):
    """Adapters of all rows but `keep`: none, one, every row another, backwards, chance."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows)
    t = torch.arange(rows, device="cuda", dtype=torch.int32)
    chance = lambda: torch.randint(-1, adapters, (rows,), generator=g, device="cuda", dtype=torch.int32)
    for index in (t * 0 - 1, t * 0 + 3, t % adapters, (rows - 1 - t) % adapters, chance(), chance(), chance()):
        yield torch.where(keep, own, index).contiguous()


# parts of 16, 32 and 64 rows, the ring's tiles of 64, 128 and 256 rows (bf16); shifted: operands at any element, few tiles and many
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rank", [5, 16, 64, 200])
@pytest.mark.parametrize("rows,k,shifted", [(6, 264, False), (16, 264, False), (30, 264, False), (50, 264, False), (64, 520, False),
                                            (300, 264, False), (1100, 1100, False), (2100, 2060, False), (4100, 2600, False),
                                            (6, 264, True), (64, 264, True), (1100, 1100, True)])
def test_a_row_does_not_see_which_adapters_the_others_have(tvg, rows, k, shifted, rank, dtype):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows + rank)
    to = torch.bfloat16 if dtype == "bf16" else torch.float32
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    c, adapters = 256, 12
    x, w = r(rows, c).to(to), (r(k, c) * c ** -0.5).to(to)
    a, b = (r(adapters, rank, c) * c ** -0.5).to(to), (r(adapters, k, rank) * rank ** -0.5).to(to)
    if shifted:
        room = torch.zeros(x.numel() + 8, dtype=to, device="cuda")
        x = room[1:1 + x.numel()].view(rows, c).copy_(x)
    keep = torch.arange(rows, device="cuda") % 5 == 2
    own = torch.randint(0, adapters, (rows,), generator=g, device="cuda", dtype=torch.int32)
    want = None
    for index in others(rows, keep, own, adapters):
        y = tvg.linear_lora_fused(x, w, a, b, index)[keep]
        want = y if want is None else want
        assert torch.equal(y, want)
