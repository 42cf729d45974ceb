"""Group norm of maps whose mean is so large that its square is beyond fp32."""
import pytest

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,groups", [((2, 7, 7, 64), 8), ((1, 300, 300, 64), 32), ((1, 700, 5000), 8), ((1, 23, 5001), 1), ((2, 190, 200, 36), 4)],
                         ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else str(v))
def test_a_mean_whose_square_is_beyond_fp32(tvg, shape, groups, dtype):
    """2.5e19 everywhere, its neighbour in the type in a few places: distances and their squares are ordinary numbers."""
    import torch
    to = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.full(shape, 2.5e19, device="cuda").to(to)
    step = 2.0 ** 57 if dtype == "bf16" else 2.0 ** 49
    flat = x.view(shape[0], -1, shape[-1])
    flat[:, 3, ::3] = (flat[:, 3, ::3].double() + step).to(to)
    y, mean, rstd = tvg.group_norm_fused(x, groups, activation=None, stats=True)
    v = x.double().view(shape[0], -1, groups, shape[-1] // groups)
    m = v.mean(dim=(1, 3))
    r = (((v - m.view(shape[0], 1, groups, 1)) ** 2).mean(dim=(1, 3)) + 1e-5) ** -0.5
    # the mean: 64 roundings of numbers no larger than the largest; its error counts in every distance and, squared, in the variance
    dm = 64 * H * v.abs().amax(dim=(1, 3))
    assert bool(((mean.double() - m).abs() <= dm).all())
    assert bool(torch.isfinite(rstd).all()) and bool((rstd > 0).all())
    low, high = ((1 / r ** 2) * (1 - 144 * H)), ((1 / r ** 2) * (1 + 144 * H) + dm ** 2)
    var = rstd.double() ** -2
    assert bool((var >= low * (1 - 4 * H)).all()) and bool((var <= high * (1 + 4 * H)).all())
    want = (v - mean.double().view(shape[0], 1, groups, 1)) * rstd.double().view(shape[0], 1, groups, 1)
    assert bool(((y.double().view(v.shape) - want).abs() <= (4 * H + HALF[dtype]) * want.abs() + 1e-37).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pixels", [49, 40000])
def test_gradients_of_constant_groups_whose_rstd_has_an_infinite_square(tvg, pixels, dtype):
    """x is the mean everywhere and rstd 1e20, as of eps 1e-40: dx is rstd (gamma dz - a), a group's mean of gamma dz, in fewer than 200 roundings of
    the terms (dy is +-1, +-2 or +-3, whose sums are exact; gamma rounds the rest)."""
    import torch
    to = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(pixels)
    x = torch.full((2, pixels, 64), 1.5, dtype=to, device="cuda")
    dy = torch.randint(1, 4, x.shape, generator=g, device="cuda") * (torch.randint(0, 2, x.shape, generator=g, device="cuda") * 2 - 1)
    dy, gamma, beta = dy.to(to), torch.rand(64, generator=g, device="cuda") + 0.5, torch.zeros(64, device="cuda")
    mean, rstd = torch.full((2, 8), 1.5, device="cuda"), torch.full((2, 8), 1e20, device="cuda")
    dx, dgamma, dbeta = tvg.group_norm_fused_backward(x, dy, mean, rstd, 8, gamma, beta)
    dz = (dy.double() * gamma.double()).view(2, pixels, 8, 8)
    a, r = dz.mean(dim=(1, 3), keepdim=True), rstd.double().view(2, 1, 8, 1)
    size = r * (dz.abs() + dz.abs().mean(dim=(1, 3), keepdim=True))
    want = r * (dz - a)
    assert bool(((dx.double().view(want.shape) - want).abs() <= 200 * H * size + HALF[dtype] * want.abs()).all())
    assert bool((dgamma == 0).all()) and torch.equal(dbeta.double(), dy.double().sum((0, 1)))
