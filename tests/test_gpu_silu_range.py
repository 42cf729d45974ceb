"""SiLU of the channels-last operators far from zero.

Tolerances in half steps H = 2^-24 of fp32, counted before any run.  SiLU in fp32: exp2 and the reciprocal two each (one step), the
correction, the sum, the product with the reciprocal and with z one each: 8.  Below 2^-126 a number has steps of 2^-149: half of
one in exp(-|z|), which z multiplies, and half of one in the result."""
import pytest

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
INF, NAN = float("inf"), float("nan")


def far(dtype):
    """Values of the type far from zero and near it, the infinities last."""
    import torch
    to = torch.bfloat16 if dtype == "bf16" else torch.float32
    some = [1e3, 1e4, 12345.0, 2.0 ** 23, 2.0 ** 24, 1e7, 1e30, 1e37, 1e38, 2.35e38, 2.4e38, 3e38, 3.38e38, 20.0, 16.5, 17.5, 60.0, 44.0, 45.0]
    near = [0.0, 1e-30, 0.5, 1.0, 1.278, 2.4, 5.0, 9.0]
    near_end = [86.0, 87.0, 87.25, 87.5, 88.0, 88.5, 89.0, 90.0, 95.0, 100.0, 103.0, 103.5, 104.0, 105.0, 150.0]
    v = some + near + near_end
    v = v + [-t for t in v] + [INF, -INF, NAN]
    return torch.tensor(v + [0.25] * (96 - len(v)), device="cuda").to(to).float()


def silu64(z):
    import torch
    z = z.double()
    return z / (1 + torch.exp(-z))


def silu_bound(want, z, dtype):
    # (bf16 forms: the reciprocal of exp(-z) is zero where it would be below 2^-126)
    return 8 * H * want.abs() + (z.double().abs() + 1) * (2.0 ** -149 if dtype == "f32" else 2.0 ** -125)


def same_or_within(got, want, bound):
    """Not a number where the formula says so, the infinity that it says, and within the bound elsewhere."""
    import torch
    got, want = got.double(), want.double()
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), (got[torch.isnan(got) != torch.isnan(want)], want[torch.isnan(got) != torch.isnan(want)])
    assert torch.equal(got[want.isinf()], want[want.isinf()])
    err = (got - want).abs()[finite]
    assert bool((err <= bound[finite]).all()), (float((err / bound[finite]).max()), want[finite][(err / bound[finite]).argmax()])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pixels", [49, 40000])
def test_silu_of_a_norm(tvg, pixels, dtype):
    """A map of zeros: z is beta, in one launch and in two."""
    import torch
    z = far(dtype)
    x = torch.zeros((2, pixels, 96), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    y = tvg.group_norm_fused(x, 8, None, z, activation="silu")
    want = silu64(z)
    same_or_within(y[1, pixels // 2], want, silu_bound(want, z, dtype) + HALF[dtype] * want.abs())
    assert torch.equal(y.view(-1, 96)[::7].nan_to_num(7), y[0, 0].nan_to_num(7).expand(y.view(-1, 96)[::7].shape))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k", [(3, 96), (1100, 1152), (2100, 2112), (4100, 2688)])
def test_silu_of_a_projection(tvg, rows, k, dtype):
    """Rows of zeros: z is the residual, or the bias."""
    import torch
    to = torch.bfloat16 if dtype == "bf16" else torch.float32
    z = far(dtype).repeat(k // 96)
    x, w = torch.zeros((rows, 64), dtype=to, device="cuda"), torch.zeros((k, 64), dtype=to, device="cuda")
    want = silu64(z)
    bound = silu_bound(want, z, dtype) + HALF[dtype] * want.abs()
    for kw in (dict(bias=z), dict(residual=z.to(to).expand(rows, k).contiguous())):
        y = tvg.linear_lora_fused(x, w, None, None, None, activation="silu", **kw)
        same_or_within(y[rows - 1], want, bound)
        assert torch.equal(y.nan_to_num(7), y[rows - 1].nan_to_num(7).expand(rows, k))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pixels", [49, 40000])
def test_derivative_of_silu(tvg, pixels, dtype):
    """One pixel with a gradient, mean 0 and rstd 1: dbeta is act'(x) there, s + z s (1 - s), whose two terms have 10 roundings
    each (s 7, z and 1 - s one each, the sum).  dgamma is x times that.  The bf16 form: exp(-z) has an error of |z| half steps of
    its own beside that, which is |z| s below zero; above, 1 - s is a difference with |z| (1 - s) + 6 half steps of 1, times z, and zero
    from z = 18 on, where 1 + exp(-z) is 1."""
    import torch
    to = torch.bfloat16 if dtype == "bf16" else torch.float32
    z = far(dtype)
    z = torch.where(torch.isfinite(z), z, torch.zeros_like(z))
    x, dy = torch.zeros((1, pixels, 96), dtype=to, device="cuda"), torch.zeros((1, pixels, 96), dtype=to, device="cuda")
    x[0, pixels // 3] = z.to(to)
    dy[0, pixels // 3] = 1
    mean, rstd = torch.zeros((1, 96), device="cuda"), torch.ones((1, 96), device="cuda")
    one, zero = torch.ones(96, device="cuda"), torch.zeros(96, device="cuda")
    _, dgamma, dbeta = tvg.group_norm_fused_backward(x, dy, mean, rstd, 96, one, zero, activation="silu")
    v = z.double()
    e = torch.exp(-v.abs())
    s, rest = torch.where(v >= 0, 1 / (1 + e), e / (1 + e)), torch.where(v >= 0, e / (1 + e), 1 / (1 + e))
    want = s + v * s * rest
    bound = 10 * H * (s + (v * s * rest).abs()) + (v.abs() + 1) * 2.0 ** -149
    if dtype == "bf16":
        bound += H * torch.where(v > 0, v.clamp(max=18) * (v.clamp(max=18) * rest + 6), v.abs() * s * (1 + v.abs())) + (v.abs() + 1) * 2.0 ** -125 * (v < 0)
    same_or_within(dbeta, want, bound)
    small = v.abs() < 1e18
    same_or_within(dgamma[small], (want * v)[small], (bound * v.abs() + H * (want * v).abs() + 2.0 ** -149)[small])
