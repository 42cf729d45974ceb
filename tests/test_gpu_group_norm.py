"""Group norm with an activation, channels last, forward and backward, against the formula in 64 bits.

Tolerances, counted in half steps h = 2^-24 of fp32 before any run:
  mean        joined from lanes, rows and chunks: at most 64 roundings of numbers no larger than max |x| of the group
  rstd        M2 is a sum of squares, 64 roundings of its terms; half of that reaches rstd, and the mean's error counts
              once more in second order only
  z           (x - mean) * (rstd gamma) + beta: the mean's error and 72 roundings of the products
  act         slope at most 1.1, exp and reciprocal within 8 roundings of the result
  y           one rounding of its type more
  sums        S1 and S2 add at most 512 terms one behind the other in any of these shapes; a term has the errors of z
"""
import pytest

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def act64(z, act):
    import torch
    return z.clamp(min=0) if act == "relu" else z * torch.sigmoid(z) if act == "silu" else z


def grad64(z, act):
    import torch
    if act == "relu":
        return (z > 0).double()
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s)) if act == "silu" else torch.ones_like(z)


def grouped(t, groups):
    """[n][...][c] -> [n][p][groups][c / groups] in 64 bits"""
    return t.double().reshape(t.shape[0], -1, groups, t.shape[-1] // groups)


def reference(x, groups, gamma, beta, eps):
    """xhat and z [n][p][c], mean, rstd [n][groups], and z's tolerance."""
    v = grouped(x, groups)
    mean = v.mean(dim=(1, 3), keepdim=True)
    var = ((v - mean) ** 2).mean(dim=(1, 3), keepdim=True)
    rstd = (var + eps) ** -0.5
    xhat = (v - mean) * rstd
    biggest = v.abs().amax(dim=(1, 3), keepdim=True)
    flat = (x.shape[0], -1, x.shape[-1])
    g = 1.0 if gamma is None else gamma.double()
    b = 0.0 if beta is None else beta.double()
    z = xhat.reshape(flat) * g + b
    # the mean's error moves every distance, and M2 by its square times the elements
    dmean = 64 * H * biggest
    drstd = rstd * (72 * H + 0.5 * (dmean * rstd) ** 2)
    tol = (dmean * rstd + xhat.abs() * (drstd / rstd)).reshape(flat) * (g if gamma is None else g.abs()) + 8 * H * z.abs() + 2 * H * (0.0 if beta is None else b.abs())
    return xhat.reshape(flat), z, mean, rstd, tol, dmean, drstd


def inputs(shape, dtype, seed, offset=0.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    c = shape[-1]
    x = r(*shape) * (torch.rand(c, generator=g, device="cuda") * 1.5 + 0.5) + r(c) + offset
    to = torch.bfloat16 if dtype == "bf16" else torch.float32
    return x.to(to), r(*shape).to(to), torch.rand(c, generator=g, device="cuda") + 0.5, r(c) * 0.3


def check_forward(tvg, x, groups, gamma, beta, act, dtype, eps=1e-5, **kw):
    import torch
    y, mean, rstd = tvg.group_norm_fused(x, groups, gamma, beta, eps=eps, activation=act, stats=True, **kw)
    torch.cuda.synchronize()
    _, z, m64, r64, tol, dmean, drstd = reference(x, groups, gamma, beta, eps)
    want = act64(z, act)
    got = y.double().reshape(want.shape)
    bound = 1.1 * tol + 8 * H * want.abs() + HALF[dtype] * want.abs() + 1e-37
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())
    assert bool(((mean.double() - m64.flatten(1)).abs() <= dmean.flatten(1) + 1e-37).all())
    assert bool(((rstd.double() - r64.flatten(1)).abs() <= drstd.flatten(1)).all())
    return y, mean, rstd


# shape, groups: whole vectors in a group, groups inside a vector, groups that straddle vectors, odd channels, one pixel,
# one channel, one group wider than a pass, channels in several blocks (the last one narrower), more rows than lanes
SHAPES = [((2, 7, 7, 64), 8), ((1, 7, 7, 512), 32), ((3, 45, 37, 84), 12), ((2, 5, 9, 320), 32), ((2, 6, 5, 96), 96),
          ((5, 3, 3, 35), 7), ((4, 1, 33), 3), ((1, 1, 1), 1), ((3, 17, 1), 1), ((2, 4, 5, 4100), 1), ((1, 9, 5000), 4),
          ((2, 11, 2600), 520), ((2, 3, 6006), 6), ((7, 64), 4), ((1, 130, 121, 16), 4), ((40, 3, 5, 24), 8), ((1, 2000, 40), 4)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", [None, "relu", "silu"])
@pytest.mark.parametrize("shape,groups", SHAPES, ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else str(v))
def test_forward(tvg, shape, groups, act, dtype):
    x, _, gamma, beta = inputs(shape, dtype, sum(shape) + groups)
    check_forward(tvg, x, groups, gamma, beta, act, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_without_parameters_and_statistics(tvg, dtype):
    import torch
    x, _, gamma, beta = inputs((3, 10, 11, 48), dtype, 5)
    for g, b in ((None, None), (gamma, None), (None, beta)):
        y, _, _ = check_forward(tvg, x, 6, g, b, "silu", dtype)
        assert torch.equal(y, tvg.group_norm_fused(x, 6, g, b, activation="silu"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_mean_far_from_zero_costs_no_digits(tvg, dtype):
    """1000 times the spread: E[x^2] - E[x]^2 would lose 20 of 24 bits.  An early outlier does no harm either."""
    for seed, offset in ((1, 1000.0), (2, -300.0)):
        x, _, gamma, beta = inputs((2, 33, 31, 40), dtype, seed, offset)
        check_forward(tvg, x, 4, gamma, beta, None, dtype)
    x[:, 0, 0] = 3e4
    check_forward(tvg, x, 4, gamma, beta, None, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_constant_groups(tvg, dtype):
    import torch
    x, _, gamma, beta = inputs((2, 9, 7, 32), dtype, 9)
    x[0] = 3.5
    y, mean, rstd = tvg.group_norm_fused(x, 4, gamma, beta, eps=1e-3, stats=True)
    assert torch.equal(y[0].float(), beta.to(x.dtype).float().expand(9, 7, 32))
    assert bool((mean[0] == 3.5).all()) and bool(((rstd[0].double() - 1e-3 ** -0.5).abs() < 1e-4).all())
    check_forward(tvg, x[1:].contiguous(), 4, gamma, beta, None, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_and_nan_stay_in_their_group(tvg, dtype):
    import torch
    x, _, gamma, beta = inputs((3, 13, 11, 40), dtype, 10)
    clean = tvg.group_norm_fused(x, 8, gamma, beta, activation="relu")
    for value in (float("nan"), float("inf"), -float("inf")):
        bad = x.clone()
        bad[1, 5, 3, 17] = value                              # group 3 of sample 1
        y = tvg.group_norm_fused(bad, 8, gamma, beta, activation="relu")
        hit = torch.zeros(y.shape, dtype=torch.bool, device="cuda")
        hit[1, :, :, 15:20] = True
        assert bool(torch.isnan(y[hit]).all()) and torch.equal(y[~hit], clean[~hit])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 2, 4])
def test_any_alignment_and_in_place(tvg, shift, dtype):
    """Tensors that start at any element, and an output over the input."""
    import torch
    shape = (2, 9, 11, 64)
    x, dy, gamma, beta = inputs(shape, dtype, 11)
    room = torch.zeros(x.numel() + 8, dtype=x.dtype, device="cuda")
    moved = room[shift:shift + x.numel()].view(shape).copy_(x)
    y, mean, rstd = check_forward(tvg, moved, 8, gamma, beta, "silu", dtype)
    dx, _, _ = tvg.group_norm_fused_backward(moved, dy, mean, rstd, 8, gamma, beta, activation="silu")
    check_backward(tvg, moved, dy, 8, gamma, beta, "silu", dtype)
    assert tvg.group_norm_fused(moved, 8, gamma, beta, activation="silu", out=moved) is moved
    assert torch.equal(moved, y)
    assert bool((room[:shift] == 0).all()) and bool((room[shift + x.numel():] == 0).all())
    moved.copy_(x)
    tvg.group_norm_fused_backward(moved, dy, mean, rstd, 8, gamma, beta, activation="silu", out=dy)
    assert torch.equal(dy, dx)


def check_backward(tvg, x, dy, groups, gamma, beta, act, dtype):
    import torch
    eps = 1e-5
    _, mean, rstd = tvg.group_norm_fused(x, groups, gamma, beta, eps=eps, activation=act, stats=True)
    dx, dgamma, dbeta = tvg.group_norm_fused_backward(x, dy, mean, rstd, groups, gamma, beta, activation=act)
    torch.cuda.synchronize()
    n, c, cpg = x.shape[0], x.shape[-1], x.shape[-1] // groups
    # the operator's own statistics: what the forward pass left
    v = grouped(x, groups)
    r = rstd.double().view(n, 1, groups, 1)
    xhat = ((v - mean.double().view(n, 1, groups, 1)) * r)
    g = torch.ones(c, dtype=torch.float64, device="cuda") if gamma is None else gamma.double()
    b = torch.zeros(c, dtype=torch.float64, device="cuda") if beta is None else beta.double()
    z = xhat.reshape(n, -1, c) * g + b
    dz = dy.double().reshape(n, -1, c) * grad64(z, act)
    xh = xhat.reshape(n, -1, c)
    # z has 4 roundings of its terms; act' has a slope below 0.6 and 16 roundings of numbers up to 1 + |z|
    dxhat = 3 * H * xh.abs()
    ez = 4 * H * (xh.abs() * g.abs() + b.abs())
    edz = dy.double().reshape(n, -1, c).abs() * ((0.6 * ez + 16 * H * (1 + z.abs())) if act == "silu" else 0 * ez)
    s1, s2 = dz.sum(1), (dz * xh).sum(1)
    e1 = edz.sum(1) + 512 * H * dz.abs().sum(1)
    e2 = (edz * xh.abs() + dz.abs() * dxhat).sum(1) + 512 * H * (dz * xh).abs().sum(1)
    if beta is None:
        assert dbeta is None
    else:
        assert bool(((dbeta.double() - s1.sum(0)).abs() <= e1.sum(0) + 1e-37).all())
    if gamma is None:
        assert dgamma is None
    else:
        assert bool(((dgamma.double() - s2.sum(0)).abs() <= e2.sum(0) + 1e-37).all())
    m = v.shape[1] * cpg
    per = lambda t: t.reshape(n, groups, cpg).sum(2).repeat_interleave(cpg, 1).unsqueeze(1)
    a, bb = per(g * s1) / m, per(g * s2) / m
    ea, eb = per(g.abs() * e1 + 64 * H * (g * s1).abs()) / m, per(g.abs() * e2 + 64 * H * (g * s2).abs()) / m
    rr = r.expand(n, 1, groups, cpg).reshape(n, 1, c)
    want = rr * (g * dz - a - xh * bb)
    terms = rr * ((g * dz).abs() + a.abs() + (xh * bb).abs())
    bound = rr * (g.abs() * edz + ea + xh.abs() * eb + dxhat * bb.abs()) + 8 * H * terms + HALF[dtype] * want.abs() + 1e-37
    err = (dx.double().reshape(want.shape) - want).abs()
    assert bool((err <= bound).all()), float((err / bound).max())
    return dx, dgamma, dbeta


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", [None, "silu"])
@pytest.mark.parametrize("shape,groups", SHAPES, ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else str(v))
def test_backward(tvg, shape, groups, act, dtype):
    x, dy, gamma, beta = inputs(shape, dtype, sum(shape) + groups + 1)
    check_backward(tvg, x, dy, groups, gamma, beta, act, dtype)


# many row chunks, more of them than one round of loads joins, one chunk of many samples, more rows than lanes of odd channels
LARGE = [((1, 300, 300, 64), 32), ((3, 112, 112, 64), 8), ((2, 190, 200, 36), 4), ((70, 60, 61, 24), 24), ((520, 100, 100, 16), 4),
         ((1, 70000, 1), 1), ((1, 40000, 3), 3), ((1, 700, 5000), 8), ((1, 23, 5001), 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,groups", LARGE, ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else str(v))
def test_large_maps(tvg, shape, groups, dtype):
    x, dy, gamma, beta = inputs(shape, dtype, sum(shape) + groups + 2)
    check_forward(tvg, x, groups, gamma, beta, "silu", dtype)
    check_backward(tvg, x, dy, groups, gamma, beta, "silu", dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_of_relu_and_without_parameters(tvg, dtype):
    """x such that no z lies near zero, where a rounding would decide."""
    import torch
    x, dy, gamma, beta = inputs((3, 8, 9, 48), dtype, 21)
    for g, b in ((gamma, beta), (None, None), (gamma, None), (None, beta)):
        xx = x.clone()
        for _ in range(20):
            _, z, *_ = reference(xx, 6, g, b, 1e-5)
            near = (z.abs() < 1e-3).reshape(xx.shape)
            if not bool(near.any()):
                break
            xx[near] += 0.25
        assert not bool(near.any())
        check_backward(tvg, xx, dy, 6, g, b, "relu", dtype)


def test_backward_against_differences(tvg):
    """The gradient's direction: sum(dx d) is the change of sum(y dy) along d.  Central differences of the forward
    formula in 64 bits, step 1e-4: their own error is of the order of 1e-8 of the third derivative."""
    import torch
    x, dy, gamma, beta = inputs((2, 6, 5, 24), "f32", 31)
    _, mean, rstd = tvg.group_norm_fused(x, 4, gamma, beta, activation="silu", stats=True)
    dx, dgamma, dbeta = tvg.group_norm_fused_backward(x, dy, mean, rstd, 4, gamma, beta, activation="silu")

    def loss(xx, g, b):
        _, z, *_ = reference(xx, 4, g, b, 1e-5)
        return float((act64(z, "silu") * dy.double().reshape(z.shape)).sum())

    gen = torch.Generator(device="cuda").manual_seed(3)
    for grad, at in ((dx, 0), (dgamma, 1), (dbeta, 2)):
        p = [x.double(), gamma.double(), beta.double()]
        d = torch.randn(p[at].shape, generator=gen, device="cuda", dtype=torch.float64)
        up, down = list(p), list(p)
        up[at], down[at] = p[at] + 1e-4 * d, p[at] - 1e-4 * d
        slope = (loss(*up) - loss(*down)) / 2e-4
        got = float((grad.double() * d).sum())
        assert abs(got - slope) <= 1e-5 * float((grad.double() * d).abs().sum()), (at, got, slope)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_streams_graphs_and_repeats(tvg, dtype):
    """The same bits from a second call, on another stream, with a workspace of the caller's, through the Python
    implementation, and from every replay of a graph between eager work."""
    import torch
    x, dy, gamma, beta = inputs((4, 28, 27, 64), dtype, 41)

    def both(**kw):
        y, mean, rstd = tvg.group_norm_fused(x, 8, gamma, beta, activation="silu", stats=True, **kw)
        return (y, mean, rstd) + tvg.group_norm_fused_backward(x, dy, mean, rstd, 8, gamma, beta, activation="silu", **kw)

    want = both()
    same = lambda got: all(torch.equal(a, b) for a, b in zip(got, want))
    assert same(both())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        got = both(stream=stream)
        side.synchronize()
        assert same(got)
    room = torch.full((1 << 22,), 0xFF, dtype=torch.uint8, device="cuda")
    assert same(both(workspace=room))
    assert same(both(workspace=room[:0]))                     # too small: one of its own
    # two calls at once, each with its own memory
    got = []
    for i in range(6):
        with torch.cuda.stream(side if i % 2 else torch.cuda.current_stream()):
            got.append(both())
    torch.cuda.synchronize()
    assert all(same(g) for g in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    for i in range(4):
        for t in captured:
            t.fill_(float("nan"))
        graph.replay()
        assert same(both())
        torch.cuda.synchronize()
        assert same(captured), i


def test_rows_beyond_32_bits_of_bytes(tvg):
    """A map of 2^31 - 2^16 bf16 elements (4.3 GB): the last sample's addresses need more than 32 bits."""
    import torch
    n, p, c = 32767, 1024, 64
    x = torch.zeros((n, p, c), dtype=torch.bfloat16, device="cuda")
    part, dy, gamma, beta = inputs((2, p, c), "bf16", 51)
    x[-2:] = part
    y, mean, rstd = tvg.group_norm_fused(x, 8, gamma, beta, activation="silu", stats=True)
    assert bool((mean[:-2] == 0).all())
    small, smean, srstd = check_forward(tvg, part, 8, gamma, beta, "silu", "bf16")
    assert bool(((y[-2:].double() - small.double()).abs() <= 2.0 ** -7 * small.double().abs() + 1e-6).all())
    g = torch.zeros_like(x)
    g[-2:] = dy
    dx, dgamma, dbeta = tvg.group_norm_fused_backward(x, g, mean, rstd, 8, gamma, beta, activation="silu", out=y)
    sdx, sdgamma, sdbeta = check_backward(tvg, part, dy, 8, gamma, beta, "silu", "bf16")
    assert bool((dx[:-2] == 0).all())
    assert bool(((dx[-2:].double() - sdx.double()).abs() <= 2.0 ** -7 * sdx.double().abs() + 1e-5).all())
    assert bool(((dgamma - sdgamma).abs() <= 1e-2).all()) and bool(((dbeta - sdbeta).abs() <= 1e-2).all())
