"""Group norm where it takes two launches, and one launch with a workspace: streams, workspaces and graphs, in place, and through
the Python implementation of the calls."""
import pytest

from test_gpu_group_norm import inputs

pytestmark = pytest.mark.gpu

# shape, groups, whether the forward and the backward call want a workspace: two launches both; two for the gradients; one and the
# sums over samples; two with groups inside and across vectors
SHAPES = [((3, 112, 112, 64), 8, True, True), ((32, 28, 28, 256), 32, False, True), ((2, 14, 14, 256), 16, False, True),
          ((2, 190, 200, 36), 4, True, True), ((1, 300, 300, 64), 32, True, True)]


def needs(tvg, x, groups):
    import torch
    kind = tvg.TVG_BF16 if x.dtype == torch.bfloat16 else tvg.TVG_F32
    d = tvg.GroupNormDesc(x.shape[0], x.shape[1] * x.shape[2], x.shape[3], groups, kind, tvg.TVG_ACT_SILU, 1e-5, 0)
    return tvg.tvg_group_norm_workspace_size(d), tvg.tvg_group_norm_backward_workspace_size(d)


def both(calls, t, groups, **kw):
    x, dy, gamma, beta = t
    y, mean, rstd = calls[0](x, groups, gamma, beta, activation="silu", stats=True, **kw)
    return (y, mean, rstd) + calls[1](x, dy, mean, rstd, groups, gamma, beta, activation="silu", **kw)


def same(got, want):
    import torch
    return all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,groups,forward,backward", SHAPES)
def test_streams_workspaces_and_graphs(tvg, shape, groups, forward, backward, dtype):
    import torch
    t = inputs(shape, dtype, sum(shape))
    calls = tvg.group_norm_fused, tvg.group_norm_fused_backward
    need = needs(tvg, t[0], groups)
    assert (need[0] > 0, need[1] > 0) == (forward, backward)
    want = both(calls, t, groups)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        got = both(calls, t, groups, stream=stream)
        side.synchronize()
        assert same(got, want)
    # a workspace of the caller's that holds NaN, exactly as large as the query says, and nothing behind it written
    room = torch.full((max(need) + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    assert same(both(calls, t, groups, workspace=room[:max(need)]), want)
    assert bool((room[max(need):] == 0xFF).all())
    # two calls at once, on other maps
    other = [v.flip(0).contiguous() if v.dim() > 1 else v for v in t]
    want2 = both(calls, other, groups)
    torch.cuda.synchronize()
    got = []
    for i in range(6):
        with torch.cuda.stream(side if i % 2 else torch.cuda.current_stream()):
            got.append(both(calls, other if i % 2 else t, groups))
    torch.cuda.synchronize()
    assert all(same(g, want2 if i % 2 else want) for i, g in enumerate(got))
    # graphs whose workspace is the capture's own, maps that change in between
    graph, x = torch.cuda.CUDAGraph(), t[0].clone()
    with torch.cuda.graph(graph):
        captured = both(calls, (x,) + tuple(t[1:]), groups)
    for i in range(4):
        x.copy_(other[0] if i % 2 else t[0])
        for v in captured:
            v.fill_(float("nan"))
        graph.replay()
        eager = both(calls, (x,) + tuple(t[1:]), groups)
        torch.cuda.synchronize()
        assert same(captured, eager), i
        assert i % 2 or same(captured, want), i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,groups,forward,backward", SHAPES)
def test_in_place(tvg, shape, groups, forward, backward, dtype):
    """y over x, dx over dy and over x."""
    import torch
    x, dy, gamma, beta = inputs(shape, dtype, sum(shape) + 1)
    y, mean, rstd, dx, dgamma, dbeta = both((tvg.group_norm_fused, tvg.group_norm_fused_backward), (x, dy, gamma, beta), groups)
    for over in ("dy", "x"):
        a, b = x.clone(), dy.clone()
        got = tvg.group_norm_fused_backward(a, b, mean, rstd, groups, gamma, beta, activation="silu", out=b if over == "dy" else a)
        assert got[0] is (b if over == "dy" else a)
        assert same(got, (dx, dgamma, dbeta)), over
    a = x.clone()
    assert tvg.group_norm_fused(a, groups, gamma, beta, activation="silu", out=a) is a and torch.equal(a, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,groups,forward,backward", SHAPES)
def test_the_python_implementation_has_the_same_bits(tvg, shape, groups, forward, backward, dtype):
    import torch
    from paper_1802_04799_amd import binding
    t = inputs(shape, dtype, sum(shape) + 2)
    want = both((tvg.group_norm_fused, tvg.group_norm_fused_backward), t, groups)
    calls = binding._CONVENIENCES["group_norm_fused"], binding._CONVENIENCES["group_norm_fused_backward"]
    assert same(both(calls, t, groups), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(calls, t, groups, stream=side)
    side.synchronize()
    assert same(got, want)
    # a call that the native path leaves to it: an eps that is no float
    import fractions
    y, mean, rstd = tvg.group_norm_fused(t[0], groups, t[2], t[3], eps=fractions.Fraction(1e-5), activation="silu", stats=True)
    assert same((y, mean, rstd), want)


# the widest rows: one group, a group of every two channels, a group of every channel; the most samples
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,groups", [((2, 1, 1, 1048575), 1), ((2, 1, 3, 1048574), 524287), ((1, 3, 1, 1048560), 1048560), ((262143, 1, 1, 64), 8),
                                          ((262143, 3, 1, 24), 1)])
def test_widest_rows_and_most_samples(tvg, shape, groups, dtype):
    """Forward as the other shapes; gradients' sums over samples are 16 chains of n / 16 terms."""
    import torch
    from test_gpu_group_norm import H, check_forward, grad64, grouped
    x, dy, gamma, beta = inputs(shape, dtype, groups)
    _, mean, rstd = check_forward(tvg, x, groups, gamma, beta, "silu", dtype)
    dx, dgamma, dbeta = tvg.group_norm_fused_backward(x, dy, mean, rstd, groups, gamma, beta, activation="silu")
    n, c = shape[0], shape[-1]
    per = lambda t: t.view(n, 1, groups, 1)
    xhat = (grouped(x, groups) - per(mean.double())) * per(rstd.double())
    xh = xhat.reshape(n, -1, c)
    z = xh * gamma.double() + beta.double()
    dz = dy.double().reshape(n, -1, c) * grad64(z, "silu")
    # a term: 20 roundings of z's size and its slope (below), the row's sums and the chain of samples
    term = 20 * H * (1 + z.abs()) * dy.double().reshape(n, -1, c).abs()
    chain = (64 + n // 16 + 16) * H
    for got, t, e in ((dbeta, dz, term), (dgamma, dz * xh, term * xh.abs())):
        want, size = t.sum((0, 1)), t.abs().sum((0, 1))
        assert bool(((got.double() - want).abs() <= e.sum((0, 1)) + chain * size + 1e-37).all())
    assert bool(torch.isfinite(dx).all())
    # dx of a few samples, from the sums in 64 bits
    g = gamma.double()
    few = slice(0, n, max(1, n // 50))
    m = xhat.shape[1] * (c // groups)
    over = lambda t: t.view(t.shape[0], -1, groups, c // groups).sum((1, 3), keepdim=True) / m
    gdz = (g * dz[few])
    a, b = over(gdz), over(gdz * xh[few])
    r = per(rstd.double())[few]
    split = lambda t: t.view(t.shape[0], -1, groups, c // groups)
    want = r * (split(gdz) - a - split(xh[few]) * b)
    size = r * (split(gdz).abs() + over(gdz.abs()) + split(xh[few]).abs() * over((gdz * xh[few]).abs()))
    tol = r * split(g * term[few]) + 520 * H * size + r * (over(g * term[few]) + split(xh[few]).abs() * over(g * term[few] * xh[few].abs()))
    half = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
    assert bool(((dx[few].double().view(want.shape) - want).abs() <= tol + half * want.abs() + 1e-37).all())
