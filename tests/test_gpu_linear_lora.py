"""Projection with a low-rank adapter chosen row by row, against the formula in 64 bits.

Tolerance, counted in half steps h = 2^-24 of fp32 before any run.  A sum of m products in fp32, in any order and with the
matrix cores' rounding of every addition (up to one step each), is within 2 m h of the sum of absolute products; what is added
one behind the other in one accumulator bounds m, and for random signs the errors grow as its root.  The bound here is
(16 + 4 sqrt(m)) h of the sum of absolute products - four standard deviations.  The adapter's middle vector has the errors of
its own sum and, in bf16, 2^-17 of its split; y one rounding of its type.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def make(rows, c, k, rank, adapters, dtype, seed, residual=False, bias=False, scale=True):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    to = torch.bfloat16 if dtype == "bf16" else torch.float32
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    p = dict(x=r(rows, c).to(to), w=(r(k, c) * c ** -0.5).to(to), a=(r(adapters, rank, c) * c ** -0.5).to(to),
             b=(r(adapters, k, rank) * rank ** -0.5).to(to))
    p["adapter"] = torch.randint(-1, adapters, (rows,), generator=g, device="cuda", dtype=torch.int32)
    p["scale"] = torch.rand(adapters, generator=g, device="cuda") + 0.5 if scale else None
    p["bias"] = r(k) if bias else None
    p["residual"] = r(rows, k).to(to) if residual else None
    return p


def wanted(p, act, dtype):
    """y in 64 bits and its tolerance."""
    import torch
    x, w = p["x"].double(), p["w"].double()
    c = x.shape[1]
    y, mag = x @ w.t(), x.abs() @ w.abs().t()
    tol = (16 + 4 * math.sqrt(c)) * H * mag
    for i in range(p["a"].shape[0]):
        at = (p["adapter"] == i).nonzero().flatten()
        if not at.numel():
            continue
        a, b = p["a"][i].double(), p["b"][i].double()
        s = 1.0 if p["scale"] is None else float(p["scale"][i])
        h, hmag = x[at] @ a.t(), x[at].abs() @ a.abs().t()
        eh = (16 + 4 * math.sqrt(c)) * H * hmag + (2.0 ** -17 if dtype == "bf16" else 2 * H) * h.abs()
        y[at] += s * (h @ b.t())
        tol[at] += abs(s) * (eh @ b.abs().t() + (16 + 4 * math.sqrt(2 * a.shape[0])) * H * (h.abs() @ b.abs().t()))
    for name in ("bias", "residual"):
        if p[name] is not None:
            y = y + p[name].double()
            tol = tol + 4 * H * p[name].double().abs()
    if act == "relu":
        y = y.clamp(min=0)
    if act == "silu":
        y = y * torch.sigmoid(y)
    return y, 1.1 * tol + 8 * H * y.abs() + HALF[dtype] * y.abs() + 1e-37


def check(tvg, p, act, dtype, **kw):
    import torch
    y = tvg.linear_lora_fused(p["x"], p["w"], p["a"], p["b"], p["adapter"], p["scale"], p["bias"], p["residual"], activation=act, **kw)
    torch.cuda.synchronize()
    want, tol = wanted(p, act, dtype)
    err = (y.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    return y


# rows, c, k, rank, adapters
SHAPES = [(1, 1024, 1024, 16, 8), (1, 1, 1, 1, 1), (2, 64, 64, 8, 1), (3, 73, 523, 4, 5), (5, 4096, 96, 16, 3), (16, 256, 256, 16, 4),
          (17, 520, 200, 12, 3), (33, 100, 36, 5, 9), (64, 1024, 512, 16, 32), (64, 4096, 256, 64, 64), (65, 512, 130, 32, 2),
          (100, 2048, 260, 17, 7), (128, 64, 1000, 128, 3), (200, 320, 320, 256, 2), (257, 384, 264, 8, 4), (300, 8, 8, 8, 2),
          (513, 136, 520, 24, 6), (777, 1000, 515, 12, 6), (1030, 256, 300, 16, 5), (70, 8200, 64, 16, 4)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,k,rank,adapters", SHAPES)
def test_projection(tvg, rows, c, k, rank, adapters, dtype):
    seed = rows + c + k + rank
    check(tvg, make(rows, c, k, rank, adapters, dtype, seed), None, dtype)
    check(tvg, make(rows, c, k, rank, adapters, dtype, seed, residual=True, bias=True, scale=False), ("relu", "silu")[seed % 2], dtype)


# ... of many tiles: 64, 128 and 256 rows and channels a tile (bf16; fp32 up to 128), ragged at both ends, reductions shorter
# than a step, ranks that are not whole 16-byte pieces, rows at any element
LARGE = [(1100, 72, 1100, 16, 5), (1100, 1000, 1100, 12, 9), (300, 64, 6000, 256, 2), (2100, 72, 2060, 40, 7), (2048, 8, 2048, 8, 3),
         (2048, 200, 2049, 5, 11), (4100, 136, 2600, 16, 30), (4100, 520, 2600, 72, 30), (4097, 40, 2570, 4, 3), (1100, 37, 1100, 7, 4)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,k,rank,adapters", LARGE)
def test_large_projection(tvg, rows, c, k, rank, adapters, dtype):
    seed = rows + c + k + rank
    check(tvg, make(rows, c, k, rank, adapters, dtype, seed), None, dtype)
    check(tvg, make(rows, c, k, rank, adapters, dtype, seed, residual=True, bias=True, scale=False), ("relu", "silu")[seed % 2], dtype)


# ... of many tiles whose rows are no whole 16-byte pieces
RAGGED = [(1100, 133, 1100, 16, 5), (2100, 515, 2060, 12, 9), (300, 1001, 6001, 20, 2), (4100, 250, 2601, 16, 30), (1100, 129, 1100, 5, 300)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,k,rank,adapters", RAGGED)
def test_large_projection_of_ragged_rows(tvg, rows, c, k, rank, adapters, dtype):
    import torch
    seed = rows + c + k + rank
    p = make(rows, c, k, rank, adapters, dtype, seed, residual=True, bias=True)
    check(tvg, p, ("relu", "silu")[seed % 2], dtype)
    # without adapters: the same product
    y = tvg.linear_lora_fused(p["x"], p["w"], None, None, None)
    none = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    assert torch.equal(y, tvg.linear_lora_fused(p["x"], p["w"], p["a"], p["b"], none))
    # an adapter of infinities, rows of NaN: the others keep their bits
    want = tvg.linear_lora_fused(p["x"], p["w"], p["a"], p["b"], p["adapter"], p["scale"], p["bias"], p["residual"])
    a, x = p["a"].clone(), p["x"].clone()
    a[0] = float("inf")
    x[1] = float("nan")
    got = tvg.linear_lora_fused(x, p["w"], a, p["b"], p["adapter"], p["scale"], p["bias"], p["residual"])
    keep = p["adapter"] != 0
    keep[1] = False
    assert bool(torch.isnan(got[1]).all()) and torch.equal(got[keep], want[keep])


# ... of few tiles, whose product is cut into parts by what h leaves of the CUs, and beside many adapters, which are not copied: a
# call without adapters may add up in another order, within the tolerance, not bit by bit.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,k,rank,adapters", [(40, 4097, 1700, 16, 5), (777, 1001, 515, 12, 6), (17, 4099, 4096, 20, 20), (2, 20001, 7000, 16, 2),
                                                      (1100, 133, 1100, 16, 200)])
def test_ragged_rows_of_few_tiles_or_many_adapters(tvg, rows, c, k, rank, adapters, dtype):
    import torch
    seed = rows + c + k + rank
    p = make(rows, c, k, rank, adapters, dtype, seed, residual=True, bias=True)
    want = check(tvg, p, None, dtype)
    none = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    bare = dict(p, adapter=none, bias=None, residual=None)
    check(tvg, bare, None, dtype)
    y = tvg.linear_lora_fused(p["x"], p["w"], None, None, None)
    y64, tol = wanted(bare, None, dtype)
    assert bool(((y.double() - y64).abs() <= tol).all())
    a, x = p["a"].clone(), p["x"].clone()
    a[0] = float("inf")
    x[1] = float("nan")
    got = tvg.linear_lora_fused(x, p["w"], a, p["b"], p["adapter"], p["scale"], p["bias"], p["residual"])
    keep = p["adapter"] != 0
    keep[1] = False
    assert bool(torch.isnan(got[1]).all()) and torch.equal(got[keep], want[keep])


def assignments(rows, adapters):
    """Rows of requests of many kinds: one adapter, none, long runs, single rows, unsorted, indices out of range."""
    import torch
    t = torch.arange(rows, device="cuda", dtype=torch.int32)
    odd = torch.full((rows,), -1, device="cuda", dtype=torch.int32)
    odd[::3], odd[1::7], odd[2::5] = adapters - 1, adapters, 2 ** 31 - 1
    odd[4::11] = -2 ** 31
    return {"one": t * 0 + adapters - 1, "none": t * 0 - 1, "runs": t // max(1, rows // adapters) % adapters,
            "single": t % adapters, "backwards": (rows - 1 - t) * 7 % adapters, "odd": odd,
            "last row": torch.where(t == rows - 1, 0, -1).int()}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,k,rank,adapters", [(40, 512, 192, 16, 40), (300, 256, 320, 8, 6), (1100, 128, 520, 32, 9), (7, 1024, 64, 20, 3),
                                                      (1100, 136, 1100, 16, 40), (2100, 72, 2060, 32, 5000), (4100, 72, 2600, 24, 60)])
def test_assignments(tvg, rows, c, k, rank, adapters, dtype):
    p = make(rows, c, k, rank, adapters, dtype, rows)
    for name, index in assignments(rows, adapters).items():
        p["adapter"] = index
        check(tvg, p, None, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k", [(1, 264), (6, 264), (50, 264), (300, 264), (1100, 264), (1100, 1100), (2100, 2060), (4100, 2600)])
def test_a_row_does_not_see_the_adapters_of_others(tvg, rows, k, dtype):
    """Adapters full of infinities and NaN, and rows of x too: the other rows keep their bits."""
    import torch
    p = make(rows, 256, k, 16, 4, dtype, rows)
    call = lambda: tvg.linear_lora_fused(p["x"], p["w"], p["a"], p["b"], p["adapter"], p["scale"])
    clean = call()
    keep = p["adapter"] != 2
    p["a"][2], p["b"][2] = float("inf"), float("nan")
    p["scale"][2] = float("nan")
    y = call()
    assert torch.equal(y[keep], clean[keep])
    assert bool(torch.isnan(y[~keep]).all())
    p["x"][rows // 2] = float("nan")
    y = call()
    keep[rows // 2] = False
    assert torch.equal(y[keep], clean[keep]) and bool(torch.isnan(y[rows // 2]).all())


def test_infinite_middle_vectors_stay_infinite(tvg):
    """An infinity in x through an adapter without zeros: infinity or NaN as in the formula, not NaN everywhere."""
    import torch
    for dtype in ("f32", "bf16"):
        p = make(20, 64, 64, 16, 2, dtype, 3)
        p["w"].zero_()
        p["w"].add_(1)
        p["a"].zero_().add_(1)
        p["b"].zero_().add_(1)
        p["x"][7, 5] = float("inf")
        p["adapter"].zero_()
        y = tvg.linear_lora_fused(p["x"], p["w"], p["a"], p["b"], p["adapter"])
        assert bool(torch.isinf(y[7]).all()) and bool(torch.isfinite(y[torch.arange(20, device="cuda") != 7]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k", [(3, 136), (40, 136), (300, 136), (1100, 1096), (2100, 2056), (4100, 2600)])
def test_any_alignment_and_surroundings(tvg, rows, k, dtype):
    """Operands that start at any element: the same result within the tolerance, and nothing beside y is written."""
    import torch
    p = make(rows, 256, k, 16, 3, dtype, 77, residual=True, bias=True)
    check(tvg, p, "silu", dtype)
    for name in ("x", "w", "a", "b", "residual"):
        t = p[name]
        room = torch.zeros(t.numel() + 8, dtype=t.dtype, device="cuda")
        p[name] = room[1:1 + t.numel()].view(t.shape).copy_(t)
        room = torch.full((rows * k + 16,), 7.0, dtype=t.dtype, device="cuda")
        out = room[3:3 + rows * k].view(rows, k)
        check(tvg, p, "silu", dtype, out=out)
        assert bool((room[:3] == 7).all()) and bool((room[3 + rows * k:] == 7).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_adapters_no_rows_and_more_dimensions(tvg, dtype):
    import torch
    p = make(30, 64, 72, 8, 2, dtype, 5)
    plain = tvg.linear_lora_fused(p["x"], p["w"], None, None, None)
    p["adapter"].fill_(-1)
    assert torch.equal(plain, check(tvg, p, None, dtype))
    assert tvg.linear_lora_fused(p["x"][:0], p["w"], p["a"], p["b"], p["adapter"][:0]).shape == (0, 72)
    p["adapter"].fill_(1)
    y = check(tvg, p, None, dtype)
    cube = tvg.linear_lora_fused(p["x"].view(2, 3, 5, 64), p["w"], p["a"], p["b"], p["adapter"], p["scale"])
    assert cube.shape == (2, 3, 5, 72) and torch.equal(cube.view(30, 72), y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k", [(1, 256), (20, 256), (64, 256), (300, 256), (1100, 1100), (2100, 2060), (4100, 2600)])
def test_streams_graphs_and_repeats(tvg, rows, k, dtype):
    """The same bits again, on another stream, with a workspace and an output of the caller's, over the residual, and from
    every replay of a graph whose adapter indices change in between."""
    import torch
    p = make(rows, 1024 if rows < 1000 else 192, k, 16, 8, dtype, rows, residual=True)
    call = lambda **kw: tvg.linear_lora_fused(p["x"], p["w"], p["a"], p["b"], p["adapter"], p["scale"], None, p["residual"], **kw)
    want = call()
    assert torch.equal(call(), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        y = call(stream=stream)
        side.synchronize()
        assert torch.equal(y, want)
    room = torch.full((1 << 23,), 0xFF, dtype=torch.uint8, device="cuda")
    assert torch.equal(call(workspace=room, out=torch.empty_like(want)), want)
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = call()
    first = p["adapter"].clone()
    for i in range(4):
        p["adapter"].copy_((first + i) % 8)
        y.fill_(float("nan"))
        graph.replay()
        eager = call()
        torch.cuda.synchronize()
        assert torch.equal(y, eager), i
        assert i > 0 or bool((first < 0).any()) or torch.equal(y, want)
    p["adapter"].copy_(first)
    # two calls at once, each with its own memory
    other = dict(p, x=p["x"].flip(0).contiguous())
    want2 = tvg.linear_lora_fused(other["x"], p["w"], p["a"], p["b"], p["adapter"], p["scale"], None, p["residual"])
    torch.cuda.synchronize()
    ys = []
    for i in range(6):
        with torch.cuda.stream(side if i % 2 else torch.cuda.current_stream()):
            ys.append(tvg.linear_lora_fused((other if i % 2 else p)["x"], p["w"], p["a"], p["b"], p["adapter"], p["scale"], None, p["residual"]))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want2 if i % 2 else want) for i, y in enumerate(ys))
    over = p["residual"].clone()
    p["residual"] = over
    assert call(out=over) is over
    assert torch.equal(over, want)
