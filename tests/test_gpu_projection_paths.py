"""Projections whose rows are copied to whole 16-byte pieces first, and those that read them at any element: streams, workspaces,
graphs and calls at once, and the Python implementation of the call."""
import pytest

from test_gpu_linear_lora import make

pytestmark = pytest.mark.gpu

# copied: a round of tiles; few tiles of much work (bf16).  Not copied: short rows; many adapters
SHAPES = [(1100, 133, 1100, 16, 8), (777, 1001, 515, 16, 8), (2100, 515, 2060, 12, 8), (64, 4097, 4096, 16, 8), (1100, 37, 1100, 7, 8),
          (1100, 133, 1100, 16, 200), (300, 264, 264, 16, 8), (64, 1024, 1024, 20, 8)]


def needed(tvg, p):
    import torch
    kind = tvg.TVG_BF16 if p["x"].dtype == torch.bfloat16 else tvg.TVG_F32
    (rows, c), (adapters, k, rank) = p["x"].shape, p["b"].shape
    return tvg.tvg_linear_lora_workspace_size(tvg.LinearLoraDesc(rows, c, k, adapters, rank, kind, 0, 0))


def call_of(f, p, **kw):
    return f(p["x"], p["w"], p["a"], p["b"], p["adapter"], p["scale"], p["bias"], p["residual"], **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,k,rank,adapters", SHAPES)
def test_streams_workspaces_and_graphs(tvg, rows, c, k, rank, adapters, dtype):
    import torch
    p = make(rows, c, k, rank, adapters, dtype, rows + c, residual=True, bias=True)
    f = tvg.linear_lora_fused
    want = call_of(f, p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        y = call_of(f, p, stream=stream)
        side.synchronize()
        assert torch.equal(y, want)
    need = needed(tvg, p)
    assert need > 0
    room = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    assert torch.equal(call_of(f, p, workspace=room[:need]), want) and bool((room[need:] == 0xFF).all())
    other = dict(p, x=p["x"].flip(0).contiguous())
    want2 = call_of(f, other)
    torch.cuda.synchronize()
    ys = []
    for i in range(6):
        with torch.cuda.stream(side if i % 2 else torch.cuda.current_stream()):
            ys.append(call_of(f, other if i % 2 else p))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want2 if i % 2 else want) for i, y in enumerate(ys))
    moving = dict(p, adapter=p["adapter"].clone(), x=p["x"].clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = call_of(f, moving)
    for i in range(4):
        moving["adapter"].copy_((p["adapter"] + i) % adapters if i else p["adapter"])
        moving["x"].copy_(other["x"] if i % 2 else p["x"])
        y.fill_(float("nan"))
        graph.replay()
        eager = call_of(f, moving)
        torch.cuda.synchronize()
        assert torch.equal(y, eager), i
        assert i or torch.equal(y, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,k,rank,adapters", SHAPES)
def test_the_python_implementation_has_the_same_bits(tvg, rows, c, k, rank, adapters, dtype):
    import torch
    from paper_1802_04799_amd import binding
    p = make(rows, c, k, rank, adapters, dtype, rows + c + 1, residual=True, bias=True)
    f = binding._CONVENIENCES["linear_lora_fused"]
    want = call_of(tvg.linear_lora_fused, p, activation="silu")
    assert torch.equal(call_of(f, p, activation="silu"), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = call_of(f, p, activation="silu", stream=side)
    side.synchronize()
    assert torch.equal(y, want)
