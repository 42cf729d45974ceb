"""The channels-last operators as a block uses them: norm with an activation, then a projection with adapters and the
residual, in a training step's and in a server's form, behind a convolution of the library."""
import pytest

pytestmark = pytest.mark.gpu


def test_block_behind_a_convolution(tvg):
    """conv (NCHW) -> rows -> x + project(silu(norm(x))), eager and as one graph, against 64 bits.  bf16 rounds after the
    convolution (the rows are the block's input), the norm and the sum: the norm's rounding, 2^-8 of each value, reaches
    y through the weights - four standard deviations of a sum of such errors."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    n, c, h = 3, 64, 14
    img, cw = r(n, 32, h, h).bfloat16(), (r(c, 32, 3, 3) * 0.06).bfloat16()
    one, zero = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
    gamma, beta, bias = r(c).abs() + 0.5, r(c) * 0.1, r(c) * 0.1
    w, a, b = (r(c, c) * 0.12).bfloat16(), (r(5, 8, c) * 0.12).bfloat16(), (r(5, c, 8) * 0.3).bfloat16()
    scale = torch.tensor([0.5, 1.0, 1.5, 2.0, 1.0], device="cuda")
    request = torch.tensor([4, -1, 2], dtype=torch.int32, device="cuda").repeat_interleave(h * h)

    def block():
        x = tvg.conv2d_fused(img, cw, one, zero, pad=1).permute(0, 2, 3, 1).contiguous()
        t = tvg.group_norm_fused(x, 8, gamma, beta, activation="silu")
        return x, tvg.linear_lora_fused(t, w, a, b, request, scale, bias, x)

    x, y = block()
    v = x.double().view(n, h * h, 8, c // 8)
    d = v - v.mean(dim=(1, 3), keepdim=True)
    z = (d / ((d * d).mean(dim=(1, 3), keepdim=True) + 1e-5).sqrt()).view(n * h * h, c) * gamma.double() + beta.double()
    t = z * torch.sigmoid(z)
    full = w.double().expand(n * h * h, c, c).clone()
    for i in range(5):
        full[request == i] += float(scale[i]) * (b[i].double() @ a[i].double())
    want = (full * t.unsqueeze(1)).sum(2) + bias.double() + x.double().view(-1, c)
    spread = ((full * t.unsqueeze(1)) ** 2).sum(2).sqrt()
    err = (y.double().view(-1, c) - want).abs()
    assert bool((err <= 4 * 2.0 ** -8 * spread + 2.0 ** -8 * want.abs() + 1e-3).all())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, captured = block()
    for _ in range(3):
        captured.fill_(float("nan"))
        graph.replay()
        _, again = block()
        torch.cuda.synchronize()
        assert torch.equal(captured, y) and torch.equal(again, y)


def test_single_tokens_have_the_prompts_result(tvg):
    """A server's two forms: the rows of a prompt one call at a time, and together.  fp32 sums in another order."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, w, a, b = r(70, 512), r(384, 512) * 0.04, r(3, 16, 512) * 0.04, r(3, 384, 16) * 0.25
    index = torch.randint(-1, 3, (70,), generator=g, device="cuda", dtype=torch.int32)
    whole = tvg.linear_lora_fused(x, w, a, b, index)
    rows = torch.cat([tvg.linear_lora_fused(x[i:i + 1], w, a, b, index[i:i + 1]) for i in range(70)])
    size = x.abs() @ w.abs().t() + (x.abs() @ a.abs().sum(0).t()) @ b.abs().sum(0).t()
    assert bool(((whole - rows).abs() <= 2 * (16 + 4 * 512 ** 0.5) * 2.0 ** -24 * size).all())
