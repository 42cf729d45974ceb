"""Projections of very many rows."""
import math

import pytest

pytestmark = pytest.mark.gpu

H = 2.0 ** -24


def check_some(y, x, w, a, b, index, at):
    """Rows `at` against 64 bits: sums of m products within (16 + 4 sqrt(m)) H of the sum of absolute ones (four standard
    deviations of roundings of one step), 2^-17 of the split of h, one rounding to bf16."""
    import torch
    xs, i = x[at].double(), index[at].long()
    own = (i >= 0) & (i < a.shape[0])
    want, size = xs @ w.double().t(), xs.abs() @ w.double().abs().t()
    tol = (16 + 4 * math.sqrt(x.shape[1])) * H * size
    for j in range(a.shape[0]):
        on = own & (i == j)
        h, hsize = xs[on] @ a[j].double().t(), xs[on].abs() @ a[j].double().abs().t()
        want[on] += h @ b[j].double().t()
        eh = (16 + 4 * math.sqrt(x.shape[1])) * H * hsize + 2.0 ** -17 * h.abs()
        tol[on] += eh @ b[j].double().abs().t() + (16 + 4 * math.sqrt(2 * a.shape[1])) * H * (h.abs() @ b[j].double().abs().t())
    assert bool(((y[at].double() - want).abs() <= tol + 2.0 ** -8 * want.abs() + 1e-37).all())


# A workgroup for every 16 rows and 16 ranks, more than 2^32 work items; x beyond 2^31 bytes, whose tiles keep the rows' order; many rows
# in the order of their adapters
@pytest.mark.parametrize("rows,c,k,rank", [(8500000, 3, 1, 256), (1100000, 1000, 64, 16), (200704, 64, 64, 16), (200704, 136, 264, 20)])
def test_many_rows(tvg, rows, c, k, rank):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows)
    r = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    x, w, a, b = r(rows, c), r(k, c) * c ** -0.5, r(3, rank, c) * c ** -0.5, r(3, k, rank) * rank ** -0.5
    index = torch.randint(-1, 4, (rows,), generator=g, device="cuda", dtype=torch.int32)
    y = tvg.linear_lora_fused(x, w, a, b, index)
    torch.cuda.synchronize()
    at = torch.cat([torch.arange(300, device="cuda"), torch.arange(rows - 300, rows, device="cuda"),
                    torch.randint(0, rows, (3000,), generator=g, device="cuda")])
    check_some(y, x, w, a, b, index, at)


@pytest.mark.parametrize("rows,c,k", [(3, (1 << 22) + 8, 5), (3, (1 << 23) + 3, 5), (40, (1 << 22) + 8, 70)])
def test_the_longest_rows(tvg, rows, c, k):
    """Rows of 8 MB and more are read at any element."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(c)
    r = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    x, w, a, b = r(rows, c), r(k, c) * c ** -0.5, r(3, 4, c) * c ** -0.5, r(3, k, 4)
    index = torch.randint(-1, 4, (rows,), generator=g, device="cuda", dtype=torch.int32)
    y = tvg.linear_lora_fused(x, w, a, b, index)
    torch.cuda.synchronize()
    check_some(y, x, w, a, b, index, torch.arange(rows, device="cuda"))
