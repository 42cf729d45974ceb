"""Refusals of the channels-last operators, on the host: through the C entry points (no device pointer is touched) and
through the Python calls (torch's fake device tensors)."""
import ctypes

import pytest

import paper_1802_04799_amd as tvg
from test_call_path import outcome

FAKE = 0x1000
NAN, INF = float("nan"), float("inf")


def norm(**kw):
    d = dict(n=2, pixels=49, c=64, groups=8, dtype=tvg.TVG_BF16, activation=tvg.TVG_ACT_SILU, eps=1e-5, flags=0)
    d.update(kw)
    return tvg.GroupNormDesc(*d.values())


def lora(**kw):
    d = dict(rows=8, c=64, k=96, adapters=4, rank=16, dtype=tvg.TVG_BF16, activation=0, flags=0)
    d.update(kw)
    return tvg.LinearLoraDesc(*d.values())


def test_struct_layouts():
    assert ctypes.sizeof(tvg.GroupNormDesc) == 32 and ctypes.sizeof(tvg.LinearLoraDesc) == 32


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), 2), (dict(pixels=0), 2), (dict(c=0), 2), (dict(groups=0), 2), (dict(groups=-8), 2), (dict(groups=7), 2),
    (dict(groups=128), 2), (dict(n=-1), 2), (dict(eps=-1e-9), 2), (dict(eps=NAN), 2), (dict(eps=INF), 2),
    (dict(dtype=2), 3), (dict(activation=3), 3), (dict(activation=-1), 3), (dict(flags=1), 3),
    (dict(n=1 << 18, pixels=1, c=8), 3), (dict(n=1, pixels=1 << 30, c=1, groups=1), 3), (dict(n=1, pixels=1, c=1 << 20), 3),
    (dict(n=1 << 14, pixels=1 << 14, c=8), 3)])
def test_norm_refuses(kw, status):
    d = norm(**kw)
    for query in (tvg.tvg_group_norm_workspace_size, tvg.tvg_group_norm_backward_workspace_size):
        with pytest.raises(tvg.TvgError) as e:
            query(d)
        assert e.value.status == status
    assert tvg.tvg_group_norm_fused(d, FAKE, None, None, FAKE, None, None, FAKE, 1 << 40, 0) == status
    assert tvg.tvg_group_norm_fused_backward(d, *[FAKE] * 9, FAKE, 1 << 40, 0) == status


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), 2), (dict(c=0), 2), (dict(k=0), 2), (dict(adapters=-1), 2), (dict(rank=0), 2), (dict(rank=257), 3),
    (dict(dtype=5), 3), (dict(activation=9), 3), (dict(flags=2), 3), (dict(rows=1 << 24), 3), (dict(c=1 << 24, k=1), 3),
    (dict(rows=1 << 20, c=4096), 3), (dict(k=1 << 20, c=4096), 3), (dict(adapters=1 << 20, c=1024, rank=8), 3),
    (dict(rows=1 << 20, k=4096), 3), (dict(adapters=1 << 22, k=1024, c=1, rank=8), 3)])
def test_projection_refuses(kw, status):
    d = lora(**kw)
    with pytest.raises(tvg.TvgError) as e:
        tvg.tvg_linear_lora_workspace_size(d)
    assert e.value.status == status
    assert tvg.tvg_linear_lora_fused(d, *[FAKE] * 9, FAKE, 1 << 40, 0) == status


def test_pointers_workspaces_and_alignment():
    d = norm()
    need, back = tvg.tvg_group_norm_workspace_size(d), tvg.tvg_group_norm_backward_workspace_size(d)
    p = FAKE
    assert tvg.tvg_group_norm_fused(None or d, 0, p, p, p, p, p, p, need, 0) == 1
    assert tvg.tvg_group_norm_fused(d, p, p, p, 0, p, p, p, need, 0) == 1
    assert tvg.tvg_group_norm_fused(d, p + 1, p, p, p, p, p, p, need, 0) == 3
    assert tvg.tvg_group_norm_fused(d, p, p + 2, p, p, p, p, p, need, 0) == 3
    for at in range(5):                                        # x, dy, mean, rstd, (gamma, beta optional), dx
        args = [p] * 9
        args[at if at < 4 else 6] = 0
        assert tvg.tvg_group_norm_fused_backward(d, *args, p, back, 0) == 1
    for ws, size in ((0, back), (p + 128, back), (p, back - 1)):
        assert tvg.tvg_group_norm_fused_backward(d, *[p] * 9, ws, size, 0) == 4
    d = norm(n=64, pixels=12544, c=256, groups=32)             # (a map that one launch cannot take)
    need = tvg.tvg_group_norm_workspace_size(d)
    assert need > 0
    for ws, size in ((0, need), (p + 128, need), (p, need - 1)):
        assert tvg.tvg_group_norm_fused(d, *[p] * 6, ws, size, 0) == 4
    d = lora()
    need = tvg.tvg_linear_lora_workspace_size(d)
    for at in (0, 1, 2, 3, 4, 8):
        args = [p] * 9
        args[at] = 0
        assert tvg.tvg_linear_lora_fused(d, *args, p, need, 0) == 1
    assert tvg.tvg_linear_lora_fused(d, p, p, p, p, p + 2, p, p, p, p, p, need, 0) == 3
    assert tvg.tvg_linear_lora_fused(d, p, p, p, p, p, p, p, p, p + 1, p, need, 0) == 3
    for ws, size in ((0, need), (p + 128, need), (p, need - 1)):
        assert tvg.tvg_linear_lora_fused(d, *[p] * 9, ws, size, 0) == 4
    assert tvg.tvg_linear_lora_fused(lora(rows=0), *[0] * 9, 0, 0, 0) == 0          # nothing to do
    assert tvg.tvg_linear_lora_workspace_size(lora(rows=0)) == 0
    assert tvg.tvg_linear_lora_workspace_size(lora(adapters=0)) < need
    lib = tvg.load()
    assert lib.tvg_group_norm_workspace_size(None, ctypes.byref(ctypes.c_size_t())) == 1
    assert lib.tvg_linear_lora_workspace_size(ctypes.byref(d), None) == 1
    assert lib.tvg_linear_lora_fused(None, *[p] * 10, 0, None) == 1


def test_a_descriptor_of_another_operator_is_refused():
    with pytest.raises(TypeError):
        tvg.tvg_group_norm_fused(lora(), *[FAKE] * 6)
    with pytest.raises(TypeError):
        tvg.tvg_linear_lora_fused(norm(), *[FAKE] * 9)


def test_python_calls_refuse():
    cases = [
        ("tvg.group_norm_fused(y, 3, stream=0)", "TvgError"), ("tvg.group_norm_fused(y, 0, stream=0)", "TvgError"),
        ("tvg.group_norm_fused(y, 4, g[:7], stream=0)", "ValueError gamma"),
        ("tvg.group_norm_fused(y, 4, g.bfloat16(), stream=0)", "TypeError gamma"),
        ("tvg.group_norm_fused(y, 4, g, g, activation='gelu', stream=0)", "ValueError activation"),
        ("tvg.group_norm_fused(y.transpose(1, 2), 4, stream=0)", "ValueError x must be contiguous"),
        ("tvg.group_norm_fused(torch.zeros(2, 5, 5, 8), 4, stream=0)", "ValueError x must be a device"),
        ("tvg.group_norm_fused(y.half(), 4, stream=0)", "TypeError unsupported"),
        ("tvg.group_norm_fused(g, 4, stream=0)", "ValueError x must be"),
        ("tvg.group_norm_fused(y, 4, eps=float('nan'), stream=0)", "TvgError"),
        ("tvg.group_norm_fused(y, 4, out=y[:1], workspace=ws, stream=0)", "ValueError out is too small"),
        ("tvg.group_norm_fused(y, 4, workspace=torch.zeros(1 << 20), stream=0)", "ValueError workspace"),
        ("tvg.group_norm_fused_backward(y, y[:1], m, m, 4, stream=0)", "ValueError dy"),
        ("tvg.group_norm_fused_backward(y, y.bfloat16(), m, m, 4, stream=0)", "TypeError dy"),
        ("tvg.group_norm_fused_backward(y, y, m, m[:1], 4, stream=0)", "ValueError rstd"),
        ("tvg.group_norm_fused_backward(y, y, None, m, 4, stream=0)", "ValueError mean"),
        ("tvg.linear_lora_fused(r, w2, a, b, i[:5], stream=0)", "ValueError adapter"),
        ("tvg.linear_lora_fused(r, w2, a, b, i.long(), stream=0)", "TypeError adapter"),
        ("tvg.linear_lora_fused(r, w2, a, None, i, stream=0)", "ValueError b"),
        ("tvg.linear_lora_fused(r, w2, a, b[:, :5], i, stream=0)", "ValueError b"),
        ("tvg.linear_lora_fused(r, w2[:, :7], a, b, i, stream=0)", "ValueError w"),
        ("tvg.linear_lora_fused(r, w2, a, b, i, g[:1], stream=0)", "ValueError scale"),
        ("tvg.linear_lora_fused(r, w2, a, b, i, None, g, stream=0)", "ValueError bias"),
        ("tvg.linear_lora_fused(r, w2, a, b, i, residual=r, stream=0)", "ValueError residual"),
        ("tvg.linear_lora_fused(r, w2, a, b, i, activation=1, stream=0)", "ValueError activation"),
        ("tvg.linear_lora_fused(r, w2.bfloat16(), a, b, i, stream=0)", "TypeError w"),
        # whole and well: as far as the fake tensors' NULL address
        ("tvg.group_norm_fused(y, 4, g, g, out=y, workspace=ws, stream=0)", "TvgError tvg_group_norm_fused: a required pointer"),
        ("tvg.group_norm_fused_backward(y, y, m, m, 4, out=y, workspace=ws, stream=0)",
         "TvgError tvg_group_norm_fused_backward: a required pointer"),
        ("tvg.linear_lora_fused(r, w2, a, b, i, out=dev(6, 24), workspace=ws, stream=0)", "TvgError tvg_linear_lora_fused: a required pointer"),
    ]
    made = """
y, g, m = dev(2, 5, 5, 8), dev(8), dev(2, 4)
r, w2, a, b, i = dev(6, 8), dev(24, 8), dev(3, 4, 8), dev(3, 24, 4), dev(6, dtype=torch.int32)
"""
    got = outcome(made + "\n".join(f"outcome(lambda: {call})" for call, _ in cases))
    assert len(got) == len(cases)
    for (call, want), line in zip(cases, got):
        assert line.startswith(want), (call, line)
