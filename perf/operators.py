"""Performance cases of the channels-last operators: group norm with an activation, forward and backward, and the
projection with low-rank adapters of many requests.  A case's ``kind`` names the operator:

  norm       group norm of a channels-last map [n][h][w][c], then an activation
  norm_grad  its gradients for x, gamma and beta, from the saved statistics
  lora       y = act(x W^T + bias + scale_a B_a (A_a x) + residual) of rows [rows][c], the adapter chosen row by row

Values: maps as convolutions leave them (every channel with an offset and a spread of its own), gradients, tokens and
weights normal, gamma U[0.5, 1.5], beta and bias U[-0.1, 0.1].  Everything is made on the GPU from the seed.
"""
import math

import torch

own = False

DTYPES = {"f32": (torch.float32, 4), "bf16": (torch.bfloat16, 2)}

# The largest listed cases; drawn ones stay below.
MOST_FLOPS = 2.8e11
MOST_ELEMENTS = 2.1e8


def listed():
    return [
        # The deepest map of a network on one image: a few kilobytes, the latency of a call.
        dict(name="norm bf16 7x7x512", kind="norm", dtype="bf16", n=1, h=7, w=7, c=512, groups=32, act="silu", stats=False),
        # A batch of early maps in training: statistics kept for the backward pass.
        dict(name="norm bf16 56x56x256 batch 32", kind="norm", dtype="bf16", n=32, h=56, w=56, c=256, groups=32, act="silu",
             stats=True),
        # Full precision, a cropped map and groups of seven channels: nothing is a round number.
        dict(name="norm f32 45x37x84 batch 5", kind="norm", dtype="f32", n=5, h=45, w=37, c=84, groups=12, act="relu",
             stats=False),
        # Offline scoring: far larger than the caches.
        dict(name="norm bf16 112x112x256 batch 64", kind="norm", dtype="bf16", n=64, h=112, w=112, c=256, groups=32,
             act="silu", stats=False),
        # The backward pass of the training batch.
        dict(name="norm_grad bf16 56x56x256 batch 32", kind="norm_grad", dtype="bf16", n=32, h=56, w=56, c=256, groups=32,
             act="silu"),
        # Fine-tuning on two images in full precision.
        dict(name="norm_grad f32 14x14x256 batch 2", kind="norm_grad", dtype="f32", n=2, h=14, w=14, c=256, groups=16,
             act="none"),
        # One token of one request: the smallest call of a server.
        dict(name="lora bf16 1 row 1024", kind="lora", dtype="bf16", rows=1, c=1024, k=1024, rank=16, adapters=8, requests=1,
             act="none", bias=False, residual=False),
        # A full batch of single tokens, every row a request of its own.
        dict(name="lora bf16 64 rows 4096", kind="lora", dtype="bf16", rows=64, c=4096, k=4096, rank=16, adapters=32,
             requests=64, act="none", bias=False, residual=True),
        # Prompts of eight requests, packed: the large matrix product.
        dict(name="lora bf16 8192 rows 4096", kind="lora", dtype="bf16", rows=8192, c=4096, k=4096, rank=32, adapters=16,
             requests=8, act="none", bias=False, residual=False),
        # Prompts and single tokens in one batch, an expanding projection with its activation.
        dict(name="lora bf16 1200 rows 2048 to 8192", kind="lora", dtype="bf16", rows=1200, c=2048, k=8192, rank=64,
             adapters=24, requests=150, act="silu", bias=True, residual=False),
        # A pruned model: no extent is a multiple of anything wide.
        dict(name="lora bf16 777 rows 1000 to 515", kind="lora", dtype="bf16", rows=777, c=1000, k=515, rank=12, adapters=6,
             requests=20, act="relu", bias=True, residual=True),
        # Full precision.
        dict(name="lora f32 512 rows 1024 to 2048", kind="lora", dtype="f32", rows=512, c=1024, k=2048, rank=8, adapters=4,
             requests=12, act="none", bias=True, residual=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Widths of a model: three in four a multiple of 64 or 8, the others of any value."""
    v, kind = _log_int(rng, lo, hi), rng.random()
    step = 64 if kind < 0.5 else 8 if kind < 0.75 else 1
    return max(step, (v + step // 2) // step * step)


def draw(rng):
    while True:
        kind = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "lora", "lora", "lora", "lora"])
        dtype = rng.choice(["f32", "bf16", "bf16"])
        if kind == "lora":
            rows = _log_int(rng, 1, 8192)
            case = dict(kind=kind, dtype=dtype, rows=rows, c=_width(rng, 64, 8192), k=_width(rng, 64, 8192),
                        rank=rng.choice([4, 8, 8, 12, 16, 16, 32, 64]), adapters=_log_int(rng, 1, 48),
                        requests=min(rows, _log_int(rng, 1, 256)), act=rng.choice(["none", "none", "relu", "silu"]),
                        bias=rng.random() < 0.4, residual=rng.random() < 0.4)
            # (full precision has an eighth of the matrix rate or less)
            if work(case)["flops"] > MOST_FLOPS / (1 if dtype == "bf16" else 8):
                continue
        else:
            h = _log_int(rng, 1, 112)
            groups = rng.choice([1, 4, 8, 12, 16, 32, 32, 32])
            case = dict(kind=kind, dtype=dtype, n=_log_int(rng, 1, 64), h=h,
                        w=h if rng.random() < 0.5 else _log_int(rng, 1, 112), c=groups * _log_int(rng, 1, 40), groups=groups,
                        act=rng.choice(["none", "silu", "silu"] + ["relu"] * (kind == "norm")))
            if kind == "norm":
                case["stats"] = rng.random() < 0.5
            # (a group of fewer elements has no statistics to speak of)
            if case["h"] * case["w"] * case["c"] // groups < 16:
                continue
            if case["n"] * case["h"] * case["w"] * case["c"] > MOST_ELEMENTS / (1 if kind == "norm" else 2):
                continue
        return case


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

class _Maker:
    def __init__(self, seed, dtype):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.dtype = DTYPES[dtype][0]

    def uniform(self, shape, lo, hi):
        return torch.rand(shape, generator=self.gen, device="cuda") * (hi - lo) + lo

    def normal(self, shape, spread=1.0):
        return (torch.randn(shape, generator=self.gen, device="cuda") * spread).to(self.dtype)


def _norm_inputs(case, seed):
    m = _Maker(seed, case["dtype"])
    shape, c = (case["n"], case["h"], case["w"], case["c"]), case["c"]
    spread, offset = m.uniform((c,), 0.5, 2.0), m.uniform((c,), -1.0, 1.0)
    x = (torch.randn(shape, generator=m.gen, device="cuda") * spread + offset).to(m.dtype)
    state = dict(x=x, gamma=m.uniform((c,), 0.5, 1.5), beta=m.uniform((c,), -0.1, 0.1), eps=1e-5)
    if case["kind"] == "norm_grad":
        state["dy"] = m.normal(shape)
        # what the forward pass left, in the precision it keeps them in
        stats = [], []
        for xi in x:
            v = xi.double().view(-1, case["groups"], c // case["groups"])
            stats[0].append(v.mean(dim=(0, 2)))
            stats[1].append((v.var(dim=(0, 2), unbiased=False) + state["eps"]).rsqrt())
        state["mean"], state["rstd"] = (torch.stack(s).float() for s in stats)
    return state


def _lora_inputs(case, seed):
    m = _Maker(seed, case["dtype"])
    rows, c, k, r, n = (case[f] for f in ("rows", "c", "k", "rank", "adapters"))
    state = dict(x=m.normal((rows, c)), w=m.normal((k, c), c ** -0.5), a=m.normal((n, r, c), c ** -0.5),
                 b=m.normal((n, k, r), 0.5 * r ** -0.5), scale=m.uniform((n,), 0.5, 2.0))
    # Requests of different lengths, one row at least each, every one with an adapter; one in ten goes without.
    cuts = torch.randperm(rows - 1, generator=m.gen, device="cuda")[:case["requests"] - 1] + 1 if rows > 1 else None
    request = torch.zeros(rows, dtype=torch.long, device="cuda")
    if cuts is not None:
        request[cuts] = 1
    request = request.cumsum(0)
    of = torch.randint(0, n, (case["requests"],), generator=m.gen, device="cuda", dtype=torch.int32)
    without = m.uniform((case["requests"],), 0.0, 1.0) < 0.1
    state["adapter"] = torch.where(without & (case["requests"] > 1), torch.full_like(of, -1), of)[request].contiguous()
    state["bias"] = m.uniform((k,), -0.1, 0.1) if case["bias"] else None
    state["residual"] = m.normal((rows, k)) if case["residual"] else None
    return state


def _inputs(case, seed):
    return (_lora_inputs if case["kind"] == "lora" else _norm_inputs)(case, seed)


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    return state


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------

def _activate(t, act):
    return torch.relu(t) if act == "relu" else t * torch.sigmoid(t) if act == "silu" else t


def _plain_norm(s, case):
    n, g = case["n"], case["groups"]
    x = s["x"].float().view(n, -1, g, case["c"] // g)
    mean = x.mean(dim=(1, 3), keepdim=True)
    centred = x - mean
    rstd = ((centred * centred).mean(dim=(1, 3), keepdim=True) + s["eps"]).rsqrt()
    z = (centred * rstd).view(s["x"].shape) * s["gamma"] + s["beta"]
    y = _activate(z, case["act"]).to(s["x"].dtype)
    return [y, mean.view(n, g), rstd.view(n, g)] if case["stats"] else [y]


def _plain_norm_grad(s, case):
    n, g, c = case["n"], case["groups"], case["c"]
    split = (n, -1, g, c // g)
    gamma, beta = s["gamma"].view(g, -1), s["beta"].view(g, -1)
    rstd = s["rstd"].view(n, 1, g, 1)
    xhat = (s["x"].float().view(split) - s["mean"].view(n, 1, g, 1)) * rstd
    dz = s["dy"].float().view(split)
    if case["act"] == "silu":
        z = xhat * gamma + beta
        sig = torch.sigmoid(z)
        dz = dz * (sig * (1.0 + z * (1.0 - sig)))
    s1, s2 = dz.sum(dim=1), (dz * xhat).sum(dim=1)
    m = s["x"][0].numel() // g
    a = (gamma * s1).sum(dim=2).view(n, 1, g, 1) / m
    b = (gamma * s2).sum(dim=2).view(n, 1, g, 1) / m
    dx = rstd * (gamma * dz - a - xhat * b)
    return [dx.view(s["x"].shape).to(s["x"].dtype), s2.sum(dim=0).view(c), s1.sum(dim=0).view(c)]


def _plain_lora(s, case):
    rows, n, r = case["rows"], case["adapters"], case["rank"]
    x = s["x"].float()
    y = x @ s["w"].float().t()
    if s["bias"] is not None:
        y = y + s["bias"]
    # every row through every adapter, all but its own taken out
    h = (x @ s["a"].float().view(n * r, -1).t()).view(rows, n, r)
    mine = (s["adapter"].view(rows, 1) == torch.arange(n, device=x.device, dtype=torch.int32)).float() * s["scale"]
    h = (h * mine.view(rows, n, 1)).view(rows, n * r)
    y = y + h @ s["b"].float().permute(0, 2, 1).reshape(n * r, -1)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return _activate(y, case["act"]).to(s["x"].dtype)


def _run_own(s, case):
    import paper_1802_04799_amd as tvg
    act = None if case["act"] == "none" else case["act"]
    if case["kind"] == "norm":
        y = tvg.group_norm_fused(s["x"], case["groups"], s["gamma"], s["beta"], eps=s["eps"], activation=act,
                                 stats=case["stats"])
        return list(y) if case["stats"] else [y]
    if case["kind"] == "norm_grad":
        return list(tvg.group_norm_fused_backward(s["x"], s["dy"], s["mean"], s["rstd"], case["groups"], s["gamma"],
                                                  s["beta"], activation=act))
    return [tvg.linear_lora_fused(s["x"], s["w"], s["a"], s["b"], s["adapter"], s["scale"], s["bias"], s["residual"],
                                  activation=act)]


def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    if case["kind"] == "norm":
        return _plain_norm(state, case)
    if case["kind"] == "norm_grad":
        return _plain_norm_grad(state, case)
    return [_plain_lora(state, case)]


def work(case):
    """Inputs read once, outputs written once; of the adapters, as many as the requests can have between them."""
    size = DTYPES[case["dtype"]][1]
    if case["kind"] == "lora":
        rows, c, k, r = case["rows"], case["c"], case["k"], case["rank"]
        used = min(case["adapters"], case["requests"])
        elements = rows * c + k * c + used * r * (c + k) + rows * k * (2 if case["residual"] else 1)
        return {"bytes": elements * size + 4 * (rows + case["adapters"] + (k if case["bias"] else 0)),
                "flops": 2 * rows * c * k + 2 * rows * r * (c + k)}
    elements, c = case["n"] * case["h"] * case["w"] * case["c"], case["c"]
    stats = 8 * case["n"] * case["groups"]
    if case["kind"] == "norm":
        return {"bytes": 2 * elements * size + 8 * c + (stats if case["stats"] else 0), "flops": 10 * elements}
    return {"bytes": 3 * elements * size + 16 * c + stats, "flops": 20 * elements}


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits, sample by sample and request by request
# ------------------------------------------------------------------------------------------------

def _exact_activation(z, act):
    if act == "relu":
        return z.clamp(min=0.0)
    return z / (1.0 + torch.exp(-z)) if act == "silu" else z


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "lora":
        x, w = s["x"].double(), s["w"].double()
        y = torch.empty((case["rows"], case["k"]), dtype=torch.float64, device="cuda")
        for lo in range(0, case["rows"], 1024):
            y[lo:lo + 1024] = torch.mm(x[lo:lo + 1024], w.t())
        for i in range(case["adapters"]):
            at = (s["adapter"] == i).nonzero().flatten()
            if at.numel():
                low = torch.mm(x[at], s["a"][i].double().t())
                y[at] += s["scale"][i].double() * torch.mm(low, s["b"][i].double().t())
        if s["bias"] is not None:
            y += s["bias"].double()
        if s["residual"] is not None:
            y += s["residual"].double()
        return [_exact_activation(y, case["act"])]
    groups, c = case["groups"], case["c"]
    gamma, beta = s["gamma"].double(), s["beta"].double()
    of = torch.arange(c, device="cuda") // (c // groups)          # the group of a channel
    count = case["h"] * case["w"] * (c // groups)

    def per_group(per_channel):
        return torch.zeros(groups, dtype=torch.float64, device="cuda").index_add_(0, of, per_channel)

    if case["kind"] == "norm":
        ys, means, rstds = [], [], []
        for image in s["x"]:
            v = image.double().reshape(-1, c)
            mean = per_group(v.sum(0)) / count
            d = v - mean[of]
            rstd = 1.0 / torch.sqrt(per_group((d * d).sum(0)) / count + s["eps"])
            ys.append(_exact_activation(d * rstd[of] * gamma + beta, case["act"]).reshape(image.shape))
            means.append(mean)
            rstds.append(rstd)
        y = torch.stack(ys)
        return [y, torch.stack(means), torch.stack(rstds)] if case["stats"] else [y]
    dgamma, dbeta, dxs = torch.zeros_like(gamma), torch.zeros_like(beta), []
    for i in range(case["n"]):
        rstd = s["rstd"][i].double()[of]
        xhat = (s["x"][i].double().reshape(-1, c) - s["mean"][i].double()[of]) * rstd
        dz = s["dy"][i].double().reshape(-1, c)
        if case["act"] == "silu":
            z = xhat * gamma + beta
            e = torch.exp(-z)
            dz = dz * ((1.0 + e + z * e) / (1.0 + e) ** 2)
        s1, s2 = dz.sum(0), (dz * xhat).sum(0)
        dgamma += s2
        dbeta += s1
        a, b = per_group(gamma * s1) / count, per_group(gamma * s2) / count
        dxs.append((rstd * (gamma * dz - a[of] - xhat * b[of])).reshape(s["x"][i].shape))
    return [torch.stack(dxs), dgamma, dbeta]
