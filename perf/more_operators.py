"""A mixture of experts around an 8-bit KAN layer, from the router's choices to the tokens' sums, and its products on 8-bit integers: the
sizes that programs call the operators at, each beside its plain form (elementary torch operations in 32 bits) and what a 64-bit
evaluation returns.

A case names the operator (op), its sizes and its types:
  sort      the choices [tokens, top] sorted by expert: the token of every sorted row, every choice's place, the groups' sizes; `skew` is
            the spread of the experts' popularity (in nats), `dropped` the share of tokens without an expert (padding, capacity)
  combine   the experts' rows [tokens * top, width] of type `y` back in the tokens' order, weighted ("weights": "none": unweighted), out
            in `out`; "train": with the gradients of the rows and of the weights
  norm      the residual's addition and the root-mean-square norm of [rows, width], out in 8-bit integers with a scale for each row
  weights   weights [experts, outputs, inputs] (experts 0: one matrix, or a batch of activations) to 8-bit integers with a scale for each
            output (token)
  product   [rows, inputs] times [outputs, inputs] transposed, both in 8-bit integers with their scales, out in `out`
  experts   the same product grouped by expert, the rows gathered
"""
from __future__ import annotations

import math

import torch

own = False          # False: the plain forms; True: this package's operators

LARGEST = 127.0      # the largest code
SMALLEST_SCALE = 2.0 ** -126
EPS = 1e-6
_TYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2, "none": 0}
_PRODUCT_MOST = 2.0 * 8192 * 4096 * 4096
_EXPERTS_MOST = 2.0 * 16384 * 2048 * 1024


def listed():
    return [
        # one token of a decoding step: latency
        {"name": "sort_token", "op": "sort", "tokens": 1, "top": 2, "experts": 8, "skew": 0.5, "dropped": 0.0},
        # a training batch over many experts, some of its tokens padding
        {"name": "sort_65536", "op": "sort", "tokens": 65536, "top": 8, "experts": 64, "skew": 0.5, "dropped": 0.1},
        # a server's decoding step, 32-bit rows as a table layer hands them on
        {"name": "combine_16", "op": "combine", "tokens": 16, "top": 2, "width": 1024, "experts": 8, "y": "f32", "weights": "f32", "out": "bf16",
         "skew": 1.0, "dropped": 0.0, "train": False},
        # an irregular width and number of choices, in training, some tokens without an expert
        {"name": "combine_ragged_1000", "op": "combine", "tokens": 1000, "top": 3, "width": 300, "experts": 12, "y": "f32", "weights": "f32", "out": "f32",
         "skew": 1.0, "dropped": 0.1, "train": True},
        # a training batch's largest
        {"name": "combine_16384", "op": "combine", "tokens": 16384, "top": 4, "width": 2048, "experts": 32, "y": "bf16", "weights": "f32", "out": "bf16",
         "skew": 0.5, "dropped": 0.0, "train": True},
        # one token of a decoding step in front of a 1024-wide layer: latency
        {"name": "norm_token", "op": "norm", "rows": 1, "width": 1024, "x": "bf16", "residual": "bf16", "strided": False},
        # the widest layer's largest batch
        {"name": "norm_32768", "op": "norm", "rows": 32768, "width": 1024, "x": "bf16", "residual": "bf16", "strided": False},
        # a few irregular experts in 32 bits, converted as a model is loaded
        {"name": "weights_ragged", "op": "weights", "experts": 8, "outputs": 300, "inputs": 200, "x": "f32"},
        # a server's decoding step: the weights' bytes
        {"name": "product_16", "op": "product", "rows": 16, "inputs": 4096, "outputs": 4096, "out": "bf16"},
        # a long prompt or a training-size batch: the matrix cores
        {"name": "product_8192", "op": "product", "rows": 8192, "inputs": 4096, "outputs": 4096, "out": "bf16"},
        # irregular experts, ragged groups, 32 bits out for a table layer behind them
        {"name": "experts_ragged", "op": "experts", "tokens": 500, "top": 3, "experts": 12, "inputs": 200, "outputs": 300,
         "out": "f32", "skew": 1.0},
        # a long prompt through many experts
        {"name": "experts_8192", "op": "experts", "tokens": 8192, "top": 2, "experts": 32, "inputs": 2048, "outputs": 1024,
         "out": "bf16", "skew": 0.5},
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):                                # half of them whole pieces of 16 or 128, half whatever comes
        w = log_int(lo, hi)
        step = rng.choice([1, 1, 16, 128])
        return max(lo, w // step * step) if w >= step else w

    op = rng.choice(["sort", "combine", "combine", "norm", "weights", "product", "product", "experts", "experts"])
    if op == "sort":
        experts = log_int(2, 256)
        top = min(rng.randint(1, 8), experts)
        return {"op": op, "tokens": max(1, min(log_int(1, 65536), (1 << 24) // experts, (1 << 19) // top)), "top": top, "experts": experts,
                "skew": rng.choice([0.0, 0.5, 1.0, 2.0]), "dropped": rng.choice([0.0, 0.1, 0.6])}
    if op == "combine":
        w, experts = width(8, 8192), log_int(2, 64)
        top = min(rng.randint(1, 8), experts)
        return {"op": op, "tokens": max(1, min(log_int(1, 16384), (1 << 26) // (w * top))), "top": top, "width": w, "experts": experts,
                "y": rng.choice(sorted(_TYPE)), "weights": rng.choice(sorted(_TYPE) + ["none"]), "out": rng.choice(sorted(_TYPE)),
                "skew": rng.choice([0.0, 0.5, 1.0]), "dropped": rng.choice([0.0, 0.1]), "train": rng.random() < 0.6}
    if op == "norm":
        w = width(8, 8192)
        return {"op": op, "rows": max(1, min(log_int(1, 32768), (1 << 25) // w)), "width": w, "x": rng.choice(sorted(_TYPE)),
                "residual": rng.choice(sorted(_TYPE) + ["none"]), "strided": rng.random() < 0.25}
    if op == "weights":
        outputs, inputs = width(16, 4096), width(16, 8192)
        experts = min(rng.choice([0, 0, 2, 8, 16]), (1 << 24) // (outputs * inputs))
        return {"op": op, "experts": experts, "outputs": outputs, "inputs": inputs, "x": rng.choice(sorted(_TYPE))}
    if op == "product":
        inputs, outputs = width(16, 8192), width(2, 8192)
        outputs = max(1, min(outputs, (1 << 25) // inputs))
        rows = min(log_int(1, 32768), (1 << 25) // max(inputs, outputs), int(_PRODUCT_MOST / (2.0 * inputs * outputs)))
        return {"op": op, "rows": max(1, rows), "inputs": inputs, "outputs": outputs, "out": rng.choice(sorted(_TYPE))}
    inputs, outputs, experts, top = width(16, 4096), width(16, 4096), rng.randint(2, 64), rng.randint(1, 4)
    outputs = max(1, min(outputs, (1 << 26) // (inputs * experts)))
    rows = min(log_int(1, 8192) * top, (1 << 24) // max(inputs, outputs), int(_EXPERTS_MOST / (4.0 * inputs * outputs)))
    return {"op": op, "tokens": max(1, rows // top), "top": min(top, experts), "experts": experts, "inputs": inputs, "outputs": outputs,
            "out": rng.choice(sorted(_TYPE)), "skew": rng.choice([0.0, 0.5, 1.0])}


# ---- inputs ------------------------------------------------------------------------------------------------------
def _codes(v):
    """int8 codes and a scale for each row of v [..., n] in 32 bits."""
    scales = (v.abs().amax(dim=-1) / LARGEST).clamp(min=SMALLEST_SCALE)
    return torch.round(v / scales[..., None]).to(torch.int8), scales


def _values(codes, scales):
    """What codes stand for, in 16 bits: a value at the border between two codes may fall to either side."""
    return codes * scales[..., None].bfloat16()


def _sorted_choices(expert, experts):
    """(token of every sorted row, place of every choice, sizes): choices without an expert come last and have no place."""
    flat, top = expert.flatten(), expert.shape[1]
    key = torch.where((flat >= 0) & (flat < experts), flat, experts)
    order = torch.sort(key, stable=True).indices
    at = torch.arange(flat.numel(), device=flat.device)
    sizes = torch.zeros(experts + 1, dtype=torch.int64, device=flat.device).scatter_add_(0, key, torch.ones_like(key))
    held = flat.numel() - sizes[experts]
    places = torch.empty_like(order).scatter_(0, order, at)
    rows = torch.where(at < held, order // top, -1)
    places = torch.where(key < experts, places, -1).view(expert.shape)
    return rows.int(), places.int(), sizes[:experts].int()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def activations(rows, width):                     # channels of different size, as a model's are
        return normal(rows, width) * torch.exp(0.7 * normal(width))

    def routed(tokens, experts, top, skew, dropped):  # the router's probabilities and choices
        logits = normal(tokens, experts) + skew * normal(experts)
        p, expert = torch.softmax(logits, dim=1).topk(top, dim=1)
        gone = torch.rand(tokens, generator=g, device="cuda") < dropped
        return p, torch.where(gone[:, None], -1, expert)

    op = case["op"]
    if op == "sort":
        _, expert = routed(case["tokens"], case["experts"], case["top"], case["skew"], case["dropped"])
        return {"op": op, "expert": expert, "experts": case["experts"]}
    if op == "combine":
        p, expert = routed(case["tokens"], case["experts"], case["top"], case["skew"], case["dropped"])
        rows, places, _ = _sorted_choices(expert, case["experts"])
        weights = None if case["weights"] == "none" else p.to(_TYPE[case["weights"]])
        out = _TYPE[case["out"]]
        return {"op": op, "y": activations(rows.numel(), case["width"]).to(_TYPE[case["y"]]), "rows": rows, "places": places, "weights": weights,
                "out": out, "grad": normal(case["tokens"], case["width"]).to(out) if case["train"] else None}
    if op == "norm":
        rows, width = case["rows"], case["width"]
        x = activations(rows, width + 24 if case["strided"] else width).to(_TYPE[case["x"]])[:, :width]
        residual = None if case["residual"] == "none" else (3.0 * activations(rows, width)).to(_TYPE[case["residual"]])
        return {"op": op, "x": x, "residual": residual, "weight": (1.0 + 0.2 * normal(width)).to(x.dtype)}
    if op == "weights":
        shape = ([case["experts"]] if case["experts"] else []) + [case["outputs"], case["inputs"]]
        return {"op": op, "weight": (normal(*shape) / math.sqrt(case["inputs"])).to(_TYPE[case["x"]])}
    shape = ([case["experts"]] if op == "experts" else []) + [case["outputs"], case["inputs"]]
    rows = case["tokens"] if op == "experts" else case["rows"]
    state = {"op": op, "out": _TYPE[case["out"]]}
    state["x"], state["x_scales"] = _codes(activations(rows, case["inputs"]))
    state["weight"], state["weight_scales"] = _codes(normal(*shape) / math.sqrt(case["inputs"]))
    if op == "experts":
        _, expert = routed(rows, case["experts"], case["top"], case["skew"], 0.0)
        state["rows"], _, state["group_sizes"] = _sorted_choices(expert, case["experts"])
    return state


# ---- one pass ----------------------------------------------------------------------------------------------------
def _plain_combine(y, places, weights, out):
    held = (places >= 0) & (places < y.shape[0])
    v = y.float()[places.long().clamp(0, y.shape[0] - 1)]                     # [tokens, top, width]
    v = torch.where(held[..., None], v if weights is None else v * weights.float()[..., None], 0.0)
    return v.sum(dim=1).to(out)


def _plain_combine_gradients(grad, y, places, weights):
    tokens, top = places.shape
    held = (places >= 0) & (places < y.shape[0])
    choice = torch.arange(tokens * top, device=y.device)
    owner = torch.full((y.shape[0] + 1,), -1, dtype=torch.int64, device=y.device)         # the choice behind every row; the last: dropped ones
    owner.scatter_(0, torch.where(held, places.long(), y.shape[0]).flatten(), choice)
    owner = owner[:-1]
    g = grad.float()[owner.clamp(min=0) // top]
    if weights is not None:
        g = g * weights.float().flatten()[owner.clamp(min=0), None]
    grad_y = torch.where(owner[:, None] >= 0, g, 0.0).to(y.dtype)
    if weights is None:
        return grad_y, None
    dot = (y.float()[places.long().clamp(0, y.shape[0] - 1)] * grad.float()[:, None, :]).sum(dim=2)
    return grad_y, torch.where(held, dot, 0.0).to(weights.dtype)


def _plain_norm(x, weight, residual):
    h = x.float() if residual is None else x.float() + residual.float()
    y = h * torch.rsqrt(h.square().mean(dim=-1, keepdim=True) + EPS) * weight.float()
    return *_codes(y), None if residual is None else h.to(residual.dtype)


def _plain_product(x, x_scales, weight, weight_scales, out):
    return (torch.matmul(x.float(), weight.float().t()) * x_scales[:, None] * weight_scales).to(out)


def _plain_experts(x, x_scales, weight, weight_scales, group_sizes, rows, out):
    """All experts as one batched product: every group is padded to the largest."""
    ends = group_sizes.long().cumsum(0)
    at = torch.arange(rows.numel(), device=x.device)
    group = torch.searchsorted(ends, at, right=True)
    place = at - (ends - group_sizes)[group]
    padded = torch.zeros((group_sizes.numel(), int(group_sizes.max()), x.shape[1]), device=x.device)
    padded[group, place] = x.float()[rows.long()]
    y = torch.bmm(padded, weight.float().transpose(1, 2).contiguous())
    return (y[group, place] * x_scales[rows.long(), None] * weight_scales[group]).to(out)


def run(state):
    s = state
    if own:
        import paper_2601_03332_amd as lk
        if s["op"] == "sort":
            return lk.lutkan_expert_sort(s["expert"], s["experts"])
        if s["op"] == "combine":
            out = lk.lutkan_expert_combine(s["y"], s["places"], s["weights"], dtype=s["out"])
            if s["grad"] is None:
                return out
            return out, *lk.lutkan_expert_combine_backward(s["grad"], s["y"], s["rows"], s["places"], s["weights"])
        if s["op"] == "norm":
            codes, scales, residual = lk.lutkan_rmsnorm_int8(s["x"], s["weight"], residual=s["residual"], eps=EPS)
            return _values(codes, scales), scales, residual
        if s["op"] == "weights":
            codes, scales = lk.lutkan_quantise_int8(s["weight"])
            return _values(codes, scales), scales
        if s["op"] == "product":
            return lk.lutkan_matmul_int8(s["x"], s["x_scales"], s["weight"], s["weight_scales"], dtype=s["out"])
        return lk.lutkan_grouped_matmul_int8(s["x"], s["x_scales"], s["weight"], s["weight_scales"], s["group_sizes"], rows=s["rows"],
                                             dtype=s["out"])
    if s["op"] == "sort":
        return _sorted_choices(s["expert"], s["experts"])
    if s["op"] == "combine":
        out = _plain_combine(s["y"], s["places"], s["weights"], s["out"])
        if s["grad"] is None:
            return out
        return out, *_plain_combine_gradients(s["grad"], s["y"], s["places"], s["weights"])
    if s["op"] == "norm":
        codes, scales, residual = _plain_norm(s["x"], s["weight"], s["residual"])
        return _values(codes, scales), scales, residual
    if s["op"] == "weights":
        codes, scales = _codes(s["weight"].float())
        return _values(codes, scales), scales
    if s["op"] == "product":
        return _plain_product(s["x"], s["x_scales"], s["weight"], s["weight_scales"], s["out"])
    return _plain_experts(s["x"], s["x_scales"], s["weight"], s["weight_scales"], s["group_sizes"], s["rows"], s["out"])


def work(case):
    """Each input once, each output once; for experts those rows of x and those experts' weights that the routing can reach."""
    if case["op"] == "sort":
        n = case["tokens"] * case["top"]
        return {"bytes": 16.0 * n + 4.0 * case["experts"], "flops": float(n)}
    if case["op"] == "combine":
        t, n, w = case["tokens"], case["tokens"] * case["top"], case["width"]
        y, out, p = n * w * float(_SIZE[case["y"]]), t * w * float(_SIZE[case["out"]]), n * (4.0 + _SIZE[case["weights"]])
        flops = 2.0 * n * w
        if not case["train"]:
            return {"bytes": y + out + p, "flops": flops}
        return {"bytes": y + out + p + (y + out + y + p + 4.0 * n + n * _SIZE[case["weights"]]), "flops": 2.5 * flops}
    if case["op"] == "norm":
        n, w = case["rows"], case["width"]
        return {"bytes": n * w * (_SIZE[case["x"]] + 2.0 * _SIZE[case["residual"]] + 1.0) + 4.0 * n + w * _SIZE[case["x"]],
                "flops": 8.0 * n * w}
    matrices = max(1, case.get("experts", 0))
    if case["op"] == "weights":
        n, k = case["outputs"], case["inputs"]
        return {"bytes": matrices * (n * k * (_SIZE[case["x"]] + 1.0) + 4.0 * n), "flops": 3.0 * matrices * n * k}
    k, n = case["inputs"], case["outputs"]
    read = case["tokens"] if case["op"] == "experts" else case["rows"]
    rows = read * case.get("top", 1)
    held = min(matrices, rows) * (n * k + 4.0 * n)
    return {"bytes": read * (k + 4.0) + held + rows * n * float(_SIZE[case["out"]]), "flops": 2.0 * rows * k * n}


# ---- the same outputs in 64 bits -----------------------------------------------------------------------------------
def _exact_values(v):
    """Row by row of the last axis: the step, and the whole steps nearest to v."""
    step = torch.maximum(v.abs().max(dim=-1).values / LARGEST, torch.full_like(v[..., 0], SMALLEST_SCALE))
    return torch.round(v / step[..., None]) * step[..., None], step


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "sort":
        return None                                                            # whole numbers
    if case["op"] == "combine":
        y, tokens = s["y"].double(), s["places"].shape[0]
        y = torch.cat([y, torch.zeros_like(y[:1])])                            # the row of dropped choices
        out, grad_y, grad_w = torch.zeros((tokens, y.shape[1]), dtype=torch.float64, device=y.device), torch.zeros_like(y), []
        for j in range(s["places"].shape[1]):
            place = s["places"][:, j].long()                                   # (-1: the last)
            w = torch.ones(tokens, dtype=torch.float64, device=y.device) if s["weights"] is None else s["weights"][:, j].double()
            out += w[:, None] * y[place]
            if s["grad"] is not None:
                grad_w.append((s["grad"].double() * y[place]).sum(dim=1))
                grad_y[place] = w[:, None] * s["grad"].double()
        if s["grad"] is None:
            return out
        return out, grad_y[:-1], None if s["weights"] is None else torch.stack(grad_w, dim=1)
    if case["op"] == "norm":
        h = s["x"].double()
        if s["residual"] is not None:
            h = h + s["residual"].double()
        y = h / torch.sqrt((h * h).sum(dim=1, keepdim=True) / h.shape[1] + EPS) * s["weight"].double()
        return *_exact_values(y), None if s["residual"] is None else h
    if case["op"] == "weights":
        return _exact_values(s["weight"].double())
    if case["op"] == "product":
        sums = s["x"].double() @ s["weight"].double().t().contiguous()
        return sums * (s["x_scales"].double()[:, None] * s["weight_scales"].double()[None, :])
    parts, first = [], 0
    for e, n in enumerate(s["group_sizes"].tolist()):
        at = s["rows"][first:first + n].long()
        sums = s["x"][at].double() @ s["weight"][e].double().t().contiguous()
        parts.append(sums * (s["x_scales"][at].double()[:, None] * s["weight_scales"][e].double()[None, :]))
        first += n
    return torch.cat(parts)
