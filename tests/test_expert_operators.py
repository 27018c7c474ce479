"""A router's choices sorted by expert, and the experts' rows joined, with the gradients, against their definitions (torch on the CPU, in 64 bits).

Bounds, from the arithmetic (u = 2^-24, half a step of fp32):
  sort      whole numbers: equal
  combine   a product and an addition per place, u of the sum of magnitudes A each: (top + 1) u A; then the output's rounding, half a step of its type
  backward  a row: one product, u; a weight's gradient: a sum of `width` products in some order, (width + 1) u A; each rounded once to its type
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2601_03332_amd as lk  # noqa: E402
from paper_2601_03332_amd import binding  # noqa: E402

DEV = "cuda:0"
gpu = pytest.mark.gpu
U = 2.0 ** -24
FLOATS = [torch.float32, torch.float16, torch.bfloat16]
HALF = {t: torch.finfo(t).eps / 2 for t in FLOATS}
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}          # half the smallest step


def choices(seed, tokens, top, experts, kind, dtype=torch.int64):
    """kind: "any" (all experts alike), "one" (a single expert), "dropped" (a third outside, on both sides), "none" (all of them)."""
    gen = torch.Generator().manual_seed(seed)
    e = torch.randint(0, experts, (tokens, top), generator=gen)
    if kind == "one":
        e.fill_(experts - 1)
    if kind in ("dropped", "none"):
        outside = torch.tensor([-1, experts, -2 ** 31, 2 ** 31 - 1] + ([2 ** 32, -2 ** 40, 2 ** 62] if dtype == torch.int64 else []))
        gone = outside[torch.randint(0, outside.numel(), (tokens, top), generator=gen)]
        e = gone if kind == "none" else torch.where(torch.rand(tokens, top, generator=gen) < 1 / 3, gone, e)
    return e.to(dtype)


def sort_reference(expert, experts):
    flat, top = expert.flatten().long(), expert.shape[1]
    key = torch.where((flat >= 0) & (flat < experts), flat, experts)
    order = torch.sort(key, stable=True).indices
    held = int((key < experts).sum())
    rows, places = torch.full_like(flat, -1), torch.full_like(flat, -1)
    rows[:held] = order[:held] // max(top, 1)
    places[order[:held]] = torch.arange(held)
    return rows.int(), places.view(expert.shape).int(), torch.bincount(key, minlength=experts + 1)[:experts].int()


SORTS = [(1, 1, 1), (1, 2, 8), (3, 1, 5), (7, 8, 8), (16, 2, 8), (64, 1, 64), (65, 1, 3), (33, 2, 63), (500, 3, 12), (1023, 1, 65), (1024, 16, 128), (4097, 4, 256), (2048, 2, 64), (2049, 2, 64),
         (2049, 8, 2048), (16384, 1, 2), (16385, 1, 33), (16384, 8, 64), (100003, 3, 7), (3, 40000, 100), (300000, 2, 1000),
         (5, 3, 2049), (8000, 2, 4096), (9000, 2, 2047), (40000, 2, 70001), (3000, 4, 1 << 20)]


@gpu
@pytest.mark.parametrize("kind", ["any", "one", "dropped", "none"])
@pytest.mark.parametrize("shape", SORTS, ids=str)
def test_sort(shape, kind):
    tokens, top, experts = shape
    for dtype in (torch.int64, torch.int32):
        print(f"case sort {shape} {kind} {dtype}", flush=True)
        e = choices(tokens + top, tokens, top, experts, kind, dtype)
        got, ref = lk.lutkan_expert_sort(e.to(DEV), experts), sort_reference(e, experts)
        for g, r, what in zip(got, ref, ("rows", "places", "group_sizes")):
            assert g.dtype == torch.int32 and torch.equal(g.cpu(), r), what


@gpu
def test_sort_of_no_tokens_and_of_strided_choices():
    rows, places, sizes = lk.lutkan_expert_sort(torch.zeros((0, 2), dtype=torch.int64, device=DEV), 5)
    assert rows.shape == (0,) and places.shape == (0, 2) and torch.equal(sizes.cpu(), torch.zeros(5, dtype=torch.int32))
    for tokens in (50, 9000):
        wide = choices(1, tokens, 7, 9, "dropped").to(DEV)
        part = wide[:, 2:5]
        for g, r in zip(lk.lutkan_expert_sort(part, 9), sort_reference(part.cpu(), 9)):
            assert torch.equal(g.cpu(), r)
        same = wide[:1, :3].expand(tokens, 3)
        for g, r in zip(lk.lutkan_expert_sort(same, 9), sort_reference(same.cpu(), 9)):
            assert torch.equal(g.cpu(), r)


# ---------------------------------------------------------------- combine and its gradients
def near(got, ref, error, what=""):
    """got: a tensor of one of the three types; ref and error: numpy, the exact value and the error before the last rounding."""
    g = got.detach().cpu().double().numpy()
    limit = error + HALF[got.dtype] * (np.abs(ref) + error) + TINY[got.dtype]
    assert np.all(np.abs(g - ref) <= limit), (what, float(np.max(np.abs(g - ref) / np.maximum(limit, 1e-300))))


def combine_reference(y, places, weights):
    """(out, A) in 64 bits."""
    y, p = y.double().numpy(), places.long().numpy()
    out, A = np.zeros((p.shape[0], y.shape[1])), np.zeros((p.shape[0], y.shape[1]))
    for j in range(p.shape[1]):
        held = (p[:, j] >= 0) & (p[:, j] < y.shape[0])
        w = np.ones(held.sum()) if weights is None else weights[:, j].double().numpy()[held]
        part = w[:, None] * y[p[held, j]]
        out[held] += part
        A[held] += np.abs(part)
    return out, A


def gradient_reference(grad, y, places, weights):
    grad, yd, p = grad.double().numpy(), y.double().numpy(), places.long().numpy()
    grad_y, grad_w, A = np.zeros(y.shape), np.zeros(p.shape), np.zeros(p.shape)
    for j in range(p.shape[1]):
        held = (p[:, j] >= 0) & (p[:, j] < y.shape[0])
        w = np.ones(held.sum()) if weights is None else weights[:, j].double().numpy()[held]
        grad_y[p[held, j]] = w[:, None] * grad[held]
        grad_w[held, j] = (grad[held] * yd[p[held, j]]).sum(1)
        A[held, j] = np.abs(grad[held] * yd[p[held, j]]).sum(1)
    return grad_y, grad_w, A


def joined(seed, tokens, top, width, experts, kind, y_type, w_type, g_type):
    gen = torch.Generator().manual_seed(seed)
    rows, places, _ = sort_reference(choices(seed, tokens, top, experts, kind), experts)
    y = torch.randn(rows.numel(), width, generator=gen).to(y_type)
    weights = None if w_type is None else torch.rand(tokens, top, generator=gen).to(w_type)
    return rows, places, y, weights, torch.randn(tokens, width, generator=gen).to(g_type)


JOINS = [(1, 1, 1, 1, "any"), (1, 2, 1024, 8, "any"), (5, 3, 7, 4, "dropped"), (16, 2, 512, 8, "any"), (100, 4, 300, 16, "dropped"), (33, 9, 513, 9, "any"), (7, 1, 8192, 2, "any"),
         (3, 2, 9001, 2, "dropped"), (2, 70, 40, 100, "dropped"), (2100, 2, 129, 3, "any"), (4, 2, 100, 3, "none"), (64, 8, 2048, 8, "any"), (3000, 3, 64, 5, "dropped")]


@gpu
@pytest.mark.parametrize("types", [(a, b, c) for a in FLOATS for b in (torch.float32, torch.bfloat16, None) for c in FLOATS] + [(torch.float32, torch.float16, torch.float32)], ids=str)
@pytest.mark.parametrize("shape", JOINS, ids=str)
def test_combine_and_its_gradients(shape, types):
    tokens, top, width, experts, kind = shape
    y_type, w_type, o_type = types
    print(f"case combine {shape} {types}", flush=True)
    rows, places, y, weights, grad = joined(tokens + width, tokens, top, width, experts, kind, y_type, w_type, o_type)
    ref, A = combine_reference(y, places, weights)
    on = [None if t is None else t.to(DEV) for t in (rows, places, y, weights, grad)]
    out = lk.lutkan_expert_combine(on[2], on[1], on[3], dtype=o_type)
    assert out.dtype == o_type and out.shape == (tokens, width)
    near(out, ref, (top + 1) * U * 1.01 * A, "out")
    # rows of no choice hold NaN: none of them is read
    filled = on[2].clone()
    filled[on[0] < 0] = float("nan")
    w = None if on[3] is None else torch.where(on[1] < 0, float("nan"), on[3])
    assert torch.equal(out, lk.lutkan_expert_combine(filled, on[1].long(), w, dtype=o_type))
    gy, gw, Aw = gradient_reference(grad, y, places, weights)
    for integers in (torch.int32, torch.int64):
        got_y, got_w = lk.lutkan_expert_combine_backward(on[4], filled, on[0].to(integers), on[1].to(integers), w)
        assert got_y.dtype == y_type and got_y.shape == y.shape
        near(got_y, gy, U * np.abs(gy), "grad_y")
        if weights is None:
            assert got_w is None
        else:
            assert got_w.dtype == w_type and got_w.shape == weights.shape
            near(got_w, gw, (width + 1) * U * 1.01 * Aw, "grad_weights")


@gpu
@pytest.mark.parametrize("width", [40, 300, 1500])
def test_gradients_against_differences(width):
    """out is linear in y and in the weights: the loss' difference over a step along a direction is the gradient's product with it, up to the
    outputs' roundings, (top + 1) u of the sums of magnitudes of both outputs."""
    tokens, top, experts = 60, 3, 7
    rows, places, y, weights, grad = [t.to(DEV) for t in joined(3, tokens, top, width, experts, "dropped", torch.float32, torch.float32, torch.float32)]
    grad_y, grad_w = lk.lutkan_expert_combine_backward(grad, y, rows, places, weights)
    gen = torch.Generator(device=DEV).manual_seed(5)
    for of_y in (True, False):
        step = torch.randn(y.shape if of_y else weights.shape, generator=gen, device=DEV)
        more, less = [(y + s * step, weights) if of_y else (y, weights + s * step) for s in (1, -1)]
        plus, minus = (lk.lutkan_expert_combine(a, places, b) for a, b in (more, less))
        difference = float(((plus.double() - minus.double()) * grad.double()).sum()) / 2
        said = float(((grad_y if of_y else grad_w).double() * step.double()).sum())
        A = sum(float((torch.from_numpy(combine_reference(a.cpu(), places.cpu(), b.cpu())[1]).to(DEV) * grad.double().abs()).sum()) for a, b in (more, less))
        moved = float((((grad_y if of_y else grad_w).double() * step.double()).abs()).sum())
        size = float((grad_y.double() * y.double()).abs().sum())   # (of the weights' gradients times the weights too)
        # the moved operands round: u of |operand| + |step|, twice over two; the gradients do: u of a row's, (width + 1) u of a weight's magnitudes
        Aw = torch.from_numpy(gradient_reference(grad.cpu(), y.cpu(), places.cpu(), weights.cpu())[2]).to(DEV)
        rounded = moved if of_y else (width + 1) * float((Aw * step.double().abs()).sum())
        assert abs(difference - said) <= 1.01 * U * ((top + 1) * A / 2 + size + moved + rounded), (of_y, difference, said)


@gpu
def test_tokens_into_the_experts_order_and_the_gradient_of_that():
    tokens, top, experts, width = 70, 3, 6, 200
    e = choices(9, tokens, top, experts, "dropped")
    rows, places, _ = sort_reference(e, experts)
    gen = torch.Generator().manual_seed(1)
    x, grad = torch.randn(tokens, width, generator=gen).bfloat16(), torch.randn(tokens * top, width, generator=gen)
    got = lk.lutkan_expert_combine(x.to(DEV), rows[:, None].to(DEV))
    assert torch.equal(got.cpu(), torch.where(rows[:, None] >= 0, x[rows.long().clamp(min=0)], torch.zeros((), dtype=x.dtype)))
    back = lk.lutkan_expert_combine(grad.to(DEV), places.to(DEV))
    ref = np.zeros((tokens, width))
    at = rows.long().numpy()
    np.add.at(ref, at[at >= 0], grad.double().numpy()[at >= 0])
    near(back, ref, (top + 1) * U * 1.01 * combine_reference(grad, places, None)[1])


@gpu
def test_combine_of_strided_rows_into_a_part_of_a_wider_output():
    tokens, top, width, experts = 45, 2, 130, 4
    rows, places, y, weights, grad = joined(8, tokens, top, width, experts, "dropped", torch.bfloat16, torch.float32, torch.float16)
    wide = torch.full((y.shape[0], width + 9), float("nan"), dtype=y.dtype, device=DEV)
    wide[:, 3:3 + width] = y.to(DEV)
    part = wide[:, 3:3 + width]
    out = torch.full((tokens, width + 6), 7.0, device=DEV)
    got = lk.lutkan_expert_combine(part, places.to(DEV), weights.to(DEV), out=out[:, 5:5 + width])
    assert got.data_ptr() == out[:, 5:].data_ptr()
    ref, A = combine_reference(y, places, weights)
    near(got, ref, (top + 1) * U * 1.01 * A)
    assert bool((out[:, :5] == 7).all()) and bool((out[:, 5 + width:] == 7).all())
    wide_grad = torch.full((tokens, width + 3), float("nan"), dtype=grad.dtype, device=DEV)
    wide_grad[:, 1:1 + width] = grad.to(DEV)
    got_y, got_w = lk.lutkan_expert_combine_backward(wide_grad[:, 1:1 + width], part, rows.to(DEV), places.to(DEV), weights.to(DEV))
    gy, gw, Aw = gradient_reference(grad, y, places, weights)
    near(got_y, gy, U * np.abs(gy))
    near(got_w, gw, (width + 1) * U * 1.01 * Aw)
    # one row of y, and one gradient, for all: stride 0
    one = y[:1].to(DEV).expand(y.shape[0], width)
    near(lk.lutkan_expert_combine(one, places.to(DEV)), *(lambda r, a: (r, (top + 1) * U * 1.01 * a))(*combine_reference(y[:1].expand(y.shape[0], width), places, None)))
    same = grad[:1].to(DEV).expand(tokens, width)
    near(lk.lutkan_expert_combine_backward(same, part, rows.to(DEV), places.to(DEV), weights.to(DEV))[0],
         *(lambda g: (g, U * np.abs(g)))(gradient_reference(grad[:1].expand(tokens, width), y, places, weights)[0]))


@gpu
def test_combine_with_places_outside_and_of_no_rows_or_tokens():
    y = torch.randn(5, 20, device=DEV)
    places = torch.tensor([[0, 5], [-1, 2 ** 31 - 1], [4, -2 ** 31]], dtype=torch.int32, device=DEV)
    out = lk.lutkan_expert_combine(y, places)
    assert torch.equal(out, torch.stack([y[0], torch.zeros(20, device=DEV), y[4]]))
    assert torch.equal(out, lk.lutkan_expert_combine(y, torch.tensor([[0, 2 ** 40], [-1, 2 ** 33], [4, -2 ** 62]], device=DEV)))
    assert not bool(lk.lutkan_expert_combine(y[:0], places).any())
    assert lk.lutkan_expert_combine(y, places[:0]).shape == (0, 20)
    grad = torch.randn(3, 20, device=DEV)
    rows = torch.tensor([0, -1, 7, 1, 2], dtype=torch.int32, device=DEV)
    gy, gw = lk.lutkan_expert_combine_backward(grad, y, rows, places, torch.ones(3, 2, device=DEV))
    assert torch.equal(gy[0], grad[0]) and torch.equal(gy[4], grad[2]) and not bool(gy[1:4].any())
    assert not bool(gw[:, 1].any()) and not bool(gw[1].any())
    gy, gw = lk.lutkan_expert_combine_backward(grad[:0], y, torch.full_like(rows, -1), places[:0], torch.ones(0, 2, device=DEV))
    assert gw.shape == (0, 2) and not bool(gy.any())
    gy, gw = lk.lutkan_expert_combine_backward(grad, y[:0], rows[:0], places, torch.ones(3, 2, device=DEV))
    assert gy.shape == (0, 20) and not bool(gw.any())


@gpu
def test_combine_of_rows_at_offsets_beyond_32_bits():
    """A y of 2^31 + elements: rows behind it are found, and gradients written there."""
    width, n = 4096, (1 << 19) + 3
    y = torch.zeros((n, width), dtype=torch.float16, device=DEV)
    y[n - 1], y[1] = 3.0, 2.0
    places = torch.tensor([[n - 1, 1]], device=DEV)
    assert torch.equal(lk.lutkan_expert_combine(y, places), torch.full((1, width), 5.0, dtype=torch.float16, device=DEV))
    rows = torch.full((n,), -1, dtype=torch.int64, device=DEV)
    rows[n - 1] = rows[1] = 0
    gy, gw = lk.lutkan_expert_combine_backward(torch.ones((1, width), dtype=torch.float16, device=DEV), y, rows, places, torch.tensor([[0.5, 0.25]], device=DEV))
    assert gw.tolist() == [[3.0 * width, 2.0 * width]]
    assert bool((gy[n - 1] == 0.5).all()) and bool((gy[1] == 0.25).all())
    gy[n - 1], gy[1] = 0, 0
    assert not bool(gy.any())


# ---------------------------------------------------------------- together
def _pass(x, w, logits, grad):
    """Tokens to their experts' order, a product there, back with weights, and the gradients of all."""
    p, expert = torch.softmax(logits, 1).topk(2, 1)
    rows, places, sizes = lk.lutkan_expert_sort(expert, logits.shape[1])
    xs = lk.lutkan_expert_combine(x, rows[:, None])
    z = xs * w
    out = lk.lutkan_expert_combine(z, places, p)
    gz, gp = lk.lutkan_expert_combine_backward(grad, z, rows, places, p)
    return out, lk.lutkan_expert_combine(gz * w, places), gp, sizes


def _given(tokens):
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    return [torch.randn(tokens, 264, generator=gen, device=DEV), torch.randn(264, generator=gen, device=DEV), torch.randn(tokens, 9, generator=gen, device=DEV),
            torch.randn(tokens, 264, generator=gen, device=DEV)]


@gpu
@pytest.mark.parametrize("tokens", [1, 100, 20000])
def test_a_pass_against_torch_on_another_stream_and_in_a_replayed_graph(tokens):
    x, w, logits, grad = given = _given(tokens)
    eager = _pass(*given)
    p, expert = torch.softmax(logits, 1).topk(2, 1)
    # the same by token, in 64 bits on the CPU: out = sum_j p_j w x, so that its gradients are sum_j p_j w g and <g, w x>
    xd, wd, pd, gd = (t.double().cpu() for t in (x, w, p, grad))
    assert torch.allclose(eager[0].double().cpu(), pd.sum(1, keepdim=True) * wd * xd, rtol=8 * U, atol=8 * U * float((wd * xd).abs().max()))
    assert torch.allclose(eager[1].double().cpu(), pd.sum(1, keepdim=True) * wd * gd, rtol=8 * U, atol=8 * U * float((wd * gd).abs().max()))
    dot = (gd * wd * xd).sum(1, keepdim=True).expand(tokens, 2)
    assert bool(((eager[2].double().cpu() - dot).abs() <= 270 * U * (gd * wd * xd).abs().sum(1, keepdim=True)).all())
    assert torch.equal(eager[3].cpu(), torch.bincount(expert.flatten().cpu(), minlength=9).int())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = _pass(*given)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _pass(*given)
    for k in range(4):
        for t in (x, logits, grad):
            t.copy_(torch.randn_like(t))
        graph.replay()
        got = [t.clone() for t in held]
        torch.cuda.synchronize()
        expected = _pass(*given)
        assert all(torch.equal(a, b) for a, b in zip(got, expected)), k
        torch.cuda.synchronize()


@gpu
@pytest.mark.parametrize("codes", ["fp8", "int8"])
@pytest.mark.parametrize("tokens", [1, 37, 600])
def test_the_block_joins_as_torch_does(tokens, codes):
    """The block's output bit for bit from its own steps with torch's sort, indexing, product and sum (two experts a token: one order of the sum)."""
    from paper_2601_03332_amd.expert_block import ExpertBlock
    rng = np.random.default_rng(tokens)
    width, inner, experts, top = 200, 48, 5, 2
    knots = (-4.0 + (np.arange(15) - 3) * 1.0).astype(np.float32)
    art = lk.lutkan_compile(inner, width, 8, 3, knots, (rng.standard_normal((inner, width, 11)) / 7).astype(np.float32), 32, lk.ASYM_UINT8, lk.CLOSED, lk.CLIP_X)

    def normal(*shape):
        return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DEV)
    norm, layer = 1 + 0.1 * normal(width), art.to_device(DEV)
    router, weights = normal(experts, width) / width ** 0.5, normal(experts, inner, width) / width ** 0.5
    block = ExpertBlock(norm, router, weights, layer, top, codes=codes)
    x, residual = normal(tokens, width).bfloat16(), normal(tokens, width)
    y, res = block(x, residual)
    kind = dict(fp8=(lk.lutkan_rmsnorm_fp8, lk.lutkan_matmul_fp8, lk.lutkan_grouped_matmul_fp8), int8=(lk.lutkan_rmsnorm_int8, lk.lutkan_matmul_int8, lk.lutkan_grouped_matmul_int8))[codes]
    c, s, r = kind[0](x, norm, residual=residual)
    p, expert = torch.softmax(kind[1](c, s, *block.router), dim=1).topk(top, dim=1)
    order = torch.sort(expert.flatten(), stable=True).indices
    z = kind[2](c, s, *block.experts, torch.bincount(expert.flatten(), minlength=experts), rows=order // top)
    back = torch.empty((tokens * top, width), device=DEV)
    back[order] = lk.lutkan_forward(layer, z)
    assert torch.equal(y, (back.view(tokens, top, width) * p[..., None]).sum(dim=1).to(x.dtype)) and torch.equal(res, r)
    none, _ = block(torch.zeros((0, width), device=DEV), torch.zeros((0, width), device=DEV))
    assert none.shape == (0, width)
    # and how far the unquantised projections are: 8 bits hold a projection to a few percent
    h = x.float() + residual
    n = h * torch.rsqrt(h.square().mean(dim=1, keepdim=True) + block.eps) * norm
    assert float((z - torch.stack([weights[e] @ n[t] for e, t in zip(expert.flatten()[order].tolist(), (order // top).tolist())])).norm() / z.norm()) < 0.06


# ---------------------------------------------------------------- refusals (nothing is launched)
def _refused(code, rc):
    assert rc == code, (rc, lk.lutkan_last_error())
    assert lk.lutkan_last_error()


def test_the_library_refuses_bad_arguments():
    import ctypes as C
    lib = lk.load_library()

    def call(f, a, changes):
        for k, v in changes.items():
            setattr(a, k, v)
        return getattr(lib, f)(C.byref(a), None)

    def sort(**changes):
        return call("lutkan_expert_sort", binding._ExpertSortArgs(4096, 4096, 4096, 4096, None, 2, 3, 0, 2, 8, 8), changes)
    _refused(-1, lib.lutkan_expert_sort(None, None))
    _refused(-2, sort(experts=5000))                                # (two passes: the orders between them)
    for change in ({"expert": None}, {"rows": None}, {"places": None}, {"group_sizes": None}, {"tokens": -1}, {"top": 0}, {"experts": 0}, {"expert_bytes": 2}):
        _refused(-1, sort(**change))
    _refused(-1, sort(tokens=100000, workspace=4098, workspace_bytes=1 << 20))
    _refused(-2, sort(tokens=100000, workspace=4096, workspace_bytes=100))
    _refused(-2, sort(tokens=100000, workspace=None, workspace_bytes=1 << 20))
    _refused(-2, sort(expert_stride=-1))
    _refused(-5, sort(experts=(1 << 20) + 1))
    _refused(-5, sort(tokens=(1 << 23) + 1))
    assert lib.lutkan_expert_sort_workspace_bytes(1024, 4, 2048) == 0 and lib.lutkan_expert_sort_workspace_bytes(100000, 2, 8) > 0
    for bad in ((-1, 2, 8), (5, 0, 8), (5, 2, 0), (5, 2, (1 << 20) + 1), (1 << 40, 2, 8)):
        assert lib.lutkan_expert_sort_workspace_bytes(*bad) == 0

    def combine(**changes):
        return call("lutkan_expert_combine", binding._ExpertCombineArgs(4096, 4096, 4096, 4096, 6, 8, 8, 3, 2, 8, 0, 0, 0, 4), changes)
    _refused(-1, lib.lutkan_expert_combine(None, None))
    for change in ({"y": None}, {"places": None}, {"out": None}, {"tokens": -1}, {"y_rows": -1}, {"top": 0}, {"width": 0}, {"y_type": 3}, {"out_type": -1}, {"weights_type": 7}, {"places_bytes": 2}):
        _refused(-1, combine(**change))
    for change in ({"y_stride": -1}, {"out_stride": 7}):
        _refused(-2, combine(**change))
    for change in ({"y_stride": 1 << 31}, {"out_stride": 1 << 31}, {"tokens": 1 << 31}, {"y_rows": 1 << 31}, {"width": (1 << 30) + 1, "out_stride": 1 << 30}):
        _refused(-5, combine(**change))
    assert combine(tokens=0, y=None, places=None, out=None) == 0

    def backward(**changes):
        return call("lutkan_expert_combine_backward",
                    binding._ExpertCombineBackwardArgs(4096, 4096, 4096, 4096, 4096, 4096, 4096, 6, 8, 8, 8, 3, 2, 8, 0, 0, 0, 4, 4), changes)
    _refused(-1, lib.lutkan_expert_combine_backward(None, None))
    for change in ({"grad": None}, {"y": None}, {"rows": None}, {"places": None}, {"weights": None}, {"grad_y": None}, {"grad_weights": None}, {"tokens": -1}, {"y_rows": -1}, {"top": 0},
                   {"width": 0}, {"grad_type": 3}, {"y_type": -1}, {"weights_type": 7}, {"rows_bytes": 2}, {"places_bytes": 1}):
        _refused(-1, backward(**change))
    for change in ({"grad_stride": -1}, {"y_stride": -1}, {"grad_y_stride": 7}):
        _refused(-2, backward(**change))
    for change in ({"grad_stride": 1 << 31}, {"y_stride": 1 << 31}, {"grad_y_stride": 1 << 31}, {"tokens": 1 << 31}, {"y_rows": 1 << 31}, {"tokens": (1 << 31) - 1, "width": 4096, "grad_y_stride": 4096}):
        _refused(-5, backward(**change))
    assert backward(tokens=0, y_rows=0, grad=None, y=None, rows=None, places=None, weights=None, grad_y=None, grad_weights=None) == 0


def _raises(words, f, *args, **kwargs):
    with pytest.raises(lk.LutKanError, match=words):
        f(*args, **kwargs)


def test_the_binding_refuses_what_is_no_tensor_of_the_gpu():
    e = torch.zeros((4, 2), dtype=torch.int64)
    for bad in (e, e.float(), e[0], None, [[1, 2]]):
        _raises("expert must be", lk.lutkan_expert_sort, bad, 5)
    y = torch.zeros(8, 16)
    _raises("CUDA tensor", lk.lutkan_expert_combine, y, e)
    _raises("shape", lk.lutkan_expert_combine, y[0], e)
    _raises("dtype", lk.lutkan_expert_combine, y.double(), e)
    _raises("CUDA tensor", lk.lutkan_expert_combine_backward, y, y, e, e)
    _raises("shape", lk.lutkan_expert_combine_backward, None, y, e, e)
    from types import SimpleNamespace
    from paper_2601_03332_amd.expert_block import ExpertBlock
    _raises("codes are", ExpertBlock, torch.ones(10), torch.zeros(4, 10), torch.zeros(4, 6, 10), SimpleNamespace(d=6, m=10), codes="int4")


@gpu
def test_the_binding_refuses_operands_that_do_not_fit():
    e = torch.zeros((4, 2), dtype=torch.int64, device=DEV)
    _raises("contiguous columns", lk.lutkan_expert_sort, torch.zeros((2, 4), dtype=torch.int64, device=DEV).t(), 5)
    _raises("experts", lk.lutkan_expert_sort, e, 0)
    _raises("experts", lk.lutkan_expert_sort, e, -3)
    _raises("experts", lk.lutkan_expert_sort, e, (1 << 20) + 1)
    _raises("experts", lk.lutkan_expert_sort, e, 1 << 40)
    _raises("0 each", lk.lutkan_expert_sort, e[:, :0], 5)
    y = torch.zeros(8, 16, device=DEV)
    _raises("places", lk.lutkan_expert_combine, y, e.float())
    _raises("places", lk.lutkan_expert_combine, y, e.cpu())
    _raises("places", lk.lutkan_expert_combine, y, e[:, 0].contiguous())
    _raises("places", lk.lutkan_expert_combine, y, torch.zeros((2, 4), dtype=torch.int64, device=DEV).t())
    _raises("weights", lk.lutkan_expert_combine, y, e, torch.ones(4, 3, device=DEV))
    _raises("weights", lk.lutkan_expert_combine, y, e, torch.ones(4, 2))
    _raises("weights", lk.lutkan_expert_combine, y, e, torch.ones(4, 4, device=DEV)[:, :2])
    _raises("weights", lk.lutkan_expert_combine, y, e, e)
    _raises("contiguous columns", lk.lutkan_expert_combine, y.t(), e)
    _raises("dtype", lk.lutkan_expert_combine, y, e, dtype=torch.int8)
    _raises("out must", lk.lutkan_expert_combine, y, e, out=torch.empty(4, 15, device=DEV))
    _raises("overlap", lk.lutkan_expert_combine, y, e, out=torch.empty(1, 16, device=DEV).expand(4, 16))
    grad, rows = torch.zeros(4, 16, device=DEV), torch.zeros(8, dtype=torch.int32, device=DEV)
    _raises("y must", lk.lutkan_expert_combine_backward, grad, y[:, :15], rows, e)
    _raises("rows must", lk.lutkan_expert_combine_backward, grad, y, rows[:7], e)
    _raises("places must", lk.lutkan_expert_combine_backward, grad, y, rows, e[:3])
    _raises("weights must", lk.lutkan_expert_combine_backward, grad, y, rows, e, torch.ones(4, 1, device=DEV))


# ---------------------------------------------------------------- the binding's two paths
def _every_call(t):
    """Each operator of this file and of the integer ones, without an output of the caller's; the tensors are made on the first call."""
    rows, width = t.shape
    gen = torch.Generator(device=DEV).manual_seed(3)
    e = torch.randint(-1, 4, (rows, 2), generator=gen, device=DEV)
    r, places, sizes = lk.lutkan_expert_sort(e, 4)
    y, p = torch.randn(2 * rows, width, generator=gen, device=DEV), torch.rand(rows, 2, generator=gen, device=DEV)
    weight, grad = torch.ones(width, device=DEV), torch.randn(rows, width, generator=gen, device=DEV)
    w, ws = lk.lutkan_quantise_int8(torch.randn(4, 20, width, generator=gen, device=DEV))
    x, xs = lk.lutkan_quantise_int8(t)
    return [lambda f, v: f("expert_sort", (v[:, :2] > 0).long(), 4), lambda f, v: f("expert_sort", (v[:, :3] * 3).int(), 3000), lambda f, v: f("expert_combine", y, places, v[:, :2].contiguous(), torch.bfloat16),
            lambda f, v: f("expert_combine", v, r[:, None], None, None), lambda f, v: f("expert_combine_backward", v, y, r, places, p),
            lambda f, v: f("expert_combine_backward", grad, y, r, places, v[:, :2].contiguous()), lambda f, v: f("expert_combine_backward", v, y, r, places, None),
            lambda f, v: f("rmsnorm_int8", v, weight, None, 1e-6), lambda f, v: f("rmsnorm_int8", t, weight, v, 1e-6), lambda f, v: f("quantise_int8", v),
            lambda f, v: f("matmul_int8", x, v[:, 0].contiguous(), w[0], ws[0], torch.float32), lambda f, v: f("matmul_int8", x, v[:, 1], w, ws, torch.bfloat16, sizes, r)]


PUBLIC = {"expert_sort": lk.lutkan_expert_sort, "expert_combine": lambda y, places, w, dtype: lk.lutkan_expert_combine(y, places, w, dtype=dtype),
          "expert_combine_backward": lk.lutkan_expert_combine_backward, "rmsnorm_int8": lambda x, w, r, eps: lk.lutkan_rmsnorm_int8(x, w, residual=r, eps=eps),
          "quantise_int8": lk.lutkan_quantise_int8,
          "matmul_int8": lambda x, xs, w, ws, dtype, *g: lk.lutkan_grouped_matmul_int8(x, xs, w, ws, g[0], rows=g[1], dtype=dtype) if g else lk.lutkan_matmul_int8(x, xs, w, ws, dtype=dtype)}


def _plain(out):
    return [o for o in (out if isinstance(out, tuple) else (out,)) if o is not None]


@gpu
def test_the_general_path_returns_what_the_native_calls_do(monkeypatch):
    t = torch.randn(37, 130, device=DEV)
    calls = _every_call(t)
    native = [_plain(call(lambda name, *args: getattr(binding._native_calls(), name)(*args), t)) for call in calls]
    monkeypatch.setattr(binding, "_native", binding._GeneralPath)
    for call, expected in zip(calls, native):
        got = _plain(call(lambda name, *args: PUBLIC[name](*args), t))
        assert len(got) == len(expected) and all(a.dtype == b.dtype and torch.equal(a, b) for a, b in zip(got, expected))


@gpu
def test_native_calls_leave_deferred_and_traced_operators_to_the_general_path():
    from torch._subclasses import FakeTensorMode
    from torch.utils._python_dispatch import TorchDispatchMode
    native = binding._native_calls()
    t = torch.randn(12, 256, device=DEV)
    calls = _every_call(t)

    def direct(name, *args):
        return getattr(native, name)(*args)
    expect = [_plain(call(direct, t)) for call in calls]
    with torch.inference_mode():
        for call, y in zip(calls, expect):
            got = _plain(call(direct, t))
            assert all(torch.equal(a, b) for a, b in zip(got, y)) and all(a.is_inference() for a in got)
    watched = t.clone().requires_grad_()                          # (no part in autograd: outputs do not require gradients)
    for call, y in zip(calls, expect):
        got = _plain(call(direct, watched))
        assert all(torch.equal(a, b) and not a.requires_grad for a, b in zip(got, y))

    class Passes(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            return func(*args, **(kwargs or {}))
    taken = []

    def ask(v):
        full = v if v.dim() == 2 else v[None].expand(12, -1)
        taken.extend(call(direct, full) for call in calls)
        return v + 1.0
    with FakeTensorMode(allow_non_fake_inputs=True) as mode:
        ask(mode.from_tensor(t))
        ask(t)
    with Passes():
        ask(t)
        general = [_plain(call(lambda name, *args: PUBLIC[name](*args), t)) for call in calls]      # the general path serves them
    assert all(torch.equal(a, b) for got, y in zip(general, expect) for a, b in zip(got, y))
    torch.func.vmap(ask)(t)
    torch.func.grad(lambda v: ask(v).sum())(t)
    torch.func.jvp(ask, (t,), (torch.ones_like(t),))
    torch.func.functionalize(ask)(t)
    torch.jit.trace(ask, (t,), check_trace=False)
    assert len(taken) == len(calls) * 8 and all(y is None for y in taken), [y is None for y in taken]
    for call, y in zip(calls, expect):                            # and nothing of it is left behind
        assert all(torch.equal(a, b) for a, b in zip(_plain(call(direct, t)), y))


# ---------------------------------------------------------------- ends of ranges
def test_more_choices_a_token_than_the_loops_count_are_refused():
    """A token's choices are looked through 64 (the rows of y: four) at a time, counted in 32 bits: the count behind the last ones has to fit them."""
    import ctypes as C
    lib = lk.load_library()
    for top in ((1 << 30) + 1, (1 << 31) - 64, (1 << 31) - 63, (1 << 31) - 1):
        a = binding._ExpertCombineArgs(4096, 4096, 4096, 4096, 6, 8, 8, 1, top, 8, 0, 0, 0, 4)
        _refused(-5, lib.lutkan_expert_combine(C.byref(a), None))
        a = binding._ExpertCombineBackwardArgs(4096, 4096, 4096, 4096, 4096, 4096, 4096, 6, 8, 8, 8, 1, top, 8, 0, 0, 0, 4, 4)
        _refused(-5, lib.lutkan_expert_combine_backward(C.byref(a), None))
    assert lib.lutkan_expert_combine(C.byref(binding._ExpertCombineArgs(None, None, None, None, 6, 8, 8, 0, 1 << 30, 8, 0, 0, 0, 4)), None) == 0


# ---------------------------------------------------------------- the sort's forms, and what its outputs hold on to
def sort_form(tokens, top, experts):
    """(several work-groups, two passes), from the workspace: counts of several work-groups, the two orders of two passes."""
    need = lk.load_library().lutkan_expert_sort_workspace_bytes(tokens, top, experts)
    orders = 8 * tokens * top if experts > 2048 else 0
    assert need >= orders
    return need > orders, experts > 2048


def test_the_sorted_shapes_reach_every_form_of_the_sort():
    forms = {shape: sort_form(*shape) for shape in SORTS}
    assert set(forms.values()) == {(a, b) for a in (False, True) for b in (False, True)}
    assert all(several == (shape[0] * shape[1] > 4096) for shape, (several, _) in forms.items())


@gpu
@pytest.mark.parametrize("general", [False, True], ids=["native", "general"])
@pytest.mark.parametrize("shape", [(1, 2, 8), (2048, 2, 64), (16384, 8, 64), (3000, 1, 4096), (40000, 2, 70001)], ids=str)
def test_a_sort_keeps_its_outputs_alone(shape, general, monkeypatch):
    """The workspace is free again once the call has returned: a program that keeps places and rows for its backward pass keeps no more than these."""
    if general:
        monkeypatch.setattr(binding, "_native", binding._GeneralPath)
    tokens, top, experts = shape
    e = choices(4, tokens, top, experts, "dropped")
    got = lk.lutkan_expert_sort(e.to(DEV), experts)
    held = sum({t.untyped_storage().data_ptr(): t.untyped_storage().nbytes() for t in got}.values())
    assert held <= sum(t.numel() * 4 + 255 for t in got)
    again = [lk.lutkan_expert_sort(e.to(DEV), experts) for _ in range(3)] + [torch.full((3 * tokens * top + 70001,), 9, dtype=torch.int32, device=DEV)]      # (in the same memory)
    for g, a, r in zip(got, again[0], sort_reference(e, experts)):
        assert torch.equal(g.cpu(), r) and torch.equal(a.cpu(), r)


@gpu
@pytest.mark.parametrize("shape", [(9000, 2, 64), (3000, 1, 4096), (9000, 2, 4096)], ids=str)
def test_sorts_in_two_replayed_graphs(shape):
    """Two sorts a graph, two graphs of one pool of memory, replayed in turn with eager calls between them."""
    tokens, top, experts = shape
    given = [choices(k, tokens, top, experts, "dropped").to(DEV) for k in range(2)]
    for e in given:
        lk.lutkan_expert_sort(e, experts)
    torch.cuda.synchronize()
    graphs, outputs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for k, graph in enumerate(graphs):
        with torch.cuda.graph(graph, pool=graphs[0].pool() if k else None):
            outputs.append([lk.lutkan_expert_sort(e, experts) for e in given])
    for k in range(4):
        for graph, out in zip(graphs, outputs):
            for i, e in enumerate(given):
                e.copy_(choices(10 * k + i, tokens, top, experts, "any" if k == 1 else "dropped"))
            graph.replay()
            torch.cuda.synchronize()
            for e, sorted_ in zip(given, out):
                eager = lk.lutkan_expert_sort(e, experts)
                assert all(torch.equal(a, b) and torch.equal(a.cpu(), r) for a, b, r in zip(sorted_, eager, sort_reference(e.cpu(), experts)))


# ---------------------------------------------------------------- the gradients, by the depth of their sums
def gradient_depth(width):
    """Roundings that a product of a weight's gradient passes through: eight fused additions for each of a lane's pieces of eight columns (up to 16 waves share a row),
    six exchanges in a wave, the waves' sums."""
    waves = min(-(-width // 512), 16)
    return 8 * -(-width // (512 * waves)) + 6 + waves


DEPTHS = [7, 300, 511, 513, 1025, 4103, 8191, 8192, 8193, 9001, 16385, 20007]


@gpu
@pytest.mark.parametrize("types", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.float32, torch.float16), (torch.float16, torch.bfloat16)], ids=str)
@pytest.mark.parametrize("width", DEPTHS)
def test_gradients_of_the_weights_by_the_depth_of_their_sums(width, types):
    """The bound is well below what one column of average size adds: 46 u of A at most, where a column holds A / width."""
    y_type, g_type = types
    tokens, top, experts = 12, 5, 7
    print(f"case depth {width} {types}", flush=True)
    rows, places, y, weights, grad = joined(width, tokens, top, width, experts, "dropped", y_type, torch.float32, g_type)
    gy, gw, A = gradient_reference(grad, y, places, weights)
    got_y, got_w = lk.lutkan_expert_combine_backward(grad.to(DEV), y.to(DEV), rows.to(DEV), places.to(DEV), weights.to(DEV))
    near(got_w, gw, gradient_depth(width) * U * 1.01 * A, "grad_weights")
    near(got_y, gy, U * np.abs(gy), "grad_y")


@gpu
@pytest.mark.parametrize("types", [(a, b) for a in FLOATS for b in FLOATS], ids=str)
@pytest.mark.parametrize("width", DEPTHS)
def test_gradients_of_the_weights_where_one_column_decides(width, types):
    """Each token's gradient has one column that is not zero, at the ends of the lanes' pieces, of the waves' and the work-group's columns and of the row: small whole
    numbers, so that the sums are exact and a column that is left out, or taken twice, shows."""
    y_type, g_type = types
    columns = sorted({c + d for c in (0, 8, 512, 1024, 4096, 8192, 16384, width // 8 * 8, width) for d in (-8, -1, 0, 1, 7)} & set(range(width)))
    tokens, top = len(columns), 5
    print(f"case column {width} {types}", flush=True)
    gen = torch.Generator().manual_seed(width)
    rows, places, _ = sort_reference(choices(width, tokens, top, 6, "any"), 6)
    y = torch.randint(1, 9, (tokens * top, width), generator=gen).to(y_type)
    weights = torch.exp2(torch.randint(-3, 4, (tokens, top), generator=gen).float())
    grad, at = torch.zeros(tokens, width, dtype=g_type), torch.tensor(columns)
    value = torch.randint(1, 9, (tokens,), generator=gen)
    grad[torch.arange(tokens), at] = value.to(g_type)
    got_y, got_w = lk.lutkan_expert_combine_backward(grad.to(DEV), y.to(DEV), rows.to(DEV), places.to(DEV), weights.to(DEV))
    assert torch.equal(got_w.cpu(), value[:, None].float() * y.float()[places.long(), at[:, None]])
    expected = torch.zeros(y.shape)
    expected[places.long()] = weights[..., None] * grad.float()[:, None, :]
    assert torch.equal(got_y.cpu().float(), expected)
