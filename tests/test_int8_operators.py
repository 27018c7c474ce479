"""The operators on 8-bit integers against their definition in 64 bits (numpy, on the CPU).

Bounds, from the arithmetic (u = 2^-24, half a step of fp32):
  product     the sum is a whole number below 2^31, held exactly; made fp32, times one scale, times the other: three roundings, 3 u of y (in fp64 for
              scales outside 2^-60 .. 2^60: one, u).  Then the rounding of the output, half a step of its type.
  rows        the scale is one division, rounded; a code is off value / scale by half and by the quotient's rounding, 2 u of it
  norm        a sum of squares of `width` terms, root, products: (width + 16) u relative for y and the scale; a code is off y / scale by half and that
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


def operands(seed, rows, k, n, experts=None):
    gen = torch.Generator().manual_seed(seed)
    lead = [] if experts is None else [experts]
    x, w = (torch.randint(-128, 128, s, generator=gen, dtype=torch.int8) for s in ((rows, k), (*lead, n, k)))
    xs = torch.exp(torch.randn(rows, generator=gen))
    ws = torch.exp(torch.randn(*lead, n, generator=gen)) * 0.01
    return x, xs, w, ws


def reference(x, xs, w, ws):
    return (x.numpy().astype(np.int64) @ w.numpy().astype(np.int64).T).astype(np.float64) * (xs.double().numpy()[:, None] * ws.double().numpy()[None, :])


def near(y, ref):
    got = y.detach().cpu().double().numpy()
    error = 3.01 * U * np.abs(ref)
    limit = error + HALF[y.dtype] * (np.abs(ref) + error) + TINY[y.dtype]
    if y.dtype == torch.float16:                                   # beyond its range: infinite
        over = np.abs(ref) > 65000
        assert np.all(np.isinf(got[np.abs(ref) > 66000]))
        got, ref, limit = got[~over], ref[~over], limit[~over]
    assert np.all(np.abs(got - ref) <= limit), float(np.max(np.abs(got - ref) / np.maximum(limit, 1e-300)))


# ---------------------------------------------------------------- products
SHAPES = [(1, 1, 1), (1, 16, 2), (3, 15, 5), (2, 17, 3), (1, 128, 16), (16, 127, 17), (17, 129, 33), (5, 144, 4), (33, 200, 300), (1, 1024, 40),
          (15, 2056, 31), (64, 256, 128), (65, 384, 130), (130, 512, 64), (257, 200, 129), (300, 640, 260), (513, 128, 516), (700, 1300, 20), (300, 1280, 900),
          (1025, 384, 1030), (2100, 256, 2050), (2000, 301, 600)]


@gpu
@pytest.mark.parametrize("dtype", FLOATS, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_product(shape, dtype):
    rows, k, n = shape
    print(f"case product {shape} {dtype}", flush=True)
    x, xs, w, ws = operands(rows * 7 + k, rows, k, n)
    y = lk.lutkan_matmul_int8(x.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV), dtype=dtype)
    assert y.shape == (rows, n) and y.dtype == dtype
    assert lk.lutkan_last_plan().startswith("int8_")
    near(y, reference(x, xs, w, ws))


@gpu
def test_product_defaults_to_32_bits_and_repeats_its_bits():
    x, xs, w, ws = (t.to(DEV) for t in operands(5, 100, 1000, 200))
    y = lk.lutkan_matmul_int8(x, xs, w, ws)
    assert y.dtype == torch.float32
    for _ in range(3):
        assert torch.equal(y, lk.lutkan_matmul_int8(x, xs, w, ws))


@gpu
@pytest.mark.parametrize("shape", [(1, 130, 20), (40, 256, 48), (70, 300, 131), (600, 512, 384), (530, 1000, 520)], ids=str)
def test_product_of_strided_unaligned_and_repeated_rows(shape):
    """Operands that are parts of wider or oddly placed buffers; what lies around them is 100 (codes) or NaN (scales), and around y stays what it was."""
    rows, k, n = shape
    print(f"case strided {shape}", flush=True)
    x, xs, w, ws = operands(11, rows, k, n)
    ref = reference(x, xs, w, ws)

    def inside(t, before, after, fill):
        wide = torch.full((t.shape[0], t.shape[1] + before + after), fill, dtype=t.dtype, device=DEV)
        wide[:, before:before + t.shape[1]] = t.to(DEV)
        return wide[:, before:before + t.shape[1]]

    for before, after in ((3, 8), (16, 32), (1, 0)):
        out = torch.full((rows, n + 5), 7.0, dtype=torch.bfloat16, device=DEV)
        y = lk.lutkan_matmul_int8(inside(x, before, after, 100), inside(xs[:, None], 1, 2, float("nan"))[:, 0], inside(w, after, before, 100), ws.to(DEV), y=out[:, 2:2 + n])
        assert y.data_ptr() == out[:, 2:].data_ptr()
        near(y, ref)
        assert bool((out[:, :2] == 7).all()) and bool((out[:, 2 + n:] == 7).all())
    one = lk.lutkan_matmul_int8(x[:1].to(DEV).expand(rows, k), xs[:1].to(DEV).expand(rows), w.to(DEV), ws.to(DEV))
    near(one, np.repeat(ref[:1], rows, 0))


@gpu
@pytest.mark.parametrize("rows", [5, 200, 1100])
def test_scales_of_any_size_reach_their_row_and_column_alone(rows):
    """Zero, the smallest and largest, infinite and NaN scales: y is what fp64 makes of them, rounded."""
    x, xs, w, ws = operands(17, rows, 300, 260)
    for i, v in enumerate((float("nan"), float("inf"), 0.0, 2.0 ** -149, 3e38, -2.0, 1e-30)):
        if i < rows - 1:
            xs[i] = v
        ws[2 * i + 1] = v
    sums = (x.numpy().astype(np.int64) @ w.numpy().astype(np.int64).T).astype(np.float64)
    with np.errstate(all="ignore"):
        ref = sums * (xs.double().numpy()[:, None] * ws.double().numpy()[None, :])
        single = ref.astype(np.float32)
    y = lk.lutkan_matmul_int8(x.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV))
    got = y.cpu().numpy()
    assert np.array_equal(np.isnan(single), np.isnan(got)) and np.array_equal(np.isinf(single), np.isinf(got))
    fine = np.isfinite(single)
    assert np.all(np.abs(got[fine] - ref[fine]) <= 3.01 * U * np.abs(ref[fine]) + 2.0 ** -149)


@gpu
@pytest.mark.parametrize("rows", [3, 70, 300, 2000])
def test_the_longest_sums_of_the_largest_codes_are_exact(rows):
    """131071 products of (-128)^2: 2^31 - 2^14, the largest whole number there is; and one that ends one below."""
    k = 131071
    x, w = torch.full((rows, k), -128, dtype=torch.int8, device=DEV), torch.full((5, k), -128, dtype=torch.int8, device=DEV)
    w[1] = 127
    w[2, k - 1] = -127
    y = lk.lutkan_matmul_int8(x, torch.ones(rows, device=DEV), w, torch.ones(5, device=DEV))
    ref = np.float32([k * 2 ** 14, -k * 127 * 128, k * 2 ** 14 - 128, k * 2 ** 14, k * 2 ** 14])
    assert np.array_equal(y.cpu().numpy(), np.repeat(ref[None], rows, 0))


@gpu
def test_product_with_no_rows():
    x, xs, w, ws = (t.to(DEV) for t in operands(1, 0, 128, 8))
    assert lk.lutkan_matmul_int8(x, xs, w, ws).shape == (0, 8)
    sizes = torch.zeros(3, dtype=torch.int32, device=DEV)
    assert lk.lutkan_grouped_matmul_int8(x, xs, w[None].expand(3, -1, -1), ws[None].repeat(3, 1), sizes).shape == (0, 8)


# ---------------------------------------------------------------- grouped
def grouped_reference(x, xs, w, ws, sizes, index, rows):
    ref, at = np.zeros((rows, w.shape[1])), 0
    source = np.arange(rows) if index is None else index.numpy()
    for e, size in enumerate(sizes):
        for s in range(at, min(at + max(size, 0), rows)):
            if 0 <= source[s] < x.shape[0]:
                ref[s] = reference(x[source[s]:source[s] + 1], xs[source[s]:source[s] + 1], w[e], ws[e])[0]
        at = min(at + max(size, 0), rows)
    return ref


# x rows, k, n, experts, sizes, rows of y (None: x's, without an index)
GROUPS = [(1, 128, 16, 1, [1], None), (7, 40, 5, 3, [2, 0, 5], None), (40, 200, 33, 4, [0, 30, 0, 3], 50), (300, 129, 70, 5, [100, 1, 99, 64, 36], 600), (130, 256, 300, 2, [65, 65], None),
          (64, 384, 130, 66, [1] * 64 + [0, 0], None), (500, 100, 20, 3, [-5, 700, 3], 520), (16, 1024, 64, 8, [4, 4, 0, 0, 8, 8, 8, 0], 32), (1500, 256, 640, 6, [600, 0, 511, 1, 257, 100], None),
          (20, 128, 8, 2, [0, 0], None), (900, 301, 520, 3, [400, 300, 100], 900), (3000, 384, 260, 4, [1000, 24, 1900, 0], 3010)]


@gpu
@pytest.mark.parametrize("integers", [torch.int32, torch.int64], ids=str)
@pytest.mark.parametrize("case", GROUPS, ids=lambda c: "-".join(str(v) for v in c[:4]))
def test_grouped_product(case, integers):
    x_rows, k, n, experts, sizes, rows = case
    print(f"case grouped {case[:4]} {integers}", flush=True)
    x, xs, w, ws = operands(x_rows + k, x_rows, k, n, experts)
    index = None
    if rows is not None:
        index = torch.randint(-2, x_rows + 2, (rows,), generator=torch.Generator().manual_seed(k))
        xs[0] = float("nan")                                       # (rows that are not there are zeros whatever the first row's scale is)
    ref = grouped_reference(x, xs, w, ws, sizes, index, rows or x_rows)
    for dtype in FLOATS:
        y = lk.lutkan_grouped_matmul_int8(x.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV), torch.tensor(sizes, dtype=integers, device=DEV),
                                          rows=None if index is None else index.to(integers).to(DEV), dtype=dtype)
        got = y.cpu().double().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        near(torch.from_numpy(np.nan_to_num(got, nan=0.0, posinf=np.inf, neginf=-np.inf)).to(dtype), np.nan_to_num(ref))


@gpu
def test_grouped_product_agrees_with_the_product_of_each_group():
    x, xs, w, ws = (t.to(DEV) for t in operands(2, 1200, 640, 384, 3))
    y = lk.lutkan_grouped_matmul_int8(x, xs, w, ws, torch.tensor([500, 0, 700], device=DEV), dtype=torch.bfloat16)
    assert torch.equal(y[:500], lk.lutkan_matmul_int8(x[:500], xs[:500], w[0], ws[0], dtype=torch.bfloat16))
    assert torch.equal(y[500:], lk.lutkan_matmul_int8(x[500:], xs[500:], w[2], ws[2], dtype=torch.bfloat16))


# ---------------------------------------------------------------- conversion of rows
def values(codes, scales):
    return codes.cpu().double().numpy() * scales.cpu().double().numpy()[..., None]


ROWS = [(1, 1), (5, 3), (1, 1024), (300, 200), (16, 1000), (2100, 130), (2050, 2048), (1100, 4100), (3, 16385), (2, 32768), (2, 32769), (1, 131071), (3, 7, 65), (8, 300, 200), (2, 0, 8), (0, 5)]


@gpu
@pytest.mark.parametrize("shape", ROWS, ids=str)
@pytest.mark.parametrize("dtype", FLOATS, ids=str)
def test_rows(shape, dtype):
    print(f"case rows {shape} {dtype}", flush=True)
    v = (torch.randn(shape, generator=torch.Generator().manual_seed(shape[-1])) * torch.exp(torch.randn(*shape[:-1], 1, generator=torch.Generator().manual_seed(1)))).to(dtype)
    codes, scales = lk.lutkan_quantise_int8(v.to(DEV))
    assert codes.dtype == torch.int8 and codes.shape == v.shape and scales.dtype == torch.float32 and scales.shape == v.shape[:-1]
    if v.numel() == 0:
        return
    exact = np.maximum(np.abs(v.float().numpy()).max(-1) / np.float32(127), np.float32(2.0 ** -126))
    assert exact.dtype == np.float32 and np.array_equal(scales.cpu().numpy(), exact)
    quotient = v.double().numpy() / exact.astype(np.float64)[..., None]
    got = codes.cpu().double().numpy()
    assert np.all(np.abs(got) <= 127) and np.all(np.abs(got - quotient) <= 0.5 + 2 * U * np.abs(quotient))


@gpu
def test_rows_of_ties_zeros_tiny_huge_and_not_finite_values():
    v = torch.zeros(9, 40)
    v[0, :8] = torch.tensor([127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5])     # scale 1: ties to even
    v[2, 3] = 2.0 ** -149
    v[3, 5], v[3, 6] = 3.4e38, -1.7e38
    v[4, 1], v[5, 39], v[6, 0] = float("nan"), float("-inf"), float("inf")
    v[7, 0], v[7, 1] = 2.0 ** -126 * 127, 2.0 ** -126 * 3
    v[8, :] = -1.0
    for wide in (40, 40000):                                       # (in registers, and read twice)
        x = torch.zeros(9, wide)
        x[:, :40] = v
        codes, scales = lk.lutkan_quantise_int8(x.to(DEV))
        assert codes[0, :8].tolist() == [127, 0, 2, 2, 0, -2, -2, 126] and scales[0] == 1
        assert not bool(codes[1].any()) and scales[1] == 2.0 ** -126
        assert not bool(codes[2].any()) and scales[2] == 2.0 ** -126
        assert codes[3, 5] == 127 and codes[3, 6] in (-63, -64) and bool(torch.isfinite(scales[3]))
        assert bool(torch.isnan(scales[4:7]).all()) and not bool(codes[4:7].any())
        assert codes[7, 0] == 127 and codes[7, 1] == 3 and scales[7] == 2.0 ** -126
        assert bool((codes[8, :40] == -127).all())


@gpu
def test_rows_of_strided_and_repeated_matrices():
    v = torch.randn(5, 40, 333, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    for part in (v[:, :, 3:130], v[:, 5:20], v[1:2].expand(6, 40, 333), v[:, :1, 1:], v[:3, :, :1], v[:, 3:4, :].expand(5, 6, 333), v.transpose(0, 1)):
        codes, scales = lk.lutkan_quantise_int8(part)
        again = lk.lutkan_quantise_int8(part.contiguous())
        assert torch.equal(codes, again[0]) and torch.equal(scales, again[1]) and codes.is_contiguous()


# ---------------------------------------------------------------- norm
def norm_reference(x, weight, residual, eps):
    h = x.double().numpy() + (0 if residual is None else residual.double().numpy())
    return h, h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * weight.double().numpy()


def assert_norm(codes, scales, y, width):
    relative = (width + 16) * U
    scale = np.maximum(np.abs(y).max(1) / 127.0, 2.0 ** -126)
    got = scales.cpu().double().numpy()
    assert np.all(np.abs(got - scale) <= relative * scale + 2.0 ** -149)
    quotient = y / got[:, None]
    assert np.all(np.abs(codes.cpu().double().numpy() - quotient) <= 0.5 + 2 * relative * np.abs(quotient))


NORMS = [(1, 1), (3, 7), (5, 130), (1, 1024), (16, 512), (300, 520), (2100, 300), (2048, 2048), (1030, 5001), (1100, 8192), (9, 16400), (2, 32768)]


@gpu
@pytest.mark.parametrize("shape", NORMS, ids=str)
def test_norm(shape):
    rows, width = shape
    gen = torch.Generator().manual_seed(width)
    for x_type, r_type, w_type in [(torch.bfloat16, torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32, torch.float32), (torch.float16, torch.float32, torch.float32),
                                   (torch.float32, None, torch.float16), (torch.bfloat16, torch.float16, torch.float32)]:
        print(f"case norm {shape} {x_type} {r_type} {w_type}", flush=True)
        x, weight = torch.randn(rows, width, generator=gen).to(x_type), (1 + 0.3 * torch.randn(width, generator=gen)).to(w_type)
        residual = None if r_type is None else (2 * torch.randn(rows, width, generator=gen)).to(r_type)
        codes, scales, out = lk.lutkan_rmsnorm_int8(x.to(DEV), weight.to(DEV), residual=None if residual is None else residual.to(DEV), eps=1e-5)
        assert codes.dtype == torch.int8 and codes.shape == (rows, width) and scales.shape == (rows,)
        h32 = x.float() + (0 if residual is None else residual.float())
        _, y = norm_reference(h32, weight, None, 1e-5)              # (the sum is fp32's by definition)
        assert_norm(codes, scales, y, width)
        assert out is None if residual is None else torch.equal(out.cpu(), h32.to(r_type))


@gpu
@pytest.mark.parametrize("width", [40, 301, 2048, 5001])
def test_norm_of_strided_rows_in_place(width):
    rows = 70
    gen = torch.Generator(device=DEV).manual_seed(width)
    wide = torch.full((rows, width + 11), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 3:3 + width] = torch.randn(rows, width, generator=gen, device=DEV)
    res = torch.full((rows, width + 4), 5.0, device=DEV)
    res[:, 1:1 + width] = torch.randn(rows, width, generator=gen, device=DEV)
    x, residual = wide[:, 3:3 + width], res[:, 1:1 + width]
    weight = torch.ones(width, device=DEV)
    expected = lk.lutkan_rmsnorm_int8(x.contiguous(), weight, residual=residual.contiguous())
    codes, scales, out = lk.lutkan_rmsnorm_int8(x, weight, residual=residual, residual_out=residual)
    assert out.data_ptr() == residual.data_ptr()
    assert all(torch.equal(a, b) for a, b in zip((codes, scales, out), expected))
    assert bool((res[:, :1] == 5).all()) and bool((res[:, 1 + width:] == 5).all())


@gpu
@pytest.mark.parametrize("rows", [8, 1100, 2100])
@pytest.mark.parametrize("width", [7, 300, 1024, 2048, 5001, 32768])
def test_norm_of_rows_beyond_the_range_of_their_squares(rows, width):
    """Rows of 2^70 and 2^-70, of a large weight beside small ones, of zeros, with NaN and infinities, among ordinary ones."""
    if rows * width > 1 << 25:
        rows = 1030
    gen = torch.Generator().manual_seed(width)
    x = torch.randn(rows, width, generator=gen)
    x[0] *= 2.0 ** 70
    x[1] *= 2.0 ** -70
    x[2] = 0
    x[3, width - 1] = float("nan")
    x[4, 0] = float("inf")
    x[5] *= 2.0 ** 124
    weight = 1 + 0.3 * torch.randn(width, generator=gen)
    weight[width // 2] = 2.0 ** 20
    codes, scales, _ = lk.lutkan_rmsnorm_int8(x.to(DEV), weight.to(DEV), eps=0.0)
    keep = torch.tensor([i for i in range(rows) if i not in (2, 3, 4)])
    _, y = norm_reference(x[keep], weight, None, 0.0)
    assert_norm(codes[keep], scales[keep], y, width)
    assert bool(torch.isnan(scales[2:5]).all()) and not bool(codes[2:5].any())                  # (0 / 0 with eps 0)
    codes, scales, _ = lk.lutkan_rmsnorm_int8(x.to(DEV), weight.to(DEV), eps=1e-6)
    assert scales[2] == 2.0 ** -126 and not bool(codes[2].any())
    _, y = norm_reference(x[keep], weight, None, 1e-6)
    assert_norm(codes[keep], scales[keep], y, width)


# ---------------------------------------------------------------- streams and graphs
def _block(x, res, weight, w, ws, experts, es, sizes, rows):
    codes, scales, res = lk.lutkan_rmsnorm_int8(x, weight, residual=res)
    again = lk.lutkan_quantise_int8(x)
    y = lk.lutkan_matmul_int8(codes, scales, w, ws, dtype=torch.bfloat16)
    z = lk.lutkan_grouped_matmul_int8(codes, scales, experts, es, sizes, rows=rows)
    return codes, scales, res, *again, y, z


def _block_inputs(rows, width, n, experts):
    gen = torch.Generator(device=DEV).manual_seed(rows)
    x, res = (torch.randn(rows, width, generator=gen, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    w, ws = lk.lutkan_quantise_int8(torch.randn(n, width, generator=gen, device=DEV))
    e, es = lk.lutkan_quantise_int8(torch.randn(experts, n, width, generator=gen, device=DEV))
    order, _, sizes = lk.lutkan_expert_sort(torch.randint(0, experts, (rows, 2), generator=gen, device=DEV), experts)
    return x, res, torch.ones(width, device=DEV), w, ws, e, es, sizes, order


@gpu
@pytest.mark.parametrize("rows", [1, 300, 1500])
def test_another_stream_and_a_replayed_graph(rows):
    given = _block_inputs(rows, 384, 200, 5)
    eager = _block(*given)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = _block(*given)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _block(*given)
    for k in range(4):
        given[0].copy_(torch.randn_like(given[0]))
        given[8].copy_(given[8].roll(k))
        graph.replay()
        got = [t.clone() for t in held]
        torch.cuda.synchronize()
        expected = _block(*given)
        assert all(torch.equal(a, b) for a, b in zip(got, expected)), k
        torch.cuda.synchronize()


# ---------------------------------------------------------------- refusals (nothing is launched)
def _refused(code, rc):
    assert rc == code, (rc, lk.lutkan_last_error())
    assert lk.lutkan_last_error()


def test_the_library_refuses_bad_arguments():
    import ctypes as C
    lib = lk.load_library()
    A, M = binding._RmsnormFp8Args, binding._MatmulFp8Args

    def norm(**changes):
        a = A(4096, 4096, 4096, 4096, 4096, 4096, 128, 128, 128, 128, 1, 2, 128, 0, 0, 0, 1e-6)
        for k, v in changes.items():
            setattr(a, k, v)
        return lib.lutkan_rmsnorm_int8(C.byref(a), None)
    _refused(-1, lib.lutkan_rmsnorm_int8(None, None))
    for change in ({"x": None}, {"weight": None}, {"codes": None}, {"scales": None}, {"residual": None}, {"residual_out": None}, {"x_type": 3}, {"residual_type": -1},
                   {"weight_type": 9}, {"eps": -1.0}, {"eps": float("nan")}, {"width": 0}, {"rows": -1}):
        _refused(-1, norm(**change))
    for change in ({"codes_stride": 127}, {"scales_stride": 0}, {"residual_out_stride": 5}, {"x_stride": -128}, {"residual_stride": -1}):
        _refused(-2, norm(**change))
    _refused(-5, norm(width=32769, codes_stride=40000, residual_out_stride=40000))
    _refused(-5, norm(x_stride=1 << 31))
    assert norm(rows=0, x=None) == 0

    def rows(x=4096, t=0, matrices=1, n=4, k=4, stride=4, matrix_stride=16, codes=4096, scales=4096):
        return lib.lutkan_quantise_int8(x, t, matrices, n, k, stride, matrix_stride, codes, scales, None)
    for change in ({"x": None}, {"codes": None}, {"scales": None}, {"t": 3}, {"n": -1}, {"k": 0}, {"matrices": -1}):
        _refused(-1, rows(**change))
    _refused(-2, rows(stride=-1))
    _refused(-2, rows(matrix_stride=-1))
    _refused(-5, rows(k=131072))
    _refused(-5, rows(stride=1 << 31))
    assert rows(matrices=0, x=None) == 0 and rows(n=0, x=None) == 0

    def product(f="lutkan_matmul_int8", **changes):
        a = M(4096, 4096, 4096, 4096, 4096, 2, 128, 1, 128, 128 * 8, 8, 2, 128, 8, 0, 3, 4096, None, 8, 8)
        for k, v in changes.items():
            setattr(a, k, v)
        return getattr(lib, f)(C.byref(a), None)
    for f in ("lutkan_matmul_int8", "lutkan_grouped_matmul_int8"):
        _refused(-1, getattr(lib, f)(None, None))
        for change in ({"x": None}, {"x_scales": None}, {"weight": None}, {"weight_scales": None}, {"y": None}, {"k": 0}, {"n": 0}, {"y_type": 3}, {"rows": -1}, {"x_rows": -1}):
            _refused(-1, product(f, **change))
        for change in ({"y_stride": 7}, {"x_stride": -1}, {"weight_stride": -1}, {"x_scales_stride": -1}, {"rows": 3}):
            _refused(-2, product(f, **change))
        for change in ({"k": 131072}, {"n": (1 << 20) + 1, "y_stride": 1 << 21}, {"x_stride": 1 << 31}, {"weight_stride": 1 << 31}, {"rows": 1 << 31, "x_rows": 1 << 31}):
            _refused(-5, product(f, **change))
        assert product(f, rows=0, x_rows=0) == 0
    f = "lutkan_grouped_matmul_int8"
    for change in ({"groups": 0}, {"group_sizes": None}, {"group_sizes_bytes": 2}, {"row_index": 4096, "row_index_bytes": 1}):
        _refused(-1, product(f, **change))
    for change in ({"weight_matrix_stride": -1}, {"row_index": 4096, "x_rows": 0}):
        _refused(-2, product(f, **change))
    _refused(-5, product(f, rows=(1 << 24) + 1, x_rows=(1 << 24) + 1))
    _refused(-5, product(f, groups=(1 << 20) + 1))


def _raises(words, f, *args, **kwargs):
    with pytest.raises(lk.LutKanError, match=words):
        f(*args, **kwargs)


def test_the_binding_refuses_tensors_of_the_wrong_shape_dtype_or_device():
    x = torch.zeros(4, 130)
    _raises("CUDA tensor", lk.lutkan_rmsnorm_int8, x, torch.ones(130))
    _raises("shape", lk.lutkan_rmsnorm_int8, x[0], torch.ones(130))
    _raises("dtype", lk.lutkan_rmsnorm_int8, x.double(), torch.ones(130))
    _raises("CUDA tensor", lk.lutkan_quantise_int8, x)
    _raises("shape", lk.lutkan_quantise_int8, x[0])
    _raises("dtype", lk.lutkan_quantise_int8, x.int())
    c = x.to(torch.int8)
    _raises("CUDA tensor", lk.lutkan_matmul_int8, c, torch.ones(4), c, torch.ones(4))
    _raises("dtype", lk.lutkan_matmul_int8, x, torch.ones(4), c, torch.ones(4))
    _raises("CUDA tensor", lk.lutkan_grouped_matmul_int8, c, torch.ones(4), c[None], torch.ones(1, 4), torch.ones(1, dtype=torch.int64))


@gpu
def test_the_binding_refuses_operands_that_do_not_fit():
    x, xs, w, ws = (t.to(DEV) for t in operands(3, 4, 130, 20, 2))
    one, ones = w[0], ws[0]
    f, g = lk.lutkan_matmul_int8, lk.lutkan_grouped_matmul_int8
    _raises("x_scales", f, x, xs[:3], one, ones)
    _raises("x_scales", f, x, xs[:, None], one, ones)
    _raises("x_scales", f, x, xs.cpu(), one, ones)
    _raises("x_scales", f, x, xs.double(), one, ones)
    _raises("weight must", f, x, xs, one[:, :129], ones)
    _raises("weight must", f, x, xs, w, ws)
    _raises("weight must", f, x, xs, one.view(torch.uint8), ones)
    _raises("weight_scales", f, x, xs, one, ws)
    _raises("contiguous columns", f, x.t().contiguous().t(), xs, one, ones)
    _raises("contiguous", f, x, xs, one, torch.ones(20, 2, device=DEV)[:, 0])
    _raises("dtype", f, x, xs, one, ones, dtype=torch.float64)
    _raises("y must", f, x, xs, one, ones, y=torch.empty(4, 21, device=DEV))
    _raises("overlap", f, x, xs, one, ones, y=torch.empty(1, 20, device=DEV).expand(4, 20))
    sizes = torch.tensor([2, 2], device=DEV)
    _raises("group_sizes", g, x, xs, w, ws, sizes[:1])
    _raises("group_sizes", g, x, xs, w, ws, sizes.cpu())
    _raises("group_sizes", g, x, xs, w, ws, sizes.float())
    _raises("rows", g, x, xs, w, ws, sizes, rows=torch.ones(4, device=DEV))
    _raises("rows", g, x, xs, w, ws, sizes, rows=sizes[None])
    _raises("y must", g, x, xs, w, ws, sizes, rows=sizes, y=torch.empty(4, 20, device=DEV))
    _raises("\\[-5\\]", f, torch.zeros((1, 131072), dtype=torch.int8, device=DEV), xs[:1], torch.zeros((1, 131072), dtype=torch.int8, device=DEV), ones[:1])
    v = torch.zeros(4, 130, device=DEV)
    _raises("weight", lk.lutkan_rmsnorm_int8, v, torch.ones(131, device=DEV))
    _raises("residual must", lk.lutkan_rmsnorm_int8, v, torch.ones(130, device=DEV), residual=v[:3])
    _raises("without a residual", lk.lutkan_rmsnorm_int8, v, torch.ones(130, device=DEV), residual_out=v)
    _raises("residual_out must", lk.lutkan_rmsnorm_int8, v, torch.ones(130, device=DEV), residual=v, residual_out=v.half())
    _raises("\\[-5\\]", lk.lutkan_rmsnorm_int8, torch.zeros(1, 40000, device=DEV), torch.ones(40000, device=DEV))
    _raises("\\[-5\\]", lk.lutkan_quantise_int8, torch.zeros(1, 131072, device=DEV))


# ---------------------------------------------------------------- converted weights, kept
@gpu
@pytest.mark.parametrize("general", [False, True], ids=["native", "general"])
@pytest.mark.parametrize("shape", [(300, 200), (8, 30, 70), (3, 40000)], ids=str)
def test_converted_weights_are_saved_and_loaded(shape, general, monkeypatch):
    """Codes and scales lie in storages of their own: formats that store whole storages, each of one type, take both."""
    import io
    if general:
        monkeypatch.setattr(binding, "_native", binding._GeneralPath)
    codes, scales = lk.lutkan_quantise_int8(torch.randn(shape, generator=torch.Generator().manual_seed(1)).to(DEV))
    held = [(t.untyped_storage().nbytes(), t.storage_offset()) for t in (codes, scales)]
    assert held == [(codes.numel(), 0), (4 * scales.numel(), 0)]
    file = io.BytesIO()
    torch.save({"codes": codes, "scales": scales}, file)
    file.seek(0)
    loaded = torch.load(file, weights_only=True)
    assert torch.equal(loaded["codes"], codes) and torch.equal(loaded["scales"], scales)


# ---------------------------------------------------------------- the norm, by the depth of its sums
SCALE_DEPTH = 33 * U
"""A lane adds at most 32 squares, one rounding each; six exchanges in a wave and at most 15 additions of the waves' sums follow, 53.  The mean has two more, and the root halves
them all: 27.5.  The root and its reciprocal, two products and the scale's quotient are one each: 32.5."""
CODE_DEPTH = 6.1 * U
"""The root cancels in y / scale: two products each in y and in the largest, the scale's quotient and the code's."""


def assert_norm_by_depth(codes, scales, y):
    scale = y.abs().amax(1) / 127
    assert bool(((scales.double() - scale).abs() <= SCALE_DEPTH * scale).all()), float((scales.double() / scale - 1).abs().max()) / U
    quotient = y / scale[:, None]
    off = (codes.double() - quotient).abs() - 0.5
    assert bool((off <= CODE_DEPTH * quotient.abs()).all()), float((off / quotient.abs()).max()) / U


@gpu
@pytest.mark.parametrize("rows", [60, 1030, 2100])
@pytest.mark.parametrize("width", [40, 511, 513, 1000, 1537, 2048, 3000, 4096, 5001, 8192, 16400, 32768])
def test_norm_where_one_column_decides(rows, width):
    """In each of the first rows one column, around the ends of lanes' columns, waves and the row, is 1000 times the others: a norm that misses it, or takes it twice, is far off.  The other
    rows are of equal size throughout: a column there is 1 / (2 width) of the scale, seven times the bound at the widest."""
    if rows * width > 20_000_000:
        rows = 1030
    gen = torch.Generator().manual_seed(width)
    x = torch.randn(rows, width, generator=gen).to(DEV)
    weight = (1 + 0.3 * torch.randn(width, generator=gen)).to(DEV)
    columns = sorted({c + d for c in (0, 8, 512, 1024, 1536, 2048, 4096, 8192, 12288, 16384, 24576, width // 8 * 8, width) for d in (-8, -1, 0, 1, 7)} & set(range(width)))
    for i in range(min(len(columns), rows)):
        x[i, columns[i]] = 1000.0 * (-1) ** i
    for power, eps in ((0, 1e-5), (70, 0.0), (-70, 0.0)):          # (squares in fp32's range, and beyond it on both sides)
        print(f"case norm depth {rows} {width} {power}", flush=True)
        h = x * 2.0 ** power
        y = h.double() / torch.sqrt(h.double().square().mean(1, keepdim=True) + eps) * weight.double()
        assert_norm_by_depth(*lk.lutkan_rmsnorm_int8(h, weight, eps=eps)[:2], y)
    half, residual = x.bfloat16(), (2 * torch.randn(rows, width, generator=gen)).half().to(DEV)
    h = half.float() + residual.float()
    y = h.double() / torch.sqrt(h.double().square().mean(1, keepdim=True) + 1e-5) * weight.bfloat16().double()
    codes, scales, out = lk.lutkan_rmsnorm_int8(half, weight.bfloat16(), residual=residual, eps=1e-5)
    assert_norm_by_depth(codes, scales, y)
    assert torch.equal(out, h.half())
