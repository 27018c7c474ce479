"""The products' tiled kernels (tiles through LDS) at the forms where they can go wrong, every output against 64 bits: operands and
outputs inside wider buffers of NaN, gathered rows, group sizes that are negative, too long or end before the rows, more groups than
a wave has lanes, codes that are NaN and scales that are not finite; and sums of small whole numbers, which have no rounding in
either matrix instruction, bit for bit.

The bounds of rounded products are those that test_fp8_operators.py derives."""
import pytest

torch = pytest.importorskip("torch")
import paper_2601_03332_amd as lk  # noqa: E402
from paper_2601_03332_amd import binding  # noqa: E402
from test_fp8_operators import DEV, F8, HALF_UNIT, VALUES, gpu, random_codes  # noqa: E402

# 32-bit output, rows, k, n, groups (0: one weight).  Rows of k % 4 == 0 lie at dword addresses here and are copied straight to LDS,
# others at odd ones.  For each of the four kinds: 64 x 64 tiles with four and two teams, 128 x 128 with two and one (and 256 x 256).
DENSE = [
    (False, 3244, 1128, 161, 0), (False, 3685, 716, 225, 0), (False, 3286, 3140, 595, 0), (False, 2378, 124, 2246, 0), (False, 3489, 264, 3001, 0),
    (False, 2449, 617, 194, 0), (False, 3278, 373, 225, 0), (False, 2978, 2109, 641, 0), (False, 3175, 121, 842, 0),
    (True, 2502, 1028, 293, 0), (True, 1924, 368, 979, 0), (True, 2712, 1668, 715, 0), (True, 3277, 120, 1674, 0),
    (True, 3043, 1071, 294, 0), (True, 2039, 1131, 461, 0), (True, 3642, 1345, 531, 0), (True, 3210, 127, 1519, 0),
]
GROUPED = [
    (False, 1331, 3116, 99, 5), (False, 2568, 788, 327, 5), (False, 2846, 3108, 835, 5), (False, 3337, 116, 965, 5), (False, 3574, 300, 3801, 5),
    (False, 1304, 1525, 97, 5), (False, 3169, 369, 194, 5), (False, 3741, 2091, 587, 5), (False, 2806, 125, 527, 5), (False, 512, 4097, 256, 8),
    (True, 3536, 1144, 129, 5), (True, 2973, 360, 514, 5), (True, 3324, 1288, 798, 5), (True, 3979, 108, 870, 5),
    (True, 3762, 1147, 163, 5), (True, 3435, 895, 237, 5), (True, 1850, 1281, 1037, 5), (True, 3965, 119, 739, 5),
    (False, 3269, 1492, 71, 75), (False, 3706, 868, 131, 75), (False, 3979, 120, 591, 75), (False, 2474, 969, 71, 75), (False, 3443, 2087, 331, 75),
    (True, 3797, 1048, 98, 75), (True, 3887, 116, 609, 75), (True, 3641, 1463, 97, 75), (True, 3797, 125, 554, 75),
]
WIDE, HALF = [torch.float32], [torch.float16, torch.bfloat16]


def name(case):
    return "-".join(str(v) for v in case)


def values_of(codes):
    return torch.from_numpy(VALUES).to(codes.device)[codes.contiguous().view(torch.uint8).long()]


def weighted(codes, scales, rows_too=False):
    """The values that codes and scales stand for, in 64 bits."""
    s = scales.double().repeat_interleave(128, -1)[..., :codes.shape[-1]]
    if rows_too:
        s = s.repeat_interleave(128, -2)[..., :codes.shape[-2], :]
    return values_of(codes) * s


def operands(seed, rows, k, n, groups):
    gen = torch.Generator().manual_seed(seed)
    lead = [groups] if groups else []
    xs = torch.exp(torch.randn(rows, -(-k // 128), generator=gen))
    ws = torch.exp(torch.randn(*lead, -(-n // 128), -(-k // 128), generator=gen)) * 0.01
    return [t.to(DEV) for t in (random_codes(gen, (rows, k)), xs, random_codes(gen, (*lead, n, k)), ws)]


def guarded(t, before, after, fill):
    """t inside a buffer that is `fill` around it: columns on both sides, and a row more at either end of each matrix."""
    raw = t.view(torch.uint8) if t.dtype == F8 else t
    wide = torch.full((*raw.shape[:-2], raw.shape[-2] + 2, raw.shape[-1] + before + after), fill, dtype=raw.dtype, device=DEV)
    part = wide[..., 1:-1, before:before + raw.shape[-1]]
    part.copy_(raw)
    return part.view(F8) if t.dtype == F8 else part


def around(k):
    """Columns before and after that leave rows at dword addresses, or put them at odd ones."""
    return (4, 8) if k % 4 == 0 else (3, 9)


def assert_plan(k):
    plan = lk.lutkan_last_plan()
    assert plan.startswith("fp8_tiled") and ("async" in plan) == (k % 4 == 0), plan


def assert_close(y, ref, A, k, dtype):
    bound = ((min(k, 128) + -(-k // 128) + 24) * 2.0 ** -23 + (0.0 if dtype == torch.float32 else 2.0 ** -10)) * A
    limit = bound + HALF_UNIT[dtype] * (ref.abs() + bound) + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    off, finite = (y.double() - ref).abs(), torch.ones_like(ref, dtype=torch.bool)
    if dtype == torch.float16:                                     # beyond its range: infinite
        finite = ref.abs() <= 65000
        assert bool(torch.isinf(y[ref.abs() > 66000]).all())
    assert bool((off[finite] <= limit[finite]).all()), float((off / limit)[finite].max())


def groups_of(sizes, rows):
    """(expert, first, end) of the groups that have rows."""
    first = 0
    for e, size in enumerate(sizes):
        end = min(first + max(size, 0), rows)
        if end > first:
            yield e, first, end
        first = end


def sizes_for(kind, groups, rows, gen):
    cuts = [0] + torch.sort(torch.randint(0, rows + 1, (groups - 1,), generator=gen)).values.tolist() + [rows]
    sizes = [b - a for a, b in zip(cuts, cuts[1:])]
    if kind == "short":                                            # empty and negative ones, and rows behind the last group
        sizes = [0 if i % 5 == 1 else s * 3 // 4 for i, s in enumerate(sizes)]
        sizes[2] = -7
    elif kind == "long":                                           # the last groups begin behind the rows' end, one before them crosses it
        sizes = [s + s // 2 + 3 for s in sizes]
        sizes[-1] = 1 << 30
    return sizes


@gpu
@pytest.mark.parametrize("case", DENSE, ids=name)
def test_tiled_product_of_guarded_operands(case):
    wide, rows, k, n, _ = case
    print(f"case tiled product {case}", flush=True)
    x, xs, w, ws = operands(rows + k, rows, k, n, 0)
    xv, wv = weighted(x, xs), weighted(w, ws, True)
    ref, A = xv @ wv.t().contiguous(), xv.abs() @ wv.abs().t().contiguous()
    before, after = around(k)
    given = guarded(x, before, after, 127), guarded(xs, 1, 2, float("nan")), guarded(w, after, before, 127), ws
    for dtype in WIDE if wide else HALF:
        out = torch.full((rows + 2, n + 5), 7.0, dtype=dtype, device=DEV)
        lk.lutkan_matmul_fp8(*given, y=out[1:-1, 2:2 + n])
        assert_plan(k)
        y = out[1:-1, 2:2 + n].clone()
        assert_close(y, ref, A, k, dtype)
        out[1:-1, 2:2 + n] = 7.0
        assert bool((out == 7).all())
        assert torch.equal(lk.lutkan_matmul_fp8(*given, dtype=dtype), y)
        repeated = lk.lutkan_matmul_fp8(given[0][5:6].expand(rows, k), given[1][5:6].expand(rows, -1), *given[2:], dtype=dtype)
        assert torch.equal(repeated, repeated[:1].expand(rows, n))
        assert_close(repeated, ref[5:6].expand(rows, n), A[5:6].expand(rows, n), k, dtype)


@gpu
@pytest.mark.parametrize("kind", ["short", "long"])
@pytest.mark.parametrize("case", GROUPED, ids=name)
def test_tiled_grouped_product_of_gathered_rows(case, kind):
    wide, rows, k, n, groups = case
    print(f"case tiled grouped {case} {kind}", flush=True)
    gen = torch.Generator().manual_seed(rows + n)
    x_rows = 300
    x, xs, w, ws = operands(rows + k, x_rows, k, n, groups)
    index = torch.randint(0, x_rows, (rows,), generator=gen)
    index[torch.randint(0, rows, (40,), generator=gen)] = -1       # rows of zeros
    index[torch.randint(0, rows, (40,), generator=gen)] = x_rows
    index[0], index[rows - 1] = x_rows - 1, 0
    sizes = sizes_for(kind, groups, rows, gen)
    xv = torch.cat([weighted(x, xs), torch.zeros(1, k, dtype=torch.float64, device=DEV)])
    from_row = torch.where((index < 0) | (index >= x_rows), x_rows, index).to(DEV)
    ref, A = (torch.zeros(rows, n, dtype=torch.float64, device=DEV) for _ in range(2))
    for e, first, end in groups_of(sizes, rows):
        wv, part = weighted(w[e], ws[e], True), xv[from_row[first:end]]
        ref[first:end], A[first:end] = part @ wv.t().contiguous(), part.abs() @ wv.abs().t().contiguous()
    before, after = around(k)
    given = guarded(x, before, after, 127), guarded(xs, 1, 2, float("nan")), guarded(w, after, before, 127), ws
    for dtype, integers in zip(WIDE if wide else HALF, [torch.int64, torch.int32] if kind == "short" else [torch.int32, torch.int64]):
        where, source = torch.tensor(sizes, dtype=integers, device=DEV), index.to(integers).to(DEV)
        out = torch.full((rows + 2, n + 5), 7.0, dtype=dtype, device=DEV)
        lk.lutkan_grouped_matmul_fp8(*given, where, rows=source, y=out[1:-1, 2:2 + n])
        assert_plan(k)
        y = out[1:-1, 2:2 + n].clone()
        assert_close(y, ref, A, k, dtype)
        assert bool((y[ref.abs().sum(1) == 0] == 0).all())
        out[1:-1, 2:2 + n] = 7.0
        assert bool((out == 7).all())
        native = binding._native_calls().matmul_fp8(*given, dtype, where, source)
        assert native is not None and torch.equal(native, y)


@gpu
@pytest.mark.parametrize("case", DENSE + GROUPED, ids=name)
def test_tiled_sums_of_whole_numbers_are_exact(case):
    """Codes 0, 1, 2 and their negatives, scales 1/2, 1 and 2: every sum is a multiple of 1/4 below 2^18, which fp32 holds, and within a
    group of eight products nothing lies 13 bits below the largest.  One input, row or column that is missing or at a wrong place
    changes outputs by at least a unit of theirs."""
    wide, rows, k, n, groups = case
    print(f"case exact {case}", flush=True)
    gen = torch.Generator().manual_seed(k)
    codes = torch.tensor([0x00, 0x38, 0x40, 0xb8, 0xc0], dtype=torch.uint8)         # 0, 1, 2, -1, -2
    lead = [groups] if groups else []

    def pick(*shape):
        return codes[torch.randint(0, 5, shape, generator=gen)].view(F8).to(DEV)

    def power(*shape):
        return torch.exp2(torch.randint(-1, 2, shape, generator=gen).float()).to(DEV)
    blocks = -(-k // 128)
    x, xs, w, ws = pick(rows, k), power(rows, blocks), pick(*lead, n, k), power(*lead, -(-n // 128), blocks)
    sizes = sizes_for("even", groups, rows, gen) if groups else [rows]
    xv, ref = weighted(x, xs), torch.zeros(rows, n, dtype=torch.float64, device=DEV)
    for e, first, end in groups_of(sizes, rows):
        ref[first:end] = xv[first:end] @ weighted(w[e] if groups else w, ws[e] if groups else ws, True).t().contiguous()
    assert float(ref.abs().max()) < 2.0 ** 18
    for dtype in WIDE if wide else HALF:
        if groups:
            y = lk.lutkan_grouped_matmul_fp8(x, xs, w, ws, torch.tensor(sizes, device=DEV), dtype=dtype)
        else:
            y = lk.lutkan_matmul_fp8(x, xs, w, ws, dtype=dtype)
        assert_plan(k)
        assert torch.equal(y, ref.float().to(dtype))


@gpu
@pytest.mark.parametrize("case", DENSE + GROUPED[:10] + [(False, 5, 300, 260, 0), (False, 200, 300, 260, 0), (False, 40, 301, 260, 0), (False, 200, 300, 260, 3)], ids=name)
def test_what_is_not_finite_reaches_its_own_rows_and_columns_alone(case):
    """NaN codes and infinite scales, in the first, a middle and the last block of the inputs, through both matrix instructions."""
    wide, rows, k, n, groups = case
    print(f"case not finite {case}", flush=True)
    x, xs, w, ws = operands(rows + n, rows, k, n, groups)
    last = -(-k // 128) - 1
    xb, wb = x.view(torch.uint8), w.view(torch.uint8)
    xb[2, k - 1], xb[rows - 1, k // 2], xs[3, last] = 127, 255, float("inf")
    one = wb[1] if groups else wb
    one[7, 0], one[n - 1, k - 1] = 255, 127
    if n > 256:
        (ws[1] if groups else ws)[1, last // 2] = float("inf")
    sizes = [rows // 4, rows // 2] + [rows // 4] * (groups - 2) if groups else [rows]
    clean = [torch.where((b & 127) == 127, torch.zeros_like(b), b).view(F8) for b in (xb, wb)]
    xv = weighted(clean[0], xs.nan_to_num(posinf=1.0))
    ref, A = (torch.zeros(rows, n, dtype=torch.float64, device=DEV) for _ in range(2))
    bad = torch.zeros(rows, n, dtype=torch.bool, device=DEV)
    for e, first, end in groups_of(sizes, rows):
        wv = weighted(clean[1][e] if groups else clean[1], (ws[e] if groups else ws).nan_to_num(posinf=1.0), True)
        ref[first:end], A[first:end] = xv[first:end] @ wv.t().contiguous(), xv[first:end].abs() @ wv.abs().t().contiguous()
        for row in (2, 3, rows - 1):
            if first <= row < end:
                bad[row] = True
        if e == 1 or not groups:
            bad[first:end, [7, n - 1]] = True
            if n > 256:
                bad[first:end, 128:256] = True
    for dtype in WIDE if wide else HALF:
        ref_now = torch.where(ref.abs() < 60000, ref, 0) if dtype == torch.float16 else ref
        kept = ref_now == ref
        if groups:
            y = lk.lutkan_grouped_matmul_fp8(x, xs, w, ws, torch.tensor(sizes, device=DEV), dtype=dtype)
        else:
            y = lk.lutkan_matmul_fp8(x, xs, w, ws, dtype=dtype)
        assert torch.equal(~torch.isfinite(y)[kept], bad[kept])
        fine = kept & ~bad
        assert_close(y[fine], ref[fine], A[fine], k, dtype)


@gpu
def test_tiled_rows_at_offsets_beyond_32_bits():
    """A few rows gathered from the end of a wide x: offsets above 2^31 that the copies into LDS hold as unsigned, and rows whose offsets do not
    fit 32 bits, which are read through registers."""
    k, n, groups, rows = 516, 2500, 5, 1174
    w, ws = operands(1, 1, k, n, groups)[2:]
    sizes = torch.tensor([200, 400, 0, 300, 274], device=DEV)
    index = torch.randint(0, 200, (rows,), generator=torch.Generator().manual_seed(2)).to(DEV)
    for stride, fits in ((20_000_000, True), (24_000_000, False)):
        x_rows = 201 if fits else 200
        print(f"case far rows {stride}", flush=True)
        store = torch.zeros(stride * (x_rows - 1) + k, dtype=torch.uint8, device=DEV)
        x = store.as_strided((x_rows, k), (stride, 1))
        small, xs = operands(3, x_rows, k, n, 0)[:2]
        x.copy_(small.view(torch.uint8))
        y = lk.lutkan_grouped_matmul_fp8(x.view(F8), xs, w, ws, sizes, rows=index, dtype=torch.bfloat16)
        plan = lk.lutkan_last_plan()
        assert plan.startswith("fp8_tiled") and ("async" in plan) == fits, plan
        expected = lk.lutkan_grouped_matmul_fp8(small, xs, w, ws, sizes, rows=index, dtype=torch.bfloat16)
        assert "async" in lk.lutkan_last_plan()
        assert torch.equal(y, expected)
        del store, x, y


# ---------------------------------------------------------------- the norm, by the depth of its sums
NORM_DEPTH = 64 * 2.0 ** -24
"""A lane adds at most 32 squares, one rounding each; six exchanges in a wave and at most 16 waves' sums follow: 54 halves of a unit
2^-23, and h, its square, the mean, the root, its reciprocal, two factors and the scale's quotient are at most ten more; a part of
them counts by half, as a root halves it."""


@gpu
@pytest.mark.parametrize("rows", [60, 1030, 2100], ids=str)
@pytest.mark.parametrize("width", [40, 511, 513, 1000, 1537, 2048, 3000, 4096, 5001, 8192, 16400, 32768])
def test_norm_where_one_column_decides(rows, width):
    """In each row one column, around the ends of lanes' columns, waves and the row, is 1000 times the others: a norm that misses it, or
    takes it twice, is far off.  The other rows are of equal size throughout."""
    if rows * width > 20_000_000:
        rows = 1030
    print(f"case norm depth {rows} {width}", flush=True)
    gen = torch.Generator().manual_seed(width)
    x = torch.randn(rows, width, generator=gen).to(DEV)
    weight = (1 + 0.3 * torch.randn(width, generator=gen)).to(DEV)
    edges = sorted({c + d for c in (0, 8, 512, 1024, 1536, 2048, 4096, 8192, 12288, 16384, 24576, width // 8 * 8, width) for d in (-8, -1, 0, 1, 7)} & set(range(width)))
    for i in range(min(len(edges), rows)):
        x[i, edges[i]] = 1000.0 * (-1) ** i
    y = x.double() / torch.sqrt(x.double().square().mean(1, keepdim=True) + 1e-5) * weight.double()
    codes, scales, _ = lk.lutkan_rmsnorm_fp8(x, weight, eps=1e-5)
    blocks = -(-width // 128)
    exact = torch.nn.functional.pad(y.abs(), (0, blocks * 128 - width)).view(rows, blocks, 128).amax(2) / 448
    assert bool(((scales.double() - exact).abs() <= NORM_DEPTH * exact).all()), float((scales.double() / exact - 1).abs().max())
    v = y / exact.repeat_interleave(128, 1)[:, :width]
    step = torch.exp2(torch.floor(torch.log2((v.abs() * (1 + 2 * NORM_DEPTH)).clamp(2.0 ** -6))).clamp(max=8) - 3)
    assert bool(((values_of(codes) - v).abs() <= 0.5 * step + 2 * NORM_DEPTH * v.abs()).all())


# ---------------------------------------------------------------- the native calls, where operators are intercepted
@gpu
def test_native_8_bit_calls_leave_deferred_and_traced_operators_to_the_general_path():
    from torch._subclasses import FakeTensorMode
    from torch.utils._python_dispatch import TorchDispatchMode
    native = binding._native_calls()
    rows, width, n = 12, 256, 20
    t = torch.randn(rows, width, device=DEV)
    weight, sizes = torch.ones(width, device=DEV), torch.tensor([5, 7], device=DEV)
    w, ws = lk.lutkan_quantise_fp8(torch.randn(n, width, device=DEV))
    e, es = lk.lutkan_quantise_fp8(torch.randn(2, n, width, device=DEV))
    codes, _, _ = lk.lutkan_rmsnorm_fp8(t, weight)
    calls = [lambda v: native.rmsnorm_fp8(v, weight, None, 1e-6), lambda v: native.rmsnorm_fp8(t, weight, v, 1e-6), lambda v: native.quantise_fp8(v),
             lambda v: native.matmul_fp8(codes, v[:, :2], w, ws, torch.float32), lambda v: native.matmul_fp8(codes, v[:, :2], e, es, torch.bfloat16, sizes, None)]

    def plain(out):
        out = out if isinstance(out, tuple) else (out,)
        return [o.view(torch.uint8) if o.dtype == F8 else o for o in out if o is not None]
    expect = [plain(call(t)) for call in calls]
    with torch.inference_mode():
        for call, y in zip(calls, expect):
            got = plain(call(t))
            assert all(torch.equal(a, b) for a, b in zip(got, y)) and all(a.is_inference() for a in got)

    class Passes(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            return func(*args, **(kwargs or {}))
    taken = []

    def ask(v):
        full = v if v.dim() == 2 else v[None].expand(rows, -1)
        taken.extend(call(full) for call in calls)
        return v + 1.0
    with FakeTensorMode(allow_non_fake_inputs=True) as mode:
        ask(mode.from_tensor(t))
        ask(t)
    with Passes():
        ask(t)
        general = lk.lutkan_rmsnorm_fp8(t, weight)                # the general path serves it
    assert torch.equal(general[0].view(torch.uint8), expect[0][0]) and torch.equal(general[1], expect[0][1])
    torch.func.vmap(ask)(t)
    torch.func.grad(lambda v: ask(v).sum())(t)
    torch.func.jvp(ask, (t,), (torch.ones_like(t),))
    torch.func.functionalize(ask)(t)
    torch.jit.trace(ask, (t,), check_trace=False)
    assert len(taken) == len(calls) * 8 and all(y is None for y in taken), [y is None for y in taken]
    for call, y in zip(calls, expect):                            # and nothing of it is left behind
        assert all(torch.equal(a, b) for a, b in zip(plain(call(t)), y))
