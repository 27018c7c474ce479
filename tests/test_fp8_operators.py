"""The 8-bit operators around a layer against their definition in 64 bits (numpy, on the CPU).

Bounds, from the arithmetic:
  product     an e4m3 product is exact in fp32.  Outputs of 32 bits: a block of at most 128 of them is summed with an error of at most 2^-23
              of the sum of magnitudes per addition (rounding or truncation), then one multiplication of scales, one fused multiply-add
              per block and at most 16 partial sums, half a unit each: (min(k, 128) + blocks + 24) 2^-23 A with A = sum of |x w| in
              values.  Outputs of 16 bits: the 8-bit matrix instruction cuts, in every group of eight products, the seven others at 2^-13 of
              the leading bit of the largest: 7 * 2^-13 of it, and A is at least the sum of the largest: 2^-10 A more.
              Then the rounding of the output, half a unit of its type.
  norm        a sum of squares of `width` terms, root, quotient: (width + 16) 2^-24 relative for y and the scales; a code is off its exact
              value y / scale by half a step of e4m3 there, plus that relative error of the value.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2601_03332_amd as lk  # noqa: E402
from paper_2601_03332_amd import binding  # noqa: E402

DEV = "cuda:0"
gpu = pytest.mark.gpu
F8 = torch.float8_e4m3fn
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}     # (bf16: 8 bits, half a unit 2^-9; twice for the value's own error)
FLOATS = [torch.float32, torch.float16, torch.bfloat16]


def _table():
    v = np.arange(256)
    e, m = (v >> 3) & 15, v & 7
    x = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    x = np.where((v & 127) == 127, np.nan, x)
    return np.where(v >= 128, -x, x)


VALUES = _table()


def decode(codes):
    return VALUES[codes.detach().cpu().contiguous().view(torch.uint8).numpy()]


def spread(scales, shape, rows_too):
    s = scales.detach().cpu().double().numpy()
    s = np.repeat(s, 128, axis=-1)[..., :shape[-1]]
    return np.repeat(s, 128, axis=-2)[..., :shape[-2], :] if rows_too else s


def random_codes(gen, shape, nan=False):
    c = torch.randint(0, 256, shape, generator=gen, dtype=torch.int32).to(torch.uint8)
    if not nan:
        c = torch.where((c & 127) == 127, torch.zeros_like(c), c)
    return c.view(F8)


def random_operands(seed, rows, k, n, experts=None):
    gen = torch.Generator().manual_seed(seed)
    lead = [] if experts is None else [experts]
    x, w = random_codes(gen, (rows, k)), random_codes(gen, (*lead, n, k))
    xs = torch.exp(torch.randn(rows, -(-k // 128), generator=gen))
    ws = torch.exp(torch.randn(*lead, -(-n // 128), -(-k // 128), generator=gen)) * 0.01
    return x, xs, w, ws


def product_reference(x, xs, w, ws):
    """(y, A): the product and the sum of its terms' magnitudes, in 64 bits."""
    xv = decode(x) * spread(xs, x.shape, False)
    wv = decode(w) * spread(ws, w.shape, True)
    return xv @ wv.T, np.abs(xv) @ np.abs(wv).T


def assert_product(y, ref, A, k):
    got = y.detach().cpu().double().numpy()
    bound = ((min(k, 128) + -(-k // 128) + 24) * 2.0 ** -23 + (0.0 if y.dtype == torch.float32 else 2.0 ** -10)) * A
    limit = bound + HALF_UNIT[y.dtype] * (np.abs(ref) + bound) + (2.0 ** -25 if y.dtype == torch.float16 else 0.0)
    if y.dtype == torch.float16:                                   # beyond its range: infinite
        over = np.abs(ref) > 65000
        assert np.all(np.isinf(got[np.abs(ref) > 66000]))
        got, ref, limit = got[~over], ref[~over], limit[~over]
    assert np.all(np.abs(got - ref) <= limit), float(np.max(np.abs(got - ref) / np.maximum(limit, 1e-300)))


# ---------------------------------------------------------------- products
SHAPES = [(1, 1, 1), (1, 16, 2), (3, 15, 5), (2, 17, 3), (1, 128, 16), (16, 127, 17), (17, 129, 33), (5, 144, 4), (33, 200, 300), (1, 1024, 40),
          (15, 2056, 31), (64, 256, 128), (65, 384, 130), (130, 512, 64), (257, 200, 129), (300, 640, 260), (513, 128, 516), (700, 1300, 20)]


@gpu
@pytest.mark.parametrize("dtype", FLOATS, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_product(shape, dtype):
    rows, k, n = shape
    print(f"case product {shape} {dtype}", flush=True)
    x, xs, w, ws = random_operands(rows * 7 + k, rows, k, n)
    ref, A = product_reference(x, xs, w, ws)
    y = lk.lutkan_matmul_fp8(x.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV), dtype=dtype)
    assert y.shape == (rows, n) and y.dtype == dtype
    assert lk.lutkan_last_plan().startswith("fp8_")
    assert_product(y, ref, A, k)


@gpu
def test_product_defaults_to_32_bits_and_repeats_its_bits():
    x, xs, w, ws = (t.to(DEV) for t in random_operands(5, 100, 1000, 200))
    y = lk.lutkan_matmul_fp8(x, xs, w, ws)
    assert y.dtype == torch.float32
    for _ in range(3):
        assert torch.equal(y, lk.lutkan_matmul_fp8(x, xs, w, ws))


@gpu
@pytest.mark.parametrize("shape", [(1, 130, 20), (40, 256, 48), (70, 300, 131), (600, 512, 384)], ids=str)
def test_product_of_strided_unaligned_and_repeated_rows(shape):
    """Operands that are parts of wider or oddly placed buffers; what lies around them is NaN, and around y stays what it was."""
    rows, k, n = shape
    print(f"case strided {shape}", flush=True)
    x, xs, w, ws = random_operands(11, rows, k, n)
    ref, A = product_reference(x, xs, w, ws)

    def inside(t, before, after, fill):
        wide = torch.full((t.shape[0], t.shape[1] + before + after), fill, dtype=torch.uint8 if t.dtype == F8 else t.dtype, device=DEV)
        raw = t.view(torch.uint8) if t.dtype == F8 else t
        wide[:, before:before + t.shape[1]] = raw.to(DEV)
        part = wide[:, before:before + t.shape[1]]
        return part.view(F8) if t.dtype == F8 else part

    for before, after in ((3, 8), (16, 32), (1, 0)):
        out = torch.full((rows, n + 5), 7.0, dtype=torch.bfloat16, device=DEV)
        y = lk.lutkan_matmul_fp8(inside(x, before, after, 127), inside(xs, 1, 2, float("nan")), inside(w, after, before, 127), ws.to(DEV), y=out[:, 2:2 + n])
        assert y.data_ptr() == out[:, 2:].data_ptr()
        assert_product(y, ref, A, k)
        assert bool((out[:, :2] == 7).all()) and bool((out[:, 2 + n:] == 7).all())
    one = lk.lutkan_matmul_fp8(x[:1].to(DEV).expand(rows, k), xs[:1].to(DEV).expand(rows, -1), w.to(DEV), ws.to(DEV))
    assert_product(one, np.repeat(ref[:1], rows, 0), np.repeat(A[:1], rows, 0), k)


@gpu
def test_product_of_nan_codes_and_of_scales_that_are_not_finite():
    """They reach the outputs of their row (of x) or column (of the weight) and no others."""
    for rows in (5, 200):
        x, xs, w, ws = random_operands(17, rows, 300, 260)
        x = x.view(torch.uint8).clone()
        x[2, 299] = 127
        w = w.view(torch.uint8).clone()
        w[7, 0] = 255
        xs[3, 1] = float("inf")
        ref, A = product_reference(torch.where((x & 127) == 127, 0, x).to(torch.uint8).view(F8), xs.nan_to_num(posinf=1.0), torch.where((w & 127) == 127, 0, w).to(torch.uint8).view(F8), ws)
        y = lk.lutkan_matmul_fp8(x.view(F8).to(DEV), xs.to(DEV), w.view(F8).to(DEV), ws.to(DEV))
        bad = ~torch.isfinite(y).cpu().numpy()
        expected = np.zeros_like(bad)
        expected[[2, 3]] = True
        expected[:, 7] = True
        assert np.array_equal(bad, expected)
        fine = ~expected
        assert_product(torch.from_numpy(y.cpu().numpy()[fine]), ref[fine], A[fine], 300)


@gpu
def test_product_with_no_rows():
    x, xs, w, ws = (t.to(DEV) for t in random_operands(5, 4, 130, 20))
    assert lk.lutkan_matmul_fp8(x[:0], xs[:0], w, ws).shape == (0, 20)
    sizes = torch.zeros(3, dtype=torch.int64, device=DEV)
    three = w.view(torch.uint8).repeat(3, 1, 1).view(F8), ws.repeat(3, 1, 1)
    assert lk.lutkan_grouped_matmul_fp8(x[:0], xs[:0], *three, sizes).shape == (0, 20)
    nothing = torch.zeros(0, dtype=torch.int64, device=DEV)
    assert lk.lutkan_grouped_matmul_fp8(x, xs, *three, sizes, rows=nothing).shape == (0, 20)


# ---------------------------------------------------------------- products grouped by expert
def grouped_reference(x, xs, w, ws, sizes, index, rows):
    y, A, first = np.zeros((rows, w.shape[1])), np.zeros((rows, w.shape[1])), 0
    index = np.arange(rows) if index is None else index.numpy()
    for e, size in enumerate(sizes):
        at = np.arange(first, min(first + max(size, 0), rows))
        first = min(first + max(size, 0), rows)
        at = at[(index[at] >= 0) & (index[at] < x.shape[0])]
        if at.size:
            src = torch.from_numpy(index[at])
            y[at], A[at] = product_reference(x.view(torch.uint8)[src].view(F8), xs[src], w[e], ws[e])
    return y, A


GROUPINGS = [
    # rows of x, rows of y (None: no index), k, n, sizes
    (40, None, 200, 70, [10, 0, 25, 5]),
    (7, 20, 129, 33, [0, 0, 20, 0]),
    (9, 30, 64, 130, [3, 4, 5]),                                   # 18 rows behind the last group
    (1, 1, 1024, 48, [0, 1]),
    (50, 200, 256, 256, [64, 65, 63, 1, 0, 7]),
    (30, 25, 300, 20, [10, -5, 40, 3]),                            # a negative size is none, the third ends with the rows
    (300, 700, 384, 140, [0, 300, 1, 17, 200, 182]),
    (60, 500, 130, 20, [(i * 7) % 13 for i in range(80)]),         # more groups than a wave has lanes
    (10, 70, 16, 5, [1] * 70),
    (2000, None, 256, 300, [900, 0, 600, 500]),
    (300, 1500, 512, 272, [130, 700, 257, 20, 393]),
]


@gpu
@pytest.mark.parametrize("integers", [torch.int32, torch.int64], ids=str)
@pytest.mark.parametrize("case", GROUPINGS, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-{c[3]}-{len(c[4])}")
def test_grouped_product(case, integers):
    x_rows, rows, k, n, sizes = case
    print(f"case grouped {x_rows} {rows} {k} {n} {sizes} {integers}", flush=True)
    x, xs, w, ws = random_operands(x_rows + k, x_rows, k, n, len(sizes))
    index = None
    if rows is not None:
        index = torch.randint(0, x_rows, (rows,), generator=torch.Generator().manual_seed(3), dtype=torch.int64)
        if rows > 8:
            index[[2, 5]] = torch.tensor([-1, x_rows])             # rows of zeros
    count = x_rows if rows is None else rows
    ref, A = grouped_reference(x, xs, w, ws, sizes, index, count)
    dtype = torch.bfloat16 if integers == torch.int32 else torch.float32
    y = torch.full((count, n), 7.0, dtype=dtype, device=DEV)
    out = lk.lutkan_grouped_matmul_fp8(x.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV), torch.tensor(sizes, dtype=integers, device=DEV),
                                       rows=None if index is None else index.to(integers).to(DEV), y=y)
    assert out is y
    assert_product(y, ref, A, k)


@gpu
def test_grouped_product_agrees_with_the_product_of_each_group():
    x, xs, w, ws = (t.to(DEV) for t in random_operands(23, 900, 512, 256, 3))
    sizes = [200, 300, 400]
    y = lk.lutkan_grouped_matmul_fp8(x, xs, w, ws, torch.tensor(sizes, device=DEV))
    first = 0
    for e, size in enumerate(sizes):
        part = lk.lutkan_matmul_fp8(x[first:first + size], xs[first:first + size], w[e], ws[e])
        assert torch.allclose(y[first:first + size], part, rtol=1e-5, atol=1e-4 * float(part.abs().max()))
        first += size


# ---------------------------------------------------------------- each kernel of the products
D16, D32, D2 = "direct rows=16 columns=16", "direct rows=16 columns=32", "direct rows=32 columns=32"
T4, T2, U2, U1, V = "tiled rows=64 columns=64 teams=4", "tiled rows=64 columns=64 teams=2", "tiled rows=128 columns=128 teams=2", "tiled rows=128 columns=128 teams=1", "tiled rows=256"
KERNELS = [
    # kernel, 32-bit output, rows, k, n, groups (0: one weight); rows of an odd k lie at odd addresses
    (D16, False, 2, 104, 17, 0), (D32, False, 337, 108, 293, 0), (D2, False, 661, 104, 258, 0), (T4, False, 701, 896, 551, 0), (T2, False, 1133, 256, 772, 0),
    (U2, False, 614, 6472, 3900, 0), (U1, False, 715, 384, 2712, 0), (V, False, 5431, 132, 2197, 0),
    (D16, False, 2, 101, 17, 0), (D32, False, 244, 105, 402, 0), (D2, False, 484, 121, 353, 0), (T4, False, 619, 2995, 809, 0), (T2, False, 1003, 995, 970, 0),
    (U2, False, 680, 4109, 4920, 0), (U1, False, 1704, 478, 1176, 0),
    (D16, False, 3, 104, 17, 2), (D32, False, 361, 104, 277, 2), (D2, False, 737, 108, 227, 2), (T4, False, 1034, 2432, 296, 3), (T2, False, 1232, 1044, 819, 2),
    (U2, False, 809, 4288, 2770, 5), (U1, False, 1174, 384, 874, 2), (V, False, 5889, 392, 2536, 3),
    (D16, False, 2, 107, 18, 2), (D32, False, 431, 117, 239, 2), (D2, False, 1481, 105, 99, 3), (T2, False, 187, 1659, 1998, 8), (T2, False, 2234, 4181, 755, 8),
    (T2, False, 1623, 745, 515, 2), (U2, False, 1626, 2406, 1448, 2), (U1, False, 1454, 241, 641, 2),
    (D16, True, 2, 104, 17, 0), (D32, True, 325, 108, 311, 0), (D2, True, 747, 112, 225, 0), (T4, True, 823, 512, 781, 0), (T2, True, 1465, 640, 476, 0),
    (U2, True, 1964, 1620, 1555, 0), (U1, True, 1425, 760, 1571, 0),
    (D16, True, 2, 101, 17, 0), (D32, True, 334, 101, 311, 0), (D2, True, 388, 109, 452, 0), (T4, True, 914, 1565, 872, 0), (T2, True, 510, 1257, 1988, 0),
    (U2, True, 1133, 1591, 1838, 0), (U1, True, 1982, 498, 1221, 0),
    (D16, True, 2, 108, 19, 2), (D32, True, 435, 104, 227, 2), (D2, True, 956, 112, 168, 3), (T4, True, 1566, 1920, 206, 2), (T2, True, 2366, 512, 542, 3),
    (U2, True, 3120, 1572, 930, 2), (U1, True, 3800, 128, 615, 2),
    (D16, True, 3, 103, 17, 2), (D32, True, 924, 101, 98, 4), (D2, True, 964, 109, 167, 3), (T4, True, 822, 2521, 550, 2), (T2, True, 218, 837, 4147, 8),
    (U2, True, 1202, 1579, 1818, 2), (U1, True, 1667, 377, 975, 2),
]


@gpu
@pytest.mark.parametrize("case", KERNELS, ids=lambda c: "-".join(str(v) for v in c))
def test_each_kernel_of_the_products(case):
    """The launch rule's every kernel, at a size that the rule sends to it; a part of the rows and columns against 64 bits, all of them
    against the bits of a second call."""
    kernel, wide, rows, k, n, groups = case
    print(f"case kernel {case}", flush=True)
    gen = torch.Generator().manual_seed(rows + k + n)
    x, xs, w, ws = random_operands(rows + 3 * k, rows, k, n, groups or None)
    dtype = torch.float32 if wide else torch.bfloat16
    on = [t.to(DEV) for t in (x, xs, w, ws)]
    if groups:
        cuts = torch.sort(torch.randint(0, rows + 1, (groups - 1,), generator=gen)).values.tolist()
        sizes = [b - a for a, b in zip([0] + cuts, cuts + [rows])]
        where = torch.tensor(sizes, device=DEV)
        call = lambda: lk.lutkan_grouped_matmul_fp8(*on, where, dtype=dtype)  # noqa: E731
    else:
        sizes, (w, ws) = [rows], (t[None] for t in (w, ws))
        call = lambda: lk.lutkan_matmul_fp8(*on, dtype=dtype)  # noqa: E731
    y = call()
    assert kernel in lk.lutkan_last_plan(), lk.lutkan_last_plan()
    assert torch.equal(y, call())
    columns = torch.unique(torch.cat([torch.randint(0, n, (150,), generator=gen), torch.tensor([0, n - 1])]))
    first = 0
    for e, size in enumerate(sizes):
        if size:
            at = first + torch.unique(torch.cat([torch.randint(0, size, (60,), generator=gen), torch.tensor([0, size - 1])]))
            xv = decode(x.view(torch.uint8)[at].view(F8)) * spread(xs[at], (len(at), k), False)
            wv = decode(w[e].view(torch.uint8)[columns].view(F8)) * spread(ws[e][columns // 128], (len(columns), k), False)
            assert_product(y.cpu()[at][:, columns], xv @ wv.T, np.abs(xv) @ np.abs(wv).T, k)
        first += size


# ---------------------------------------------------------------- norm and conversion
def step_of(v):
    """Distance of neighbouring e4m3 values around |v|."""
    e = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
    return 2.0 ** (np.minimum(e, 8) - 3)


def assert_codes(codes, scales, value, scale, relative):
    """codes, scales: the kernel's; value, scale: in 64 bits, spread over the elements."""
    got = scales
    assert np.all(np.abs(got - scale) <= relative * scale), float(np.max(np.abs(got / scale - 1)))
    v = value / scale
    limit = 0.5 * step_of(np.abs(v) * (1 + 2 * relative)) + 2 * relative * np.abs(v)
    assert np.all(np.abs(codes - v) <= limit), float(np.max(np.abs(codes - v) - limit))


def row_scales(y):
    rows, width = y.shape
    nb = -(-width // 128)
    padded = np.pad(np.abs(y), ((0, 0), (0, nb * 128 - width))).reshape(rows, nb, 128)
    return np.maximum(padded.max(-1) / 448.0, 2.0 ** -126)


NORMS = [(1, 1), (1, 8), (2, 7), (1, 127), (3, 128), (5, 129), (4, 300), (1, 1024), (9, 1030), (130, 512), (2, 4096), (1, 5000), (3, 8192), (1, 16400), (2, 32768),
         (2100, 40), (2049, 1000), (2048, 2048), (1100, 1500), (1030, 3000), (1025, 5001)]


@gpu
@pytest.mark.parametrize("shape", NORMS, ids=str)
def test_norm(shape):
    rows, width = shape
    rng = np.random.default_rng(rows * 31 + width)
    picks = [(a, b) for a in FLOATS for b in FLOATS + [None]]
    for xt, rt in picks if rows * width < 20000 else picks[::5]:
        print(f"case norm {shape} {xt} {rt}", flush=True)
        x = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(xt)
        r = None if rt is None else torch.from_numpy(2 * rng.standard_normal(shape).astype(np.float32)).to(rt)
        weight = torch.from_numpy(1 + 0.3 * rng.standard_normal(width).astype(np.float32)).to(FLOATS[(rows + width) % 3])
        h = x.double().numpy() + (0 if r is None else r.double().numpy())
        y = h / np.sqrt((h * h).mean(1, keepdims=True) + 1e-5) * weight.double().numpy()
        codes, scales, out = lk.lutkan_rmsnorm_fp8(x.to(DEV), weight.to(DEV), residual=None if r is None else r.to(DEV), eps=1e-5)
        assert codes.dtype == F8 and codes.shape == shape and scales.shape == (rows, -(-width // 128))
        exact = row_scales(y)
        assert_codes(decode(codes), spread(scales, shape, False), y, np.repeat(exact, 128, 1)[:, :width], (width + 16) * 2.0 ** -24)
        if r is None:
            assert out is None
        else:
            assert out.dtype == rt
            assert np.all(np.abs(out.double().cpu().numpy() - h) <= HALF_UNIT[rt] * np.abs(h) + 2.0 ** -24 * np.abs(h) + 2.0 ** -25)


@gpu
@pytest.mark.parametrize("width", [40, 301, 2048, 5001])
def test_norm_of_strided_rows_in_place(width):
    rng = np.random.default_rng(width)
    for rows in (3, 2500):
        wide = torch.from_numpy(rng.standard_normal((rows, width + 9)).astype(np.float32)).to(torch.bfloat16).to(DEV)
        res = torch.from_numpy(rng.standard_normal((rows, width + 3)).astype(np.float32)).to(DEV)
        weight = torch.ones(width, dtype=torch.float16, device=DEV)
        x, r = wide[:, 5:5 + width], res[:, 1:1 + width]
        before = res.clone()
        fresh = lk.lutkan_rmsnorm_fp8(x.contiguous(), weight, residual=r.contiguous())
        codes, scales, out = lk.lutkan_rmsnorm_fp8(x, weight, residual=r, residual_out=r)
        assert out is r
        assert torch.equal(codes.view(torch.uint8), fresh[0].view(torch.uint8)) and torch.equal(scales, fresh[1]) and torch.equal(out, fresh[2])
        assert torch.equal(res[:, :1], before[:, :1]) and torch.equal(res[:, 1 + width:], before[:, 1 + width:])


@gpu
def test_norm_of_zeros_tiny_huge_and_not_finite_rows():
    x = torch.zeros(6, 300)
    x[1] = 1e-30
    x[2] = 1e18
    x[3, 4] = float("inf")
    x[4, 200] = float("nan")
    x[5, 0] = 1.0
    weight = torch.ones(300)
    codes, scales, _ = lk.lutkan_rmsnorm_fp8(x.to(DEV), weight.to(DEV), eps=1e-6)
    v = decode(codes) * spread(scales, x.shape, False)
    assert np.all(v[0] == 0) and np.all(np.abs(v[1] - 1e-27) <= 1e-28)
    assert np.all(np.abs(v[2] - 1.0) <= 1e-5)
    finite = np.arange(300) != 4
    assert np.isnan(v[3, 4]) and np.isnan(v[3, :128]).all() and np.all(v[3, 128:] == 0) and finite.sum() == 299
    assert np.isnan(v[4]).all()
    assert abs(v[5, 0] - 1 / np.sqrt(1 / 300 + 1e-6)) < 1e-3 and np.all(v[5, 1:] == 0)
    codes, scales, _ = lk.lutkan_rmsnorm_fp8(x[:1].to(DEV), weight.to(DEV), eps=0.0)          # 0 / 0
    assert np.isnan(decode(codes) * spread(scales, (1, 300), False)).all()
    assert lk.lutkan_rmsnorm_fp8(x[:0].to(DEV), weight.to(DEV))[0].shape == (0, 300)


@gpu
@pytest.mark.parametrize("shape", [(1, 1), (5, 3), (128, 128), (129, 127), (300, 200), (16, 1000), (3, 130, 260), (2, 7, 128), (1, 256, 512)], ids=str)
@pytest.mark.parametrize("dtype", FLOATS, ids=str)
def test_weights(shape, dtype):
    rng = np.random.default_rng(sum(shape))
    w = torch.from_numpy((rng.standard_normal(shape) * np.exp(rng.standard_normal(shape))).astype(np.float32)).to(dtype)
    wide = torch.full((*shape[:-1], shape[-1] + 3), float("nan"), dtype=dtype, device=DEV)
    wide[..., 1:1 + shape[-1]] = w.to(DEV)
    for given in (w.to(DEV), wide[..., 1:1 + shape[-1]]):
        codes, scales = lk.lutkan_quantise_fp8(given)
        assert codes.shape == w.shape and scales.shape == (*shape[:-2], -(-shape[-2] // 128), -(-shape[-1] // 128))
        v = w.double().numpy()
        n, k = shape[-2:]
        exact = np.zeros(scales.shape)
        for r in range(scales.shape[-2]):
            for c in range(scales.shape[-1]):
                exact[..., r, c] = np.maximum(np.abs(v[..., 128 * r:128 * r + 128, 128 * c:128 * c + 128]).max((-1, -2)) / 448.0, 2.0 ** -126)
        assert_codes(decode(codes), spread(scales, shape, True), v, spread(torch.from_numpy(exact), shape, True), 2.0 ** -22)


@gpu
def test_weights_that_are_not_finite_stand_for_nan_in_their_block_alone():
    w = torch.ones(256, 256)
    w[3, 200], w[130, 5] = float("nan"), float("-inf")
    codes, scales = lk.lutkan_quantise_fp8(w.to(DEV))
    v = decode(codes) * spread(scales, w.shape, True)
    assert np.isnan(v[:128, 128:]).all() and np.isnan(v[128:, :128]).all()
    assert np.all(np.abs(v[:128, :128] - 1) < 1e-6) and np.all(np.abs(v[128:, 128:] - 1) < 1e-6)


# ---------------------------------------------------------------- streams and graphs
def _block(x, res, weight, w, ws, experts, es, sizes, rows):
    codes, scales, res = lk.lutkan_rmsnorm_fp8(x, weight, residual=res)
    y = lk.lutkan_matmul_fp8(codes, scales, w, ws, dtype=torch.bfloat16)
    z = lk.lutkan_grouped_matmul_fp8(codes, scales, experts, es, sizes, rows=rows)
    return codes.view(torch.uint8), scales, res, y, z


def _block_inputs(rows, width, n, experts):
    gen = torch.Generator(device=DEV).manual_seed(rows)
    x, res = (torch.randn(rows, width, generator=gen, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    w, ws = lk.lutkan_quantise_fp8(torch.randn(n, width, generator=gen, device=DEV))
    e, es = lk.lutkan_quantise_fp8(torch.randn(experts, n, width, generator=gen, device=DEV))
    which = torch.randint(0, experts, (2 * rows,), generator=gen, device=DEV)
    order = torch.sort(which, stable=True).indices
    return x, res, torch.ones(width, device=DEV), w, ws, e, es, torch.bincount(which, minlength=experts), order // 2


@gpu
@pytest.mark.parametrize("rows", [1, 300])
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
        return lib.lutkan_rmsnorm_fp8(C.byref(a), None)
    _refused(-1, lib.lutkan_rmsnorm_fp8(None, None))
    for change in ({"x": None}, {"weight": None}, {"codes": None}, {"scales": None}, {"residual": None}, {"residual_out": None}, {"x_type": 3}, {"residual_type": -1},
                   {"weight_type": 9}, {"eps": -1.0}, {"eps": float("nan")}, {"width": 0}, {"rows": -1}):
        _refused(-1, norm(**change))
    for change in ({"codes_stride": 127}, {"scales_stride": 0}, {"residual_out_stride": 5}, {"x_stride": -128}, {"residual_stride": -1}):
        _refused(-2, norm(**change))
    _refused(-5, norm(width=32769, codes_stride=40000, scales_stride=400, residual_out_stride=40000))
    _refused(-5, norm(x_stride=1 << 31))
    assert norm(rows=0, x=None) == 0

    def weights(w=4096, t=0, matrices=1, n=4, k=4, stride=4, matrix_stride=16, codes=4096, scales=4096):
        return lib.lutkan_quantise_fp8(w, t, matrices, n, k, stride, matrix_stride, codes, scales, None)
    for change in ({"w": None}, {"codes": None}, {"scales": None}, {"t": 3}, {"n": 0}, {"k": 0}, {"matrices": -1}):
        _refused(-1, weights(**change))
    _refused(-2, weights(stride=-1))
    _refused(-5, weights(matrices=1 << 40))
    assert weights(matrices=0, w=None) == 0

    def product(f="lutkan_matmul_fp8", **changes):
        a = M(4096, 4096, 4096, 4096, 4096, 2, 128, 1, 128, 128 * 8, 8, 2, 128, 8, 0, 3, 4096, None, 8, 8)
        for k, v in changes.items():
            setattr(a, k, v)
        return getattr(lib, f)(C.byref(a), None)
    for f in ("lutkan_matmul_fp8", "lutkan_grouped_matmul_fp8"):
        _refused(-1, getattr(lib, f)(None, None))
        for change in ({"x": None}, {"x_scales": None}, {"weight": None}, {"weight_scales": None}, {"y": None}, {"k": 0}, {"n": 0}, {"y_type": 3}, {"rows": -1}, {"x_rows": -1}):
            _refused(-1, product(f, **change))
        for change in ({"y_stride": 7}, {"x_stride": -1}, {"weight_stride": -1}, {"x_scales_stride": -1}, {"rows": 3}):
            _refused(-2, product(f, **change))
        for change in ({"k": (1 << 20) + 1}, {"n": (1 << 20) + 1, "y_stride": 1 << 21}, {"x_stride": 1 << 31}, {"weight_stride": 1 << 31}, {"rows": 1 << 31, "x_rows": 1 << 31}):
            _refused(-5, product(f, **change))
        assert product(f, rows=0, x_rows=0) == 0
    f = "lutkan_grouped_matmul_fp8"
    for change in ({"groups": 0}, {"group_sizes": None}, {"group_sizes_bytes": 2}, {"row_index": 4096, "row_index_bytes": 1}):
        _refused(-1, product(f, **change))
    for change in ({"weight_matrix_stride": -1}, {"row_index": 4096, "x_rows": 0}):
        _refused(-2, product(f, **change))
    _refused(-5, product(f, rows=(1 << 24) + 1, x_rows=(1 << 24) + 1))


def test_the_binding_refuses_tensors_of_the_wrong_shape_dtype_or_device():
    def refused(words, f, *args, **kwargs):
        with pytest.raises(lk.LutKanError, match=words):
            f(*args, **kwargs)
    x = torch.zeros(4, 130)
    refused("CUDA tensor", lk.lutkan_rmsnorm_fp8, x, torch.ones(130))
    refused("shape", lk.lutkan_rmsnorm_fp8, x[0], torch.ones(130))
    refused("dtype", lk.lutkan_rmsnorm_fp8, x.double(), torch.ones(130))
    refused("shape", lk.lutkan_rmsnorm_fp8, None, torch.ones(130))
    refused("CUDA tensor", lk.lutkan_quantise_fp8, x)
    refused("shape", lk.lutkan_quantise_fp8, x[0])
    refused("dtype", lk.lutkan_quantise_fp8, x.int())
    c = x.to(F8)
    refused("CUDA tensor", lk.lutkan_matmul_fp8, c, torch.ones(4, 2), c, torch.ones(1, 2))
    refused("dtype", lk.lutkan_matmul_fp8, x, torch.ones(4, 2), c, torch.ones(1, 2))
    sizes = torch.ones(1, dtype=torch.int64)
    refused("group_sizes", lk.lutkan_grouped_matmul_fp8, c, torch.ones(4, 2), c[None], torch.ones(1, 1, 2), sizes)
    refused("group_sizes", lk.lutkan_grouped_matmul_fp8, c, torch.ones(4, 2), c[None], torch.ones(1, 1, 2), sizes.float())


@gpu
def test_the_binding_refuses_operands_that_do_not_fit():
    def refused(words, f, *args, **kwargs):
        with pytest.raises(lk.LutKanError, match=words):
            f(*args, **kwargs)
    x, xs, w, ws = (t.to(DEV) for t in random_operands(3, 4, 130, 20, 2))
    one, ones = w[0], ws[0]
    refused("x_scales", lk.lutkan_matmul_fp8, x, xs[:, :1], one, ones)
    refused("weight must", lk.lutkan_matmul_fp8, x, xs, one[:, :129], ones)
    refused("weight must", lk.lutkan_matmul_fp8, x, xs, w, ws)
    refused("weight_scales", lk.lutkan_matmul_fp8, x, xs, one, ws)
    refused("contiguous columns", lk.lutkan_matmul_fp8, x.t().contiguous().t(), xs, one, ones)
    refused("contiguous", lk.lutkan_matmul_fp8, x, xs, one, torch.ones(2, 4, device=DEV)[:1, ::2])
    refused("is on cpu|CUDA", lk.lutkan_matmul_fp8, x, xs.cpu(), one, ones)
    refused("dtype", lk.lutkan_matmul_fp8, x, xs, one, ones, dtype=torch.float64)
    refused("y must", lk.lutkan_matmul_fp8, x, xs, one, ones, y=torch.empty(4, 21, device=DEV))
    refused("overlap", lk.lutkan_matmul_fp8, x, xs, one, ones, y=torch.empty(1, 20, device=DEV).expand(4, 20))
    sizes = torch.tensor([2, 2], device=DEV)
    refused("one element", lk.lutkan_grouped_matmul_fp8, x, xs, w, ws, sizes[:1])
    refused("rows", lk.lutkan_grouped_matmul_fp8, x, xs, w, ws, sizes, rows=torch.ones(4, device=DEV))
    refused("y must", lk.lutkan_grouped_matmul_fp8, x, xs, w, ws, sizes, rows=sizes, y=torch.empty(4, 20, device=DEV))
    v = torch.zeros(4, 130, device=DEV)
    refused("weight", lk.lutkan_rmsnorm_fp8, v, torch.ones(131, device=DEV))
    refused("residual must", lk.lutkan_rmsnorm_fp8, v, torch.ones(130, device=DEV), residual=v[:3])
    refused("without a residual", lk.lutkan_rmsnorm_fp8, v, torch.ones(130, device=DEV), residual_out=v)
    refused("residual_out must", lk.lutkan_rmsnorm_fp8, v, torch.ones(130, device=DEV), residual=v, residual_out=v.half())
    refused("EUNSUPPORTED|\\[-5\\]", lk.lutkan_rmsnorm_fp8, torch.zeros(1, 40000, device=DEV), torch.ones(40000, device=DEV))


# ---------------------------------------------------------------- the operators together, and their code
@gpu
@pytest.mark.parametrize("tokens", [1, 37, 600])
def test_expert_block(tokens):
    """The block's output from its own codes and routing: the experts' products in 64 bits, the table layer's kernel on them, and the
    weighted sum over a token's experts.  Bound: the products' as above; the layer is Lipschitz between its table's points (its steps
    at the knots are small and rare), and bf16 rounds the output: 2 % of the output's norm covers all of it."""
    from paper_2601_03332_amd.expert_block import ExpertBlock
    rng = np.random.default_rng(tokens)
    width, inner, experts, top = 200, 48, 5, 2
    knots = (-4.0 + (np.arange(15) - 3) * 1.0).astype(np.float32)
    art = lk.lutkan_compile(inner, width, 8, 3, knots, (rng.standard_normal((inner, width, 11)) / 7).astype(np.float32), 32, lk.ASYM_UINT8, lk.CLOSED, lk.CLIP_X)
    layer = art.to_device(DEV)

    def normal(*shape):
        return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DEV)
    norm = 1 + 0.1 * normal(width)
    block = ExpertBlock(norm, normal(experts, width) / width ** 0.5, normal(experts, inner, width) / width ** 0.5, layer, top)
    x, residual = normal(tokens, width).bfloat16(), normal(tokens, width)
    y, res = block(x, residual)
    assert torch.equal(res, x.float() + residual) and y.dtype == torch.bfloat16
    codes, scales, _ = lk.lutkan_rmsnorm_fp8(x, norm, residual=residual)
    p, expert = torch.softmax(lk.lutkan_matmul_fp8(codes, scales, *block.router), 1).topk(top, 1)
    codes, scales, w, ws = codes.cpu(), scales.cpu(), block.experts[0].cpu(), block.experts[1].cpu()
    out = np.zeros((tokens, width))
    for place in range(top):
        z = np.zeros((tokens, inner), np.float32)
        for e in range(experts):
            at = torch.where(expert[:, place].cpu() == e)[0]
            if at.numel():
                z[at.numpy()] = product_reference(codes.view(torch.uint8)[at].view(F8), scales[at], w[e], ws[e])[0]
        out += p[:, place, None].cpu().numpy() * lk.lutkan_forward(layer, torch.from_numpy(z).to(DEV)).cpu().numpy()
    assert np.linalg.norm(y.float().cpu().numpy() - out) <= 0.02 * np.linalg.norm(out)


def test_m0_is_only_touched_by_the_lds_copies_in_the_products_kernels(tmp_path):
    """The copies into LDS write M0 inside inline-asm blocks and declare it clobbered, which is sound while the compiler keeps nothing in
    M0 there: in the generated code every mention of it lies in such a block."""
    import os
    import re
    import subprocess
    from paper_2601_03332_amd import build as lib_build
    out = tmp_path / "matmul.s"
    cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + lib_build.HIPCC_FLAGS + ["-I", os.path.join(lib_build.ROOT, "include"), "-I", lib_build.CSRC, "-x", "hip",
                                                                                      "--cuda-device-only", "-S", os.path.join(lib_build.CSRC, "lutkan_fp8_matmul.hip"), "-o", str(out)]
    subprocess.run(cmd, check=True, capture_output=True)
    kernels, inside_asm, current = 0, False, None
    for line in open(out):
        text = line.strip()
        if re.match(r"_Z\S*fp8_tiled_kernel\S*:", text):
            current, kernels = text.split(":")[0], kernels + 1
        elif text.startswith(".Lfunc_end"):
            current = None
        elif text.startswith(";;#ASM"):
            inside_asm = text.startswith(";;#ASMSTART")
        elif current and not text.startswith(";") and re.search(r"\bm0\b", text.split(";")[0]):
            assert inside_asm, f"compiler-generated use of m0 in {current}: {text}"
    assert kernels >= 16
