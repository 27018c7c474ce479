"""The 8-bit operators at the ends of their ranges."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")
import paper_2601_03332_amd as lk  # noqa: E402
from paper_2601_03332_amd import binding  # noqa: E402
from test_fp8_operators import DEV, F8, gpu  # noqa: E402


# ---------------------------------------------------------------- more than one launch holds (fewer than 2^32 threads)
@gpu
def test_norm_of_more_rows_than_one_launch_holds():
    """A wave a row: 2^26 rows are 2^32 threads.  The rows on both sides of every 2^24 rows as a short call gives them: a launch
    of 2^32 threads and more runs a part of them, without an error."""
    rows, width = (1 << 26) + 4099, 8
    print(f"case norm {rows} x {width}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(rows, width, generator=gen, device=DEV, dtype=torch.bfloat16)
    residual = torch.randn(rows, width, generator=gen, device=DEV, dtype=torch.float16)
    weight = 1 + 0.1 * torch.randn(width, generator=gen, device=DEV)
    codes, scales, out = lk.lutkan_rmsnorm_fp8(x, weight, residual=residual)
    for end in [i << 24 for i in range(1, 5)] + [2100, rows]:
        at = slice(end - 2100, min(end + 2100, rows))
        part = lk.lutkan_rmsnorm_fp8(x[at], weight, residual=residual[at])
        assert torch.equal(codes[at].view(torch.uint8), part[0].view(torch.uint8)) and torch.equal(scales[at], part[1]) and torch.equal(out[at], part[2])


@gpu
def test_weights_of_more_blocks_than_one_launch_holds():
    """A work-group of 256 threads a block: 2^24 blocks are 2^32 threads."""
    matrices = (1 << 24) + 3
    print(f"case weights {matrices} of 1 x 1", flush=True)
    w = torch.randn(matrices, 1, 1, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV, dtype=torch.bfloat16)
    codes, scales = lk.lutkan_quantise_fp8(w)
    expected = (w.float().abs() / torch.full((1,), 448.0, device=DEV)).clamp(min=2.0 ** -126)
    assert bool(((scales - expected).abs() <= 2.0 ** -22 * expected).all())
    assert torch.equal(codes.view(torch.uint8), torch.where(w < 0, 0xfe, 0x7e).to(torch.uint8).masked_fill_(w == 0, 0))


@gpu
def test_product_of_more_rows_than_one_launch_of_small_tiles_holds():
    """2^23 work-groups of 512 threads are 2^32: such calls take larger tiles.  The rows are overlapping windows, four codes apart, of one line
    of codes 1, -1 and 0, whose sums are whole numbers and have no rounding."""
    rows, k = (1 << 29) + 77, 256
    print(f"case product {rows} x {k} -> 1", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(3)
    codes = torch.tensor([0x00, 0x38, 0xb8], dtype=torch.uint8, device=DEV)
    line = codes[torch.randint(0, 3, (1 << 16,), generator=gen, device=DEV)].repeat((4 * rows + k) // (1 << 16) + 1)
    w = codes[torch.randint(0, 3, (1, k), generator=gen, device=DEV)].view(F8)
    one = torch.ones(1, 2, device=DEV)
    x = line.as_strided((rows, k), (4, 1)).view(F8)
    y = lk.lutkan_matmul_fp8(x, one.expand(rows, 2), w, one)
    short = lk.lutkan_matmul_fp8(x[:(1 << 14) + 100], one.expand((1 << 14) + 100, 2), w, one)
    assert int(short.abs().max()) > 0
    assert torch.equal(short[:100], short[1 << 14:])               # (the line repeats itself)
    assert torch.equal(y, short[:1 << 14].repeat(rows // (1 << 14) + 1, 1)[:rows])


def test_products_that_no_launch_holds_are_refused():
    lib = lk.load_library()
    rows = (1 << 31) - 1
    a = binding._MatmulFp8Args(4096, 4096, 4096, 4096, 4096, rows, 1, 1, 1, 1, 1, rows, 1, 1, 0, 1, 4096, None, 8, 8)
    assert lib.lutkan_matmul_fp8(C.byref(a), None) == -5, lk.lutkan_last_error()
    rows, groups, n = 1 << 24, 1 << 17, 1 << 14
    a = binding._MatmulFp8Args(4096, 4096, 4096, 4096, 4096, rows, 16, 1, 16, 16 * n, n, rows, 16, n, 2, groups, 4096, None, 8, 8)
    assert lib.lutkan_grouped_matmul_fp8(C.byref(a), None) == -5, lk.lutkan_last_error()


# ---------------------------------------------------------------- lengths beyond 32 bits
@gpu
def test_the_binding_refuses_lengths_beyond_32_bits():
    """The library's widths, inputs, outputs and groups are 32-bit numbers: a longer tensor is refused, not cut to its low bits."""
    def refused(f, *args, **kwargs):
        with pytest.raises(lk.LutKanError, match="2147483647"):
            f(*args, **kwargs)
    much = (1 << 32) + 1                                           # cut to 32 bits: 1
    w = torch.zeros(1, 1, dtype=torch.bfloat16, device=DEV)
    refused(lk.lutkan_quantise_fp8, w.expand(much, 1))
    refused(lk.lutkan_quantise_fp8, w[None].expand(2, much, 1))
    one, scale = torch.zeros(1, 1, dtype=torch.uint8, device=DEV).view(F8), torch.ones(1, 1, device=DEV)
    refused(lk.lutkan_matmul_fp8, one, scale, one.expand(much, 1), torch.ones(-(-much // 128), 1, device=DEV))
    refused(lk.lutkan_grouped_matmul_fp8, one, scale, one[None].expand(1, much, 1), torch.ones(1, -(-much // 128), 1, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV))
    wide = torch.empty((1 << 32) + 128, dtype=torch.bfloat16, device=DEV)
    refused(lk.lutkan_rmsnorm_fp8, wide[None], wide)


@gpu
@pytest.mark.parametrize("shape", [(1, (1 << 31) - 1), ((1 << 31) - 1, 1)], ids=str)
def test_weights_of_the_longest_rows_and_columns(shape):
    """2^31 - 1 inputs or outputs: places near the end pass 2^31 when eight columns, or a block, are added.  Nothing behind the codes and
    scales is written."""
    n, k = shape
    print(f"case weights {shape}", flush=True)
    count, last = n * k, (n * k - 1) // 128 * 128
    w = torch.ones(count, dtype=torch.bfloat16, device=DEV)
    w[-1] = -2.0
    codes = torch.full((count + 64,), 0x55, dtype=torch.uint8, device=DEV)
    scales = torch.full((last // 128 + 2,), 7.0, device=DEV)
    lib = lk.load_library()
    assert lib.lutkan_quantise_fp8(w.data_ptr(), 2, 1, n, k, k, count, codes.data_ptr(), scales.data_ptr(), None) == 0
    torch.cuda.synchronize()
    assert bool((codes[:last] == 0x7e).all()) and bool((codes[last:count - 1] == 0x76).all()) and int(codes[count - 1]) == 0xfe      # 448; 224, -448
    assert bool((codes[count:] == 0x55).all())
    assert bool((scales[:-2] - 1 / 448).abs().max() <= 2.0 ** -31) and abs(float(scales[-2]) * 448 - 2) <= 2.0 ** -20 and float(scales[-1]) == 7.0


def test_more_groups_than_the_search_counts_are_refused():
    """The search for a tile's group steps through the sizes in 32 bits: near 2^31 groups the step passes them and does not end.  Long before
    that a work-group's walk takes longer than its products."""
    for groups in ((1 << 20) + 1, (1 << 31) - 1):
        a = binding._MatmulFp8Args(4096, 4096, 4096, 4096, 4096, 1, 16, 1, 16, 0, 1, 1, 16, 1, 2, groups, 4096, None, 4, 8)
        assert lk.load_library().lutkan_grouped_matmul_fp8(C.byref(a), None) == -5, lk.lutkan_last_error()
        assert "groups" in lk.lutkan_last_error()


@gpu
def test_the_most_groups():
    """2^20 groups of one row, none or two, all with the same weight: the product with one weight, bit for bit (whole numbers)."""
    groups, k, n = 1 << 20, 16, 4
    gen = torch.Generator(device=DEV).manual_seed(4)
    sizes = torch.zeros(groups, dtype=torch.int32, device=DEV)
    sizes[torch.randint(0, groups, (40,), generator=gen, device=DEV)] = 1
    sizes[groups - 1] = 2
    rows = int(sizes.sum()) + 1                                    # and one behind the last group
    print(f"case groups {groups}, rows {rows}", flush=True)
    codes = torch.tensor([0x00, 0x38, 0xb8], dtype=torch.uint8, device=DEV)
    x, w = (codes[torch.randint(0, 3, shape, generator=gen, device=DEV)] for shape in ((rows, k), (n, k)))
    one = torch.ones(1, 1, device=DEV)
    y = lk.lutkan_grouped_matmul_fp8(x.view(F8), one.expand(rows, 1), w.view(F8).expand(groups, n, k), torch.ones(groups, 1, 1, device=DEV), sizes)
    expected = lk.lutkan_matmul_fp8(x.view(F8), one.expand(rows, 1), w.view(F8), one)
    expected[rows - 1] = 0
    assert torch.equal(y, expected)


# ---------------------------------------------------------------- rows whose squares are beyond the type
@gpu
@pytest.mark.parametrize("rows", [8, 1100, 2100])
@pytest.mark.parametrize("width", [7, 300, 1024, 2048, 5001, 32768])
def test_norm_of_rows_whose_squares_are_beyond_the_type(rows, width):
    """A row of values above 1.8e19, or without eps one below 1e-19, has a norm like any other, to what sums in fp32 give: 64 * 2^-24.  The rows around
    it, one with an infinity and one of zeros are what they are without it."""
    print(f"case huge and tiny rows {rows} {width}", flush=True)
    if rows * width > 12_000_000:
        rows = 1026 if width < 20000 else 40
    depth = 64 * 2.0 ** -24
    gen = torch.Generator(device=DEV).manual_seed(width)
    x = torch.randn(rows, width, generator=gen, device=DEV)
    x = torch.where(x.abs() < 2.0 ** -6, torch.full_like(x, 0.5), x)
    one = torch.ones(width, device=DEV)
    for eps in (0.0, 1e-6):
        plain = lk.lutkan_rmsnorm_fp8(x, one, eps=eps)
        given = x.clone()
        for row, factor in enumerate((1e19, 1e20, 1e30, 3.0e38 / float(x[3].abs().max()), 1e-18, 1e-24, 1e-36)):
            given[row] = x[row] * factor
        given[7, width - 1] = float("inf")
        codes, scales, _ = lk.lutkan_rmsnorm_fp8(given, one, eps=eps)
        h = given[:7].double()
        y = h / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
        blocks = -(-width // 128)
        exact = torch.nn.functional.pad(y.abs(), (0, blocks * 128 - width)).view(7, blocks, 128).amax(2) / 448
        assert bool(((scales[:7].double() - exact).abs() <= depth * exact).all()), eps
        got, v = codes[:7].float().double(), y / exact.repeat_interleave(128, 1)[:, :width]
        step = torch.exp2(torch.floor(torch.log2((v.abs() * (1 + 2 * depth)).clamp(2.0 ** -6))).clamp(max=8) - 3)
        assert bool(((got - v).abs() <= 0.5 * step + 2 * depth * v.abs()).all()), eps
        value = codes[7].float() * scales[7].repeat_interleave(128)[:width]
        edge = (width - 1) // 128 * 128
        assert bool(torch.isnan(value[edge:]).all()) and bool((value[:edge] == 0).all())
        assert torch.equal(codes[8:].view(torch.uint8), plain[0][8:].view(torch.uint8)) and torch.equal(scales[8:], plain[1][8:])


# ---------------------------------------------------------------- large products that cancel
@gpu
@pytest.mark.parametrize("shape", [(5, 384, 40), (3000, 384, 2048)], ids=str)
def test_large_products_that_cancel(shape):
    """448 * 448 and its negative side by side, and products of at most 1 among them.  Outputs of 32 bits: a sum of a block is off by at most
    2^-23 of its largest partial sum, 448^2, per addition (128, and 3 blocks): 131 * 2^-23 * 448^2 = 3.2.  Those of 16 bits keep 13 bits below the
    leading bit of 448^2: seven products in a group of eight, 16 groups, 3 blocks, 2^17 * 2^-13 each, and the output's rounding."""
    rows, k, n = shape
    print(f"case cancel {shape}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(k)
    codes = torch.tensor([0x00, 0x30, 0x38, 0xb0, 0xb8], dtype=torch.uint8, device=DEV)        # 0, 1/2, 1, -1/2, -1
    x, w = (codes[torch.randint(0, 5, (count, k), generator=gen, device=DEV)] for count in (rows, n))
    large = torch.randperm(k // 2, generator=gen, device=DEV)[:k // 16] * 2
    x[:, large], x[:, large + 1], w[:, large], w[:, large + 1] = 0x7e, 0xfe, 0x7e, 0x7e        # 448, -448; 448, 448
    value = torch.zeros(256, dtype=torch.float64, device=DEV)
    value[[0x30, 0x38, 0xb0, 0xb8]] = torch.tensor([0.5, 1, -0.5, -1], dtype=torch.float64, device=DEV)
    ref = value[x.long()] @ value[w.long()].t().contiguous()       # (the large ones add to 0 exactly)
    xs, ws = torch.ones(rows, k // 128, device=DEV), torch.ones(-(-n // 128), k // 128, device=DEV)
    for dtype, bound in ((torch.float32, 3.2), (torch.float16, 7 * 16 * 3 * 16.0), (torch.bfloat16, 7 * 16 * 3 * 16.0)):
        y = lk.lutkan_matmul_fp8(x.view(F8), xs, w.view(F8), ws, dtype=dtype)
        off = float((y.double() - ref).abs().max())
        print(f"{dtype}: {off} of values to {float(ref.abs().max())}", flush=True)
        assert off <= bound


# ---------------------------------------------------------------- the block
def test_the_block_refuses_a_router_that_does_not_fit_its_experts():
    """A router of more rows than there are experts would pick experts that do not exist."""
    from types import SimpleNamespace
    from paper_2601_03332_amd.expert_block import ExpertBlock
    layer, norm = SimpleNamespace(d=6, m=10), torch.ones(10)
    for shape in ((5, 10), (3, 10), (4, 9), (40,)):
        with pytest.raises(lk.LutKanError, match="router is"):
            ExpertBlock(norm, torch.zeros(shape), torch.zeros(4, 6, 10), layer)
    with pytest.raises(lk.LutKanError, match="experts are"):
        ExpertBlock(norm, torch.zeros(4, 10), torch.zeros(6, 10), layer)


# ---------------------------------------------------------------- scales whose product is out of range
@gpu
@pytest.mark.parametrize("case", [(False, 1, 300, 40, 0), (True, 1, 300, 40, 0), (False, 33, 301, 50, 3), (True, 70, 300, 260, 0), (False, 2449, 617, 194, 0), (True, 2502, 1028, 293, 0),
                                  (False, 3489, 264, 3001, 0), (False, 2846, 3108, 835, 5), (True, 3642, 1345, 531, 0), (True, 3979, 236, 870, 5)], ids=str)
def test_scales_whose_product_is_beyond_the_type(case):
    """scale(x) * scale(w) beyond 2^128 with both finite: a block whose sum is zero adds nothing, one whose sum is small adds what it comes to;
    infinite scales and NaN codes stay what they are."""
    wide, rows, k, n, groups = case
    print(f"case scales {case}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(k)
    blocks, lead = -(-k // 128), [groups] if groups else []
    ones = torch.tensor([0x38, 0xb8], dtype=torch.uint8, device=DEV)

    def signs(*shape):
        return ones[torch.randint(0, 2, shape, generator=gen, device=DEV)]
    x, w = signs(rows, k), signs(*lead, n, k)
    xs, ws = torch.ones(rows, blocks, device=DEV), torch.ones(*lead, -(-n // 128), blocks, device=DEV)
    ws[..., 0] = 2.0 ** 60
    every = torch.arange(rows, device=DEV)
    xs[every % 3 == 0, 0] = 2.0 ** 100                             # times 2^60: beyond the type.  Codes of zero in every other of these rows,
    x[every % 3 == 0, :128] = 0
    x[every % 6 == 3, 5] = 0x01                                    # 2^-9, the smallest code, in the others, whose scale is 2^70: 2^121
    xs[every % 6 == 3, 0] = 2.0 ** 70
    sizes = [rows // 2, rows - rows // 2] + [0] * (groups - 2) if groups else [rows]
    xd, wd = (torch.where((c & 0x80) != 0, -1.0, 1.0).double() * torch.where((c & 0x7f) == 1, 2.0 ** -9, torch.where((c & 0x7f) == 0, 0.0, 1.0)).double() for c in (x, w))
    ref, first = torch.zeros(rows, n, dtype=torch.float64, device=DEV), 0
    for e, size in enumerate(sizes):
        at = slice(first, first + size)
        ws_e, wd_e = (ws[e], wd[e]) if groups else (ws, wd)
        sw = ws_e.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
        ref[at] = (xd[at] * xs[at].double().repeat_interleave(128, 1)[:, :k]) @ (wd_e * sw).t().contiguous()
        first += size
    for dtype in [torch.float32] if wide else [torch.bfloat16]:
        def call():
            if groups:
                return lk.lutkan_grouped_matmul_fp8(x.view(F8), xs, w.view(F8), ws, torch.tensor(sizes, device=DEV), dtype=dtype)
            return lk.lutkan_matmul_fp8(x.view(F8), xs, w.view(F8), ws, dtype=dtype)
        y = call()
        assert bool(torch.isfinite(y).all())
        # rows of zeros in the first block: whole numbers below 2^13, exact before the output's rounding; the others: 2^121 times what fp32 rounds
        zero = every % 6 == 0
        assert torch.equal(y[zero], ref[zero].float().to(dtype))
        other = every % 6 == 3
        assert bool(((y[other].double() - ref[other]).abs() <= (2.0 ** -22 if wide else 2.0 ** -7) * ref[other].abs()).all())
        rest = every % 3 != 0                                      # first block 2^60 times a whole number: the rest is below its last bit
        assert bool(((y[rest].double() - ref[rest]).abs() <= (2.0 ** -22 if wide else 2.0 ** -7) * ref[rest].abs() + 2.0 ** 14).all())
        kept = xs[0, 0].item()
        xs[0, 0] = float("inf")
        got = call()
        assert not bool(torch.isfinite(got[0]).any()) and torch.equal(got[1:], y[1:])
        xs[0, 0] = kept
        x[0, k - 1] = 0x7f
        got = call()
        assert bool(torch.isnan(got[0]).all()) and torch.equal(got[1:], y[1:])
        x[0, k - 1] = 0x38


# ---------------------------------------------------------------- the copies into LDS
def test_every_copy_into_lds_preserves_m0_where_that_is_switched_on(tmp_path):
    """kLdsDmaPreservesM0 is for a compiler that keeps values in M0: with it, every copy in the products' kernels saves M0 and puts it back."""
    import os
    import re
    import shutil
    import subprocess
    from paper_2601_03332_amd import build as lib_build
    for name in os.listdir(lib_build.CSRC):
        if name.endswith(".h") or name == "lutkan_fp8_matmul.hip":
            shutil.copy(os.path.join(lib_build.CSRC, name), tmp_path / name)
    header = (tmp_path / "lutkan_device.h").read_text()
    assert header.count("kLdsDmaPreservesM0 = false") == 1
    (tmp_path / "lutkan_device.h").write_text(header.replace("kLdsDmaPreservesM0 = false", "kLdsDmaPreservesM0 = true"))
    out = tmp_path / "matmul.s"
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + lib_build.HIPCC_FLAGS +
                   ["-I", os.path.join(lib_build.ROOT, "include"), "-I", str(tmp_path), "-x", "hip", "--cuda-device-only", "-S", str(tmp_path / "lutkan_fp8_matmul.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    copies = {"global_load_lds_dword": 0, "global_load_lds_dwordx4": 0}
    block = []
    for line in open(out):
        text = line.strip()
        if text.startswith(";;#ASMSTART"):
            block = []
        elif text.startswith(";;#ASMEND"):
            for load in (t.split()[0] for t in block if t.startswith("global_load_lds")):
                copies[load] += 1
                saved = re.fullmatch(r"s_mov_b32 (s\d+), m0", block[0])
                assert saved and block[-1] == f"s_mov_b32 m0, {saved.group(1)}", block
        else:
            block.append(text.split(";")[0].strip())
    assert min(copies.values()) > 0


def test_registers_spill_only_in_the_kernels_that_are_priced_for_it(tmp_path):
    """The tiled kernels into 32 bits that copy through registers hold more than fits, but for 64 x 64 with two teams; no other kernel of the
    products has scratch memory."""
    import os
    import re
    import subprocess
    from paper_2601_03332_amd import build as lib_build
    out = tmp_path / "matmul.s"
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + lib_build.HIPCC_FLAGS +
                   ["-I", os.path.join(lib_build.ROOT, "include"), "-I", lib_build.CSRC, "-x", "hip", "--cuda-device-only", "-S", os.path.join(lib_build.CSRC, "lutkan_fp8_matmul.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    scratch = dict(re.findall(r"\.name: +(_Z\S*lutkan_fp8_\S+)\n(?:.*\n)*?.*\.private_segment_fixed_size: +(\d+)", out.read_text()))
    assert len(scratch) >= 40
    for kernel, size in scratch.items():
        shape = re.search(r"tiled_kernelI(?:Li\d+E){4}Li(\d)ELb1ELb[01]ELb0E", kernel)       # (teams; 32 bits; grouped or not; through registers)
        small = "tiled_kernelILi2ELi2E" in kernel
        if shape and not (small and shape.group(1) == "2"):
            assert int(size) <= 128, (kernel, size)
        else:
            assert int(size) == 0, (kernel, size)
