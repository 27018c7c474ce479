"""Every kernel of the integer products by the launch rule, ends of ranges, and the generated code of the copies into LDS.

Sums of whole numbers with scales of 1 are exact in fp32 below 2^24: outputs are equal to them, bit for bit."""
import os
import re
import subprocess

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2601_03332_amd as lk  # noqa: E402
from paper_2601_03332_amd import binding  # noqa: E402

DEV = "cuda:0"
gpu = pytest.mark.gpu


def codes(gen, *shape, most=127):
    return torch.randint(-most, most + 1, shape, generator=gen, device=DEV, dtype=torch.int8)


def guarded(t, before, after):
    """t as a part of wider rows whose other bytes are 100."""
    wide = torch.full((*t.shape[:-1], t.shape[-1] + before + after), 100, dtype=t.dtype, device=DEV)
    part = wide[..., before:before + t.shape[-1]]
    part.copy_(t)
    return part


# kernel, rows, k, n, groups (0: one weight), bytes before a row (4: rows at dword addresses, 3: not)
KERNELS = [("int8_direct rows=16 columns=16", 4, 4201, 297, 0, 3), ("int8_direct rows=16 columns=16", 4, 4200, 87, 0, 4),
           ("int8_direct rows=16 columns=16", 4, 4201, 98, 4, 3), ("int8_direct rows=16 columns=16", 11, 4200, 135, 12, 4),
           ("int8_direct rows=16 columns=32", 83, 4049, 1844, 0, 3), ("int8_direct rows=16 columns=32", 255, 4180, 625, 0, 4),
           ("int8_direct rows=16 columns=32", 36, 4177, 2030, 3, 3), ("int8_direct rows=16 columns=32", 42, 4044, 1635, 4, 4),
           ("int8_tiled rows=64 columns=64 teams=2; ", 303, 4185, 2336, 0, 3), ("int8_tiled rows=64 columns=64 teams=2 async", 593, 4196, 1177, 0, 4),
           ("int8_tiled rows=64 columns=64 teams=2; ", 530, 4161, 1360, 5, 3), ("int8_tiled rows=64 columns=64 teams=2 async", 779, 4172, 497, 12, 4),
           ("int8_tiled rows=128 columns=128 teams=1; ", 6404, 105, 2406, 0, 3), ("int8_tiled rows=128 columns=128 teams=1 async", 2666, 4100, 1167, 0, 4),
           ("int8_tiled rows=128 columns=128 teams=1; ", 6739, 65, 3828, 3, 3), ("int8_tiled rows=128 columns=128 teams=1 async", 2850, 3652, 1120, 4, 4),
           ("int8_tiled rows=128 columns=256", 2573, 4036, 2145, 0, 4), ("int8_tiled rows=128 columns=256", 7059, 164, 3785, 12, 4),
           ("int8_tiled rows=256 columns=256", 3680, 2116, 3968, 0, 4), ("int8_tiled rows=256 columns=256", 6405, 2180, 2219, 5, 4)]


@gpu
@pytest.mark.parametrize("case", KERNELS, ids=lambda c: "-".join(str(v) for v in c))
def test_each_kernel(case):
    """Exact sums, operands inside wider buffers, rows gathered, a group without rows and one with a single one, rows behind the last; in all three types."""
    plan, rows, k, n, groups, before = case
    print(f"case kernel {case}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(rows + k)
    most = 127 if k * 127 * 127 < 1 << 24 else int((((1 << 24) - 1) / k) ** 0.5)
    x, w = codes(gen, rows, k, most=most), codes(gen, *([groups] if groups else []), n, k, most=most)
    ones = torch.ones(rows, device=DEV)
    out = torch.full((rows, n + 3), 7.0, device=DEV)
    if not groups:
        ref = (x.double() @ w.double().t().contiguous())
        y = lk.lutkan_matmul_int8(guarded(x, before, 8 - before), ones, guarded(w, before, 8 - before), torch.ones(n, device=DEV), y=out[:, 1:1 + n])
    else:
        index = torch.randint(-1, rows, (rows,), generator=gen, device=DEV)
        rest, sizes = rows, []
        for g in range(groups):                                    # (a single row, none, the others about even, some behind the last)
            sizes.append(1 if g == 0 else 0 if g == 1 and groups > 2 else max(1, int(0.95 * rest / (groups - g))))
            rest -= sizes[-1]
        ref, first = torch.zeros(rows, n, dtype=torch.float64, device=DEV), 0
        for g, size in enumerate(sizes):
            at = index[first:first + size]
            ref[first:first + size] = torch.where(at[:, None] >= 0, x[at.clamp(min=0)].double(), 0.0) @ w[g].double().t().contiguous()
            first += size
        y = lk.lutkan_grouped_matmul_int8(guarded(x, before, 8 - before), ones, guarded(w, before, 8 - before), torch.ones(groups, n, device=DEV),
                                          torch.tensor(sizes, device=DEV), rows=index, y=out[:, 1:1 + n])
    assert plan in lk.lutkan_last_plan(), lk.lutkan_last_plan()
    assert torch.equal(y.double(), ref)
    assert bool((out[:, :1] == 7).all()) and bool((out[:, 1 + n:] == 7).all())
    for dtype in (torch.float16, torch.bfloat16):                  # the same sums, rounded once
        args = (x, ones, w, torch.ones(w.shape[:-1], device=DEV))
        got = lk.lutkan_matmul_int8(*args, dtype=dtype) if not groups else lk.lutkan_grouped_matmul_int8(*args, torch.tensor(sizes, device=DEV), rows=index, dtype=dtype)
        assert torch.equal(got, ref.float().to(dtype))


# tile, rows, k, n, groups: no block of k to a few more than the buffers, and a last one that is not whole
SHORT = [("64 columns=64", 6519, 36, 304, 0), ("64 columns=64", 349, 64, 5329, 0), ("64 columns=64", 8173, 100, 227, 0), ("64 columns=64", 4093, 128, 232, 0),
         ("64 columns=64", 7388, 192, 112, 0), ("64 columns=64", 2507, 200, 670, 0), ("64 columns=64", 1150, 256, 822, 0), ("64 columns=64", 519, 320, 1671, 0),
         ("64 columns=64", 2277, 384, 390, 0), ("64 columns=64", 210, 448, 3313, 0), ("64 columns=64", 971, 512, 899, 0), ("128 columns=128", 7234, 36, 2118, 0),
         ("128 columns=128", 3902, 64, 4183, 0), ("128 columns=128", 4331, 100, 1825, 0), ("128 columns=128", 4701, 128, 1641, 0), ("128 columns=128", 4187, 192, 3872, 0),
         ("128 columns=128", 7546, 200, 2094, 0), ("128 columns=128", 5924, 256, 2594, 0), ("128 columns=128", 3872, 320, 4200, 0), ("128 columns=128", 5462, 384, 2923, 0),
         ("128 columns=128", 7569, 448, 2136, 0), ("128 columns=128", 2017, 512, 1969, 0), ("128 columns=256", 4852, 36, 3982, 5), ("128 columns=256", 4478, 64, 4237, 5),
         ("128 columns=256", 7827, 100, 2493, 5), ("128 columns=256", 3808, 128, 5047, 5), ("128 columns=256", 4569, 192, 4285, 5), ("128 columns=256", 3033, 200, 5767, 5),
         ("128 columns=256", 3205, 256, 5625, 5), ("128 columns=256", 3348, 320, 5791, 5), ("128 columns=256", 3375, 384, 5098, 5), ("128 columns=256", 5330, 448, 3719, 5),
         ("128 columns=256", 3657, 512, 5033, 5), ("256 columns=256", 7264, 128, 1666, 5), ("256 columns=256", 7880, 192, 1711, 5), ("256 columns=256", 7476, 200, 1440, 5),
         ("256 columns=256", 6496, 256, 2043, 5), ("256 columns=256", 5572, 320, 2397, 5), ("256 columns=256", 6413, 384, 1977, 5), ("256 columns=256", 2141, 448, 5506, 5),
         ("256 columns=256", 3807, 512, 3532, 5)]


@gpu
@pytest.mark.parametrize("case", SHORT, ids=lambda c: "-".join(str(v) for v in c))
def test_rows_of_few_blocks_in_each_tiled_kernel(case):
    tile, rows, k, n, groups = case
    print(f"case short {case}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(rows + k)
    x, w = codes(gen, rows, k), codes(gen, *([groups] if groups else []), n, k)
    if not groups:
        y, ref = lk.lutkan_matmul_int8(x, torch.ones(rows, device=DEV), w, torch.ones(n, device=DEV)), x.double() @ w.double().t().contiguous()
    else:
        sizes = [rows // groups] * (groups - 1) + [rows - rows // groups * (groups - 1) - 7]
        y = lk.lutkan_grouped_matmul_int8(x, torch.ones(rows, device=DEV), w, torch.ones(groups, n, device=DEV), torch.tensor(sizes, device=DEV))
        parts = [v.double() @ w[g].double().t().contiguous() for g, v in enumerate(x.split(sizes + [7])[:groups])]
        ref = torch.cat(parts + [torch.zeros(7, n, dtype=torch.float64, device=DEV)])
    assert f"int8_tiled rows={tile}" in lk.lutkan_last_plan(), lk.lutkan_last_plan()
    assert torch.equal(y.double(), ref)


@gpu
@pytest.mark.parametrize("shape", [(40, 300, 70), (1030, 640, 1290), (4100, 260, 2050)], ids=str)
def test_an_output_does_not_depend_on_the_rows_and_columns_around_it(shape):
    """Sums are exact and every kernel rounds in one order: parts of a product are equal to products of the parts, scales of any size among them."""
    rows, k, n = shape
    gen = torch.Generator(device=DEV).manual_seed(k)
    x, w = codes(gen, rows, k), codes(gen, n, k)
    xs, ws = torch.exp(torch.randn(rows, generator=gen, device=DEV)), torch.exp(torch.randn(n, generator=gen, device=DEV))
    xs[3], ws[5], xs[rows - 1] = 1e-30, 1e25, 3e-39
    y = lk.lutkan_matmul_int8(x, xs, w, ws)
    for r, c in ((slice(0, 7), slice(0, 9)), (slice(rows - 33, rows), slice(n // 2, n)), (slice(2, 4), slice(3, n))):
        assert torch.equal(y[r, c], lk.lutkan_matmul_int8(x[r], xs[r], w[c], ws[c]))


@gpu
def test_rows_at_offsets_beyond_32_bits():
    """Operands and outputs whose last rows begin more than 2^32 bytes behind the first."""
    rows, k, n, stride = 600, 256, 40, 8 << 20
    gen = torch.Generator(device=DEV).manual_seed(1)
    wide = torch.empty(rows * stride, dtype=torch.int8, device=DEV)
    x = torch.as_strided(wide, (rows, k), (stride, 1))
    x.copy_(codes(gen, rows, k))
    w = codes(gen, n, k)
    ref = (x.double() @ w.double().t().contiguous()).float()
    ones = torch.ones(rows, device=DEV)
    assert torch.equal(lk.lutkan_matmul_int8(x, ones, w, torch.ones(n, device=DEV)), ref)
    index = torch.arange(rows - 1, -1, -1, device=DEV)
    got = lk.lutkan_grouped_matmul_int8(x, ones, w[None], torch.ones(1, n, device=DEV), torch.tensor([rows], device=DEV), rows=index)
    assert torch.equal(got, ref.flip(0))
    got = lk.lutkan_matmul_int8(codes(gen, 70, k), torch.ones(70, device=DEV), x, ones)       # (as a weight)
    assert got.shape == (70, rows)
    assert torch.equal(lk.lutkan_matmul_int8(w, torch.ones(n, device=DEV), x, ones), ref.t())
    c, s = lk.lutkan_quantise_int8(torch.as_strided(wide.view(torch.float16), (rows, 8), (stride // 2, 1)).zero_())
    assert not bool(c.any()) and bool((s == 2.0 ** -126).all())


@gpu
def test_many_groups():
    groups, k, n = 70001, 32, 16
    gen = torch.Generator(device=DEV).manual_seed(2)
    sizes = torch.randint(-1, 2, (groups,), generator=gen, device=DEV)
    rows = int(sizes.clamp(min=0).sum()) + 5
    x, w = codes(gen, rows, k), codes(gen, groups, n, k)
    y = lk.lutkan_grouped_matmul_int8(x, torch.ones(rows, device=DEV), w, torch.ones(groups, n, device=DEV), sizes)
    of = torch.repeat_interleave(torch.arange(groups, device=DEV), sizes.clamp(min=0))
    ref = (x[:rows - 5].float()[:, None, :] * w[of].float()).sum(2)
    assert torch.equal(y[:rows - 5], ref) and not bool(y[rows - 5:].any())


def test_products_that_no_launch_holds_are_refused():
    import ctypes as C
    lib = lk.load_library()
    a = binding._MatmulFp8Args(4096, 4096, 4096, 4096, 4096, (1 << 31) - 1, 16, 1, 16, 16, 1 << 20, (1 << 31) - 1, 16, 1 << 20, 0, 1, 4096, None, 8, 8)
    assert lib.lutkan_matmul_int8(C.byref(a), None) == -5
    assert "too many outputs" in lk.lutkan_last_error()


# ---------------------------------------------------------------- launches of more rows than one holds
@gpu
def test_rows_and_tokens_of_more_than_one_launch():
    """Launches hold fewer than 2^32 threads: 2^26 - 1 rows of four to a work-group of 256, and as many tokens of a wave each."""
    rows = (1 << 26) + 3
    x = (torch.arange(rows, device=DEV) % 251).half()[:, None] - 125
    codes8, scales = lk.lutkan_quantise_int8(x)
    assert torch.equal(codes8, (torch.sign(x) * 127).to(torch.int8))
    assert torch.equal(scales, (x.float().abs()[:, 0] / torch.full((1,), 127.0, device=DEV)).clamp(min=2.0 ** -126))      # (by a number torch multiplies by its reciprocal)
    del codes8, scales
    out = torch.empty_like(x)
    codes8, scales, out = lk.lutkan_rmsnorm_int8(x, torch.ones(1, device=DEV), residual=x, eps=0.5, residual_out=out)
    assert torch.equal(out, x + x) and torch.equal(codes8, (torch.sign(x) * 127).to(torch.int8))
    del codes8, scales, out
    places = (torch.arange(rows, device=DEV, dtype=torch.int32) % 7)[:, None]
    y = torch.arange(5, device=DEV, dtype=torch.float16)[:, None] + 1
    got = lk.lutkan_expert_combine(y, places)
    assert torch.equal(got[:, 0], torch.where(places[:, 0] < 5, places[:, 0] + 1, 0).half())


# ---------------------------------------------------------------- generated code
@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    from paper_2601_03332_amd import build as lib_build
    out = tmp_path_factory.mktemp("asm") / "matmul.s"
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + lib_build.HIPCC_FLAGS + ["-I", os.path.join(lib_build.ROOT, "include"), "-I", lib_build.CSRC, "-x", "hip",
                                                                                               "--cuda-device-only", "-S", os.path.join(lib_build.CSRC, "lutkan_int8_matmul.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    return out.read_text()


def test_no_kernel_spills_registers(assembly):
    scratch = dict(re.findall(r"\.name: +(_Z\S*lutkan_int8_\S+)\n(?:.*\n)*?.*\.private_segment_fixed_size: +(\d+)", assembly))
    assert len(scratch) >= 20 and set(scratch.values()) == {"0"}, scratch


def test_the_copies_into_lds_alone_touch_m0_and_their_scalars_are_settled(assembly):
    """The copies write M0 inside inline-asm blocks and declare it clobbered: every mention of it lies in such a block.  And the scalar registers of a copy's address,
    which the compiler's own spacing of instructions does not see inside the block, are not written by a vector instruction within the five steps before it."""
    kernels, copies, inside, kernel, before = 0, 0, False, None, []
    for line in assembly.split("\n"):
        text = line.strip()
        if re.match(r"_Z\S*int8_tiled_kernel\S*:", text):
            kernel, kernels, before = text.split(":")[0], kernels + 1, []
            continue
        if text.startswith(".Lfunc_end"):
            kernel = None
        elif text.startswith(";;#ASM"):
            inside = text.startswith(";;#ASMSTART")
        code = text.split(";")[0].strip()
        if not kernel or not code or code.startswith("."):
            continue
        if re.search(r"\bm0\b", code):
            assert inside, f"compiler-generated use of m0 in {kernel}: {text}"
        copy = re.match(r"global_load_lds_dword\S* \S+ s\[(\d+):(\d+)\]", code)
        if copy:
            copies += 1
            low, high, steps = int(copy.group(1)), int(copy.group(2)), 0
            for earlier in reversed(before):
                written = re.match(r"v_(?:readlane|readfirstlane)_b32 s(\d+)", earlier)
                assert steps >= 5 or not (written and low <= int(written.group(1)) <= high), (kernel, earlier, code)
                nop = re.match(r"s_nop (\d+)", earlier)
                steps += 1 + (int(nop.group(1)) if nop else 0)
        before = before[-11:] + [code]
    assert kernels >= 10 and copies >= 100
