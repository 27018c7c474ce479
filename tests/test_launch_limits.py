"""A launch holds fewer than 2^32 threads, and one of more runs a part of them without an error: the layers' calls with so many rows that a
kernel would need more are refused."""
import ctypes as C

import numpy as np
import pytest

import paper_2601_03332_amd as lk
from paper_2601_03332_amd import CLIP_X, CLOSED, SYM_INT8, binding

DEV = "cuda:0"


def compiled(d, m, **options):
    knots = (-1.0 + (np.arange(11) - 3) * 0.5).astype(np.float32)
    coef = np.random.default_rng(d).standard_normal((d, m, 7)).astype(np.float32)
    return lk.lutkan_compile(d, m, 4, 3, knots, coef, 16, SYM_INT8, CLOSED, CLIP_X, **options)


@pytest.mark.parametrize("algo", [lk.ALGO_AUTO, lk.ALGO_TILED, lk.ALGO_GATHER])
@pytest.mark.parametrize("m", [4, 64, 300])
def test_forward_calls_of_too_many_rows_are_refused(m, algo):
    lib, art = lk.load_library(), compiled(40, m)
    dl, bl = binding._DevLayer(), binding._SplineDevLayer()
    assert lib.lutkan_dev_layer_init(art._h, C.byref(dl)) == 0 and lib.bspline_dev_layer_init(art._h, C.byref(bl)) == 0
    dl.table, dl.algo, bl.coef_table, bl.algo = 4096, algo, 4096, algo
    for B in (1 << 34, 1 << 36):
        assert lib.lutkan_forward(C.byref(dl), 4096, B, 1 << 60, None, 1 << 20, 1 << 58, None) == -5, lk.lutkan_last_error()
        assert lib.bspline_kan_forward(C.byref(bl), 4096, B, 1 << 60, 1 << 20, 1 << 58, None) == -5, lk.lutkan_last_error()


def test_chains_and_statistics_of_too_many_rows_are_refused():
    lib, art = lk.load_library(), compiled(2, 1)
    dl = binding._DevLayer()
    assert lib.lutkan_dev_layer_init(art._h, C.byref(dl)) == 0
    dl.table = 4096
    for B in (1 << 26, 1 << 30):                                   # a wave a row
        assert lib.lutkan_chain_forward((binding._DevLayer * 1)(dl), 1, 4096, B, 1 << 40, None, None, None) == -5, lk.lutkan_last_error()
    B = 1 << 30                                                    # 64 rows to a work-group of 256 threads
    assert lib.lutkan_error_stats(4096, 4096, B, 1, 4096, 1, -1.0, 1.0, None, 0, 4096, 4096, 1 << 40, None) == -5, lk.lutkan_last_error()


@pytest.mark.gpu
def test_a_chain_just_below_and_at_the_limit():
    torch = pytest.importorskip("torch")
    layer = compiled(2, 1).to_device(DEV)
    line = torch.linspace(-1.2, 1.2, 2 << 12, device=DEV).view(-1, 2)
    expected = lk.lutkan_chain_forward([layer], line)
    rows = 1 << 26
    x = line.repeat(rows // line.shape[0], 1)
    print(f"case chain {rows} rows", flush=True)
    with pytest.raises(lk.LutKanError, match="too large"):
        lk.lutkan_chain_forward([layer], x)
    y = lk.lutkan_chain_forward([layer], x[:rows - 4])             # 2^32 - 256 threads
    assert torch.equal(y, expected.repeat(rows // line.shape[0], 1)[:rows - 4])
