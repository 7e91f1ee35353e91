"""The fp64 reference of the microscaled formats and of the 8-bit GQA cache, pinned by hand-worked values and by the formats' definitions."""
import numpy as np
import pytest

from oracle import mx
from oracle.fp8 import e4m3_decode, e4m3_encode


def test_grids_are_the_formats():
    assert mx.E4M3[-1] == 448 and mx.E4M3[1] == 2.0 ** -9 and len(mx.E4M3) == 127
    assert np.array_equal(mx.E4M3, e4m3_decode(np.arange(127)))


def test_rounding_agrees_with_the_codes():
    x = np.random.default_rng(0).normal(size=4000) * np.exp2(np.random.default_rng(1).integers(-12, 8, 4000))
    x = np.clip(x, -448, 448)
    assert np.array_equal(mx.nearest(x, mx.E4M3), e4m3_decode(e4m3_encode(x)))
    assert mx.nearest([17, 19, 232, 248, 2.0 ** -10, 3 * 2.0 ** -10], mx.E4M3).tolist() == [16, 20, 224, 256, 0, 2.0 ** -8]
    assert mx.nearest([.25, .75, 1.25, 1.75, 2.5, 3.5, 5, -5.01], mx.E2M1).tolist() == [0, 1, 1, 2, 2, 4, 4, -6]


@pytest.mark.parametrize("grid, top", [(mx.E4M3, 448.0), (mx.E2M1, 6.0)])
def test_scale_is_the_smallest_that_holds(grid, top):
    assert mx.scale_byte([0, top, np.nextafter(top, 1e9), top / 2, 1e-40, top * 2.0 ** -126], grid).tolist() == [1, 127, 128, 126, 1, 1]
    a = np.abs(np.random.default_rng(2).normal(size=1000)) * np.exp2(np.random.default_rng(3).integers(-100, 100, 1000))
    b = mx.scale_byte(a, grid)
    assert (a <= top * np.exp2(b - 127.0)).all() and (a > top * np.exp2(b - 128.0)).all()


def test_cache_values():
    c = mx.Cache8(1, 2)
    c.write(0, [[[1.0, 448.0]]])                      # scale 1
    assert c.b[0, 0] == 127 and c.rows[0, 0].tolist() == [1.0, 448.0]
    c.write(1, [[[460.0, 17.0]]])                     # scale 2: 230 to 224 (steps of 16); 17 / 2 = 8.5 to the even code, 8
    assert c.b[0, 0] == 128 and c.rows[:, 0].tolist() == [[1.0, 448.0], [448.0, 16.0]]
    c.write(2, [[[2.0 ** -9, 3 * 2.0 ** -10]]])       # half of the smallest code, 2 2^-9: to 0; three quarters of it: to that code
    assert c.rows[2, 0].tolist() == [0.0, 2.0 ** -8]
    c.write(16 * 0, [[[1.0, 2.0]]])                   # from the block's first row on: anew, the rows behind are gone
    assert len(c.rows) == 1 and c.b[0, 0] == 127 - 7


def test_cache_of_one_block_is_one_quantisation():
    rows = np.random.default_rng(4).normal(size=(16, 3, 8))
    c = mx.Cache8(3, 8)
    c.write(0, rows)
    flat, b = mx.quantise(rows.transpose(1, 0, 2).reshape(3, -1), mx.E4M3, 128)
    assert np.array_equal(c.rows, flat.reshape(3, 16, 8).transpose(1, 0, 2)) and np.array_equal(c.b[0], b[:, 0])


def test_bf16_rounding():
    x = np.random.default_rng(5).normal(size=1000).astype(np.float32)
    bits = x.view(np.uint32).astype(np.uint64)
    want = (((bits + 0x7FFF + ((bits >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)
    assert np.array_equal(mx.to_bf16(x), want.astype(np.float64))
