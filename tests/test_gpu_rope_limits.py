"""Rotation of numbers at the ends of their types, on the GPU against the formula (a c - b s, a s + b c) in 64 bits."""
import numpy as np
import pytest
import test_gpu_cache8 as base

from oracle import cache8 as o

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout", [o.ADJACENT, o.HALVES])
@pytest.mark.parametrize("hd,rot", [(64, 64), (80, 20), (128, 32)])
def test_infinities_turn_as_the_formula_says(gpu_device, dtype, layout, hd, rot):
    """An infinity in the first, the second or both channels of a pair; NaN; neighbours stay what they are."""
    b, rng = base._b(), np.random.default_rng(hd)
    x = base._rounded(rng.standard_normal((8, 2, hd)), dtype)
    first, second = (0, 1) if layout == o.ADJACENT else (0, rot // 2)
    inf = np.inf
    pairs = [(inf, 1.0), (1.0, inf), (-inf, 1.0), (1.0, -inf), (inf, inf), (inf, -inf), (np.nan, 1.0), (1.0, np.nan)]
    for n, (p, q) in enumerate(pairs):
        x[n, 0, first], x[n, 0, second] = p, q
    cos, sin = base._tables(rng.integers(1, 5000, 8), rot)
    assert (np.abs(cos[:, 0]) > 1e-4).all() and (np.abs(sin[:, 0]) > 1e-4).all()
    c64, s64 = cos.astype(np.float64), sin.astype(np.float64)
    with np.errstate(invalid="ignore"):
        want = o.rotate(x, c64, s64, layout)
    got = base._np(b.rope(base._dev(x, base._type(dtype)), base._dev(cos), base._dev(sin), layout=layout))
    fin = np.isfinite(want)
    assert np.isinf(want).sum() >= 8 and np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    x0 = np.where(np.isfinite(x), x, 0.0)
    bound = base._rot_error(x0, c64, s64, layout)
    assert np.all(np.abs(got[fin] - want[fin]) <= (bound + base._half(dtype, np.where(fin, want, 0.0) + bound))[fin])


@pytest.mark.parametrize("layout", [o.ADJACENT, o.HALVES])
def test_products_beyond_fp32_are_infinities(gpu_device, layout):
    """The largest numbers under tables of an amplitude above 1: what passes fp32 is an infinity of the right sign."""
    b, big = base._b(), 3.0e38
    x = np.ones((4, 1, 64))
    first, second = (0, 1) if layout == o.ADJACENT else (0, 32)
    for n, (p, q) in enumerate([(0.0, big), (0.0, -big), (big, 0.0), (-big, 0.0)]):
        x[n, 0, first], x[n, 0, second] = p, q
    cos, sin = (3.0 * t for t in base._tables(np.full(4, 1), 64))
    got = base._np(b.rope(base._dev(x).float(), base._dev(cos.astype(np.float32)), base._dev(sin.astype(np.float32)), layout=layout))
    with np.errstate(over="ignore"):
        want = o.rotate(x, cos.astype(np.float64), sin.astype(np.float64), layout).astype(np.float32).astype(np.float64)
    assert np.array_equal(got[:, 0, [first, second]], want[:, 0, [first, second]]) and np.isinf(want).sum() == 8
