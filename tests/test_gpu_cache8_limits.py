"""The paged 8-bit cache at the ends of its range, on the GPU against the fp64 oracle: scales of values from 2^-100 to 2^119, pages of
zeros, which are stored with the smallest scale.  Tolerances are those of test_gpu_cache8.py, which derives them: relative to the
weighted sum of magnitudes, so that neither the size of the values nor the order of the pages enters."""
import numpy as np
import pytest
import test_gpu_cache8 as base

from oracle import cache8 as o

pytestmark = pytest.mark.gpu

# (heads per kv head, new tokens): few columns, and many (16-bit queries)
FEW, MANY = (2, 1), (4, 40)


def _pages(rng, dtype, columns, exps, hd=64, codes_of=None):
    """One sequence whose page i of values has the scale 2^exps[i]; codes_of(i) gives its codes, None: random ones."""
    rep, new = columns
    case = base._attend_case(rng, dtype, 1, rep, hd, [64 * len(exps) - new], [new], sharp=0.1)
    cu, table, lengths, codes, scales, q = case
    for i, e in enumerate(exps):
        page = table[0, i]
        scales[page, 0, 1] = 2.0**e
        c = codes_of(i) if codes_of else None
        if c is not None:
            codes[page, 0, 1] = c
    return case


def _compare(case, dtype, hd=64, **kw):
    cu, table, lengths, codes, scales, q = case
    got = base._np(base._attend(case, dtype, 0.1, **kw))
    base._check_attention(got, o.attend(codes, scales, q, cu, table, lengths, 0.1, **kw), dtype, hd, int(lengths[0]), q)


@pytest.mark.parametrize("dtype,columns", [("fp32", FEW), ("bf16", FEW), ("bf16", MANY)])
@pytest.mark.parametrize("exp", [-100, -92, -80, -41])
@pytest.mark.parametrize("pages", [1, 9])
def test_values_that_are_all_small(gpu_device, dtype, columns, exp, pages):
    """The weights of the first page keep their bits, whatever its scale."""
    _compare(_pages(np.random.default_rng(70 + pages), dtype, columns, [exp] * pages), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("seqs,rep,new,full,zeros,behind", [(16, 2, 1, 8, 16, 12), (16, 2, 1, 24, 12, 0), (16, 2, 1, 0, 30, 6),
                                                            (1, 8, 256, 72, 3, 0), (1, 8, 256, 72, 12, 0), (1, 8, 256, 66, 12, 8)])
def test_pages_of_zeros_behind_values_of_one_sign(gpu_device, dtype, seqs, rep, new, full, zeros, behind):
    """Pages of 448s, pages of zeros with the smallest scale, and pages of 448s again, enough of them that one wavefront meets all
    three kinds: few columns of 32 kv heads and 16 sequences, and a chunk with an item for every workgroup (16-bit queries)."""
    rng, heads, hd, pages = np.random.default_rng(71), 32, 64, full + zeros + behind
    case = base._attend_case(rng, dtype, heads, rep, hd, [64 * pages - new] * seqs, [new] * seqs, sharp=0.1)
    cu, table, lengths, codes, scales, q = case
    for i in range(pages):
        at = table[:, i]
        zero = full <= i < full + zeros
        codes[at, :, 1], scales[at, :, 1] = (0, 2.0**-100) if zero else (0x7E, 1.0)
    base._attend_heads(case, dtype, 0.1, 0, 0, heads, rep, hd, (0, heads - 1) if new == 1 else (heads - 1,))


@pytest.mark.parametrize("dtype,columns", [("fp32", FEW), ("bf16", FEW), ("bf16", MANY)])
@pytest.mark.parametrize("exps", [[60 - i for i in range(150)], [-90 + i for i in range(150)], [0, -100, 80, -100] * 12, [80] + [-100] * 30,
                                  [-60, 0, 60, 0] * 3, [75] * 2 + [-100] * 8])
def test_scales_that_fall_and_rise(gpu_device, dtype, columns, exps):
    case = _pages(np.random.default_rng(72), dtype, columns, exps, codes_of=lambda i: 0x70 + i % 9)
    _compare(case, dtype)


@pytest.mark.parametrize("dtype,columns", [("fp32", (2, 3)), ("bf16", (2, 3)), ("bf16", (4, 80)), ("bf16", (4, 200))])
@pytest.mark.parametrize("large,small", [(30, -20), (-20, 30), (0, -45), (-90, -40), (32, -32), (-32, 32)])
def test_rows_whose_windows_see_other_scales(gpu_device, dtype, columns, large, small):
    """Neighbouring rows share a block of columns: one sees a page of a scale that another's window hides, or that lies behind it."""
    exps = [large] + [small] * 3 + [large]
    case = _pages(np.random.default_rng(73), dtype, columns, exps)
    for window in (1, 3, 64, 65, 130):
        _compare(case, dtype, window=window)


@pytest.mark.parametrize("dtype,columns", [("fp32", FEW), ("bf16", FEW), ("fp32", MANY), ("bf16", MANY), ("bf16", (4, 300))])
@pytest.mark.parametrize("exps,code", [([112], 0x7E), ([112] * 40, 0x7E), ([119] * 12, 0x7E), ([120] * 7, 0x70), ([119, -100, 60] * 9, 0x7E)])
def test_values_near_the_end_of_fp32(gpu_device, dtype, columns, exps, code):
    """Means of values as large as fp32 holds, of rows that one workgroup takes and of rows that several join."""
    case = _pages(np.random.default_rng(74), dtype, columns, exps + [0] * (5 if columns[1] > 64 else 0), codes_of=lambda i: code if i < len(exps) else None)
    _compare(case, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("hd,rot,layout", [(64, 32, o.HALVES), (128, 128, o.ADJACENT), (256, 64, o.ADJACENT), (256, 256, o.HALVES)])
@pytest.mark.parametrize("amplitude", [1.2, 0.3, 1.0, 2.0**-40, 2.0**45])
def test_keys_come_back_from_tables_of_any_amplitude(gpu_device, dtype, hd, rot, layout, amplitude):
    """Appended and read with the same tables, as contexts that are stretched have them: the keys, but for their codes' rounding."""
    torch, b, rng = base._t(), base._b(), np.random.default_rng(hd + rot)
    heads, n = 2, 150
    cu, table, lengths, n_pages = base._step(rng, [0], [n])
    codes, scales = base._random_pool(rng, n_pages, heads, hd)
    k, v = (base._rounded(rng.standard_normal((n, heads, hd)), dtype) for _ in range(2))
    t = base._type(dtype)
    cos, sin = b.rope_tables(base._dev(np.arange(1000, 1000 + n)), rot, base=500000.0, factor=8.0, orig_len=8192.0, amplitude=amplitude)
    cache = b.Cache8(base._dev(codes), base._dev(scales.astype(np.float32)))
    args = base._i32(table), base._i32(lengths)
    cache.append(base._dev(k, t), base._dev(v, t), base._i32(cu), *args, cos=cos, sin=sin, layout=layout)
    gk, gv = (base._np(x) for x in cache.read(n, base._i32(cu), base._i32([0]), *args, dtype=t, cos=cos, sin=sin, layout=layout))
    pages, sc = cache.pages.cpu().numpy(), base._np(cache.scales)
    wk, wv = o.read(pages, sc, n, cu, [0], table, lengths, base._np(cos), base._np(sin), layout)
    # the rotation: two roundings; cos^2 + sin^2: two, of which one of the smaller square; its reciprocal and the product: two, or
    # none where it is 1 but for 2^-22, the tables' own rounding.  Each is 2^-24 of a channel, which is at most its pair's length.
    size = o.read(pages, sc, n, cu, [0], table, lengths)[0]
    err = (8 if amplitude != 1.0 else 6) * 2.0**-24 * 2.0**0.5 * np.abs(size).max(axis=2, keepdims=True) / amplitude
    assert np.all(np.abs(gk - wk) <= err + base._half(dtype, np.abs(wk) + err))
    assert np.all(np.abs(gv - wv) <= base._half(dtype, wv))
    # against the keys themselves: half a step of each code, and a pair turned back mixes its two errors
    x = o.rotate(k, base._np(cos), base._np(sin), layout)
    half = np.maximum(2.0**-4 * np.abs(x), 2.0**-10 * sc[table[0, np.arange(n) // 64], :, 0, None])
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if layout == o.ADJACENT else (slice(0, rot // 2), slice(rot // 2, rot))
    pair = np.hypot(half[..., first], half[..., second]) / amplitude * 1.001
    for part in (first, second):
        off = np.abs(gk[..., part] - k[..., part])
        assert np.all(off <= pair + err + base._half(dtype, np.abs(k[..., part]) + pair))


@pytest.mark.parametrize("heads,rep,hd", [(32, 8, 64), (4, 4, 128)])
def test_one_workspace_serves_a_chunk_and_the_steps_behind_it(gpu_device, heads, rep, hd):
    """The workspace of the largest step, for that step (whole items, where there are 32 heads) and for smaller ones down to one row."""
    torch, b, rng = base._t(), base._b(), np.random.default_rng(75)
    cu, table, lengths, codes, scales, q = base._attend_case(rng, "bf16", heads, rep, hd, [100], [260])
    cache = b.Cache8(base._dev(codes), base._dev(scales.astype(np.float32)))
    dq = base._dev(q, base._type("bf16"))
    ws = torch.empty(cache.workspace_bytes(dq, 1), dtype=torch.uint8, device="cuda")
    assert all(cache.workspace_bytes(dq[:n], 1) <= ws.numel() for n in range(1, 261))
    for n in (260, 1, 40, 8, 9, 128):
        args = base._i32([0, n]), base._i32(table), base._i32([100 + n])
        got = cache.attend(dq[:n], *args, scale=0.1, workspace=ws)
        pick = slice(rep, 2 * rep)
        want = o.attend(codes[:, 1:2], scales[:, 1:2], q[:n, pick], [0, n], table, [100 + n], 0.1)
        base._check_attention(base._np(got)[:, pick], want, "bf16", hd, 100 + n, q)


def test_windows_beyond_32_bits_are_refused(gpu_device):
    """The entry point takes 32 bits: a larger number must not become another one (2^32 would be no window at all)."""
    b = base._b()
    case = base._attend_case(np.random.default_rng(76), "bf16", 1, 2, 64, [100], [1])
    for kw in (dict(window=2**32), dict(window=2**31), dict(window=2**40 + 5), dict(window=5, sinks=2**32 + 4)):
        with pytest.raises(ValueError):
            base._attend(case, "bf16", 0.1, **kw)
    for kw in (dict(window=-1), dict(window=5, sinks=-1)):
        with pytest.raises(b.RvqError):
            base._attend(case, "bf16", 0.1, **kw)
