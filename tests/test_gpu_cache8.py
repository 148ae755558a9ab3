"""Rotary tables, rotation and the paged 8-bit cache on the GPU against the fp64 oracle (oracle/cache8.py), through the binding.

Tolerances, all derived beforehand.
  tables     the angle in quarter turns is a 64-bit product: error <= |p| 2^-51 of a turn's angle; its remainder is rounded to
             fp32 (<= 2^-26 quarter turns), sine and cosine are good to 2 units of 2^-24, the amplitude rounds once.
  rotation   three fp32 roundings of products and a sum: 3 * 2^-24 (|a c| + |b s|), then half a step of the type.
  codes      a code's value is within half a step of the number; the number is known to the rotation's error.
  read       the rotation's error and half a step of the type.
  attention  a score is off by E = scale sum |q| |k| times (2^-21 for two-term queries, 2^-22 of the row's largest element for the
             16-bit ones, and fp32 products and sums: head_dim + 8 roundings at most), a weight by the factor e^E, by 2^-11
             where it is rounded to fp16 (2^-21 with fp32 queries) and 2^-22 from exp2; sums over N tokens add (N / 32 + 48) 2^-23.
             All of it acts on sum w |v|; then half a step of the type."""
import numpy as np
import pytest

from oracle import cache8 as o

pytestmark = pytest.mark.gpu

EPS = {"fp32": 2.0**-24, "bf16": 2.0**-8, "fp16": 2.0**-11}  # half a step, relative


def _t():
    import torch
    return torch


def _b():
    from paper_2410_15704_amd import binding
    return binding


def _type(name):
    torch = _t()
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def _dev(a, dtype=None):
    torch = _t()
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _i32(a):
    return _dev(np.asarray(a, dtype=np.int32))


def _np(t):
    return t.detach().double().cpu().numpy()


def _rounded(a, name):
    """The numbers that inputs of that type hold."""
    return _np(_dev(np.asarray(a, dtype=np.float64)).to(_type(name)))


def _half(name, y):
    """Half a step of the type at y."""
    tiny = {"fp32": 2.0**-149, "bf16": 2.0**-133, "fp16": 2.0**-24}[name]
    return EPS[name] * np.abs(y) * (1 + 2.0**-7) + tiny


def _rot_error(x, cos, sin, layout):
    """3 * 2^-24 (|a c| + |b s|) in every rotated channel."""
    return 3 * 2.0**-24 * o.rotate(np.abs(x), np.abs(cos), np.abs(sin) * -1, layout).clip(0) + 3 * 2.0**-24 * (
        np.abs(o.rotate(np.abs(x), np.abs(cos), np.abs(sin), layout)) + np.abs(x))


def _random_pool(rng, n_pages, heads, hd, spread=2):
    """Any finite codes and power-of-two scales: what other sequences left."""
    codes = rng.integers(0, 254, (n_pages, heads, 2, 64 * hd)).astype(np.uint8)
    codes[(codes & 127) == 127] = 5
    return codes, 2.0 ** rng.integers(-9 - spread, -9 + spread + 1, (n_pages, heads, 2))


def _step(rng, olds, news, extra=1):
    """cu, table, lengths and page count of sequences that hold `olds` tokens and bring `news`."""
    lengths = [a + n for a, n in zip(olds, news)]
    counts = [-(-x // 64) for x in lengths]
    n_pages = sum(counts) + 2
    order = rng.permutation(n_pages)
    table = np.full((len(news), max(counts + [1]) + extra), -1, dtype=np.int32)
    at = 0
    for i, c in enumerate(counts):
        table[i, :c] = order[at : at + c]
        at += c
    return np.concatenate([[0], np.cumsum(news)]).astype(np.int32), table, np.array(lengths, dtype=np.int32), n_pages


# ---- tables and rotation -----------------------------------------------------------------------
@pytest.mark.parametrize("rot", [2, 6, 64, 128, 250, 1026])
@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0, factor=8.0, orig_len=8192.0, alpha=1.0, beta=4.0, amplitude=1.2),
                                dict(factor=4.0), dict(base=1e6, factor=0.5, orig_len=100.0, alpha=-1.0, beta=0.5)])
def test_tables(gpu_device, rot, kw):
    b, rng = _b(), np.random.default_rng(rot)
    for pos in ([0], [1, 2, 3, 131071, 1 << 20, 2**31 - 1, -5], rng.integers(0, 1 << 20, 777)):
        cos, sin = b.rope_tables(_dev(np.asarray(pos, dtype=np.int64)), rot, **kw)
        wc, ws = o.tables(pos, rot, **kw)
        bound = kw.get("amplitude", 1.0) * (np.abs(np.asarray(pos, dtype=np.float64))[:, None] * 2.0**-50 + 1.6 * 2.0**-26 + 4 * 2.0**-24)
        assert np.all(np.abs(_np(cos) - wc) <= bound) and np.all(np.abs(_np(sin) - ws) <= bound)


def _tables(positions, rot):
    cos, sin = o.tables(positions, rot)
    return cos.astype(np.float32), sin.astype(np.float32)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout", [o.ADJACENT, o.HALVES])
@pytest.mark.parametrize("N,heads,hd,rot", [(1, 1, 64, 64), (5, 3, 128, 64), (300, 8, 128, 128), (2, 2, 1024, 16), (7, 40, 256, 256),
                                            (3, 2, 80, 20), (4, 5, 66, 66), (2, 3, 2, 2), (3, 1, 1040, 32)])
def test_rope(gpu_device, dtype, layout, N, heads, hd, rot):
    torch, b, rng = _t(), _b(), np.random.default_rng(N * hd + rot)
    x = _rounded(rng.standard_normal((N, heads, hd)), dtype)
    cos, sin = _tables(rng.integers(0, 100000, N), rot)
    want = o.rotate(x, cos.astype(np.float64), sin.astype(np.float64), layout)
    bound = _rot_error(x, cos.astype(np.float64), sin.astype(np.float64), layout)
    bound = bound + _half(dtype, np.abs(want) + bound)
    dx, dc, ds = _dev(x, _type(dtype)), _dev(cos), _dev(sin)
    fused = torch.randn(N, heads + 3, hd, device="cuda").to(_type(dtype))
    fused[:, 1 : 1 + heads] = dx
    odd = torch.zeros(N * heads * (hd + 3) + 1, device="cuda", dtype=_type(dtype))[1:].view(N, heads, hd + 3)[..., :hd]
    odd.copy_(dx)
    swapped = dx.transpose(0, 1).contiguous().transpose(0, 1)
    kept = fused.clone()
    first = None
    for name, src, out in (("whole", dx, None), ("fused", fused[:, 1 : 1 + heads], None), ("odd strides", odd, None), ("heads first", swapped, None),
                           ("into heads first", dx, torch.empty_like(swapped)), ("in place", dx.clone(), "x"),
                           ("in place, fused", fused[:, 1 : 1 + heads], "x")):
        y = b.rope(src, dc, ds, layout=layout, out=src if out == "x" else out)
        got = _np(y)
        assert np.all(np.abs(got - want) <= bound), name
        assert np.array_equal(got[..., rot:], x[..., rot:]), name
        first = got if first is None else first
        assert np.array_equal(got, first), name  # the same roundings whatever the strides
    assert torch.equal(fused[:, 0], kept[:, 0]) and torch.equal(fused[:, 1 + heads :], kept[:, 1 + heads :])


def test_rotation_turns_keys_as_the_decode_of_codes_does(gpu_device):
    """rvq_rope in the adjacent layout is the rotation of rvq_decode_rope: rotated queries and keys meet."""
    torch, b = _t(), _b()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    q = b.Quantizer(d=128, dhat=32, depth=4, K=64, out_dtype=b.F32)
    q.set_codebooks(torch.randn(4, 64, 32, device="cuda", generator=gen))
    codes = torch.randint(0, 64, (50, 4, 4), device="cuda", generator=gen).short()
    std = torch.rand(50, device="cuda", generator=gen).half() + 0.5
    cos, sin = b.rope_tables(torch.arange(1000, 1050, device="cuda"), 128)
    want = q.decode_rope(codes, std, cos, sin, 128)
    got = b.rope(q.decode(codes, std).view(50, 1, 128), cos, sin).view(50, 128)
    plain = q.decode(codes, std).abs().amax()
    assert float((got - want).abs().amax()) <= 8 * 2.0**-24 * 2 * float(plain)
    q.close()


# ---- append ------------------------------------------------------------------------------------
APPENDS = [  # tokens that sequences hold, and bring
    ([0], [1]), ([63], [1]), ([64], [1]), ([5], [59]), ([5], [60]), ([0], [64]), ([0], [65]), ([130], [200]),
    ([0, 10, 63, 64, 100], [3, 0, 2, 70, 1]), ([7] * 70, [1] * 70), ([3, 9], [0, 0]), (list(range(130)), [2] * 130),
]


def _append_case(rng, dtype, heads, hd, rot, layout, olds, news, big=1.0, extra_rows=0):
    cu, table, lengths, n_pages = _step(rng, olds, news)
    rows = int(cu[-1]) + extra_rows
    codes, scales = _random_pool(rng, n_pages, heads, hd)
    k = _rounded(big * rng.standard_normal((rows, heads, hd)) * np.exp(rng.standard_normal((heads, hd))), dtype)
    v = _rounded(rng.standard_normal((rows, heads, hd)), dtype)
    cos, sin = _tables(rng.integers(0, 5000, rows), rot) if rot else (None, None)
    return cu, table, lengths, codes, scales, k, v, cos, sin


def _check_append(got_codes, got_scales, want, before, case):
    """Scales and untouched codes equal; a new code's value as near to the exact number as half a step and the rotation's error allow."""
    codes, scales, exact = want
    cu, table, lengths, _, _, k, v, cos, sin = case
    hd = k.shape[2]
    assert np.array_equal(got_scales, scales)
    touched = np.zeros(codes.shape, dtype=bool)
    for (page, h, kind, slot), x in exact.items():
        shape = (64, hd) if kind == 0 else (hd, 64)
        at = (slot, slice(None)) if kind == 0 else (slice(None), slot)
        touched[page, h, kind].reshape(shape)[at] = True
        s = scales[page, h, kind]
        val = o.VALUES[got_codes[page, h, kind].reshape(shape)[at]] * s
        fin = np.isfinite(x)
        assert np.isnan(val[~fin]).all()
        e = np.floor(np.log2(np.maximum(np.abs(x[fin]) / s, 2.0**-6)))
        half = 2.0 ** (e - 4) * s
        # rotation: |a c| + |b s| <= sqrt(2) times the pair's length <= 2 times the largest number of the vector
        err = (0 if kind or cos is None else 3 * 2.0**-24 * 2 * np.abs(x[fin]).max(initial=0.0) * 1.5)
        assert np.all(np.abs(val[fin] - x[fin]) <= half * (1 + 2.0**-20) + 2 * err), (page, h, kind, slot)
    same = (got_codes == codes) | ((got_codes & 127) == 0) & ((codes & 127) == 0)
    assert same[~touched].all()
    assert same.mean() > 0.999


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads,hd,rot,layout", [(2, 64, 64, o.ADJACENT), (1, 128, 128, o.HALVES), (3, 128, 32, o.HALVES), (1, 256, 128, o.ADJACENT),
                                                 (2, 128, 0, o.ADJACENT), (2, 256, 256, o.HALVES), (1, 64, 16, o.HALVES)])
def test_append(gpu_device, dtype, heads, hd, rot, layout):
    torch, b = _t(), _b()
    for n, (olds, news) in enumerate(APPENDS):
        if len(olds) > 8 and (dtype != "bf16" or hd != 128):
            continue
        rng = np.random.default_rng(100 * n + hd + rot)
        case = _append_case(rng, dtype, heads, hd, rot, layout, olds, news, big=30.0 if n % 2 else 1.0, extra_rows=2)
        cu, table, lengths, codes, scales, k, v, cos, sin = case
        want = o.append(codes, scales, k, v, cu, table, lengths, None if cos is None else cos.astype(np.float64),
                        None if sin is None else sin.astype(np.float64), layout)
        k[int(cu[-1]) :], v[int(cu[-1]) :] = np.nan, np.inf  # padding rows: not looked at
        cache = b.Cache8(_dev(codes), _dev(scales.astype(np.float32)))
        fused = torch.zeros(k.shape[0], 2 * heads + 1, hd, device="cuda", dtype=_type(dtype))  # strided rows
        fused[:, 1::2], fused[:, 2::2] = _dev(k, _type(dtype)), _dev(v, _type(dtype))
        args = (_i32(cu), _i32(table), _i32(lengths))
        kw = dict(cos=None if cos is None else _dev(cos), sin=None if sin is None else _dev(sin), layout=layout)
        cache.append(fused[:, 1::2], fused[:, 2::2], *args, **kw)
        got = cache.pages.cpu().numpy(), _np(cache.scales)
        _check_append(*got, want, codes, case)
        cache.append(fused[:, 1::2], fused[:, 2::2], *args, **kw)  # again: the same codes and scales
        assert np.array_equal(cache.pages.cpu().numpy(), got[0]) and np.array_equal(_np(cache.scales), got[1])


def test_append_keeps_what_is_not_finite_apart(gpu_device):
    b, rng = _b(), np.random.default_rng(8)
    case = _append_case(rng, "fp32", 2, 64, 0, o.ADJACENT, [60, 0, 0], [10, 1, 70])
    cu, table, lengths, codes, scales, k, v, _, _ = case
    k[0, 0, 3], k[4, 1, 9], v[2, 0, 0], v[10] = np.nan, np.inf, -np.inf, np.nan  # row 10: nothing finite at all
    k[11, 0] = 0.0
    k[12, 1, 5], v[13, 0, 6] = 3e38, 1e-42
    want = o.append(codes, scales, k, v, cu, table, lengths)
    cache = b.Cache8(_dev(codes), _dev(scales.astype(np.float32)))
    cache.append(_dev(k.astype(np.float32)), _dev(v.astype(np.float32)), _i32(cu), _i32(table), _i32(lengths))
    _check_append(cache.pages.cpu().numpy(), _np(cache.scales), want, codes, case)


def test_append_of_growing_tokens_rounds_earlier_codes_again(gpu_device):
    """65 single steps into two pages, every token twice as large as the one before now and then."""
    b, rng = _b(), np.random.default_rng(9)
    hd, heads = 128, 2
    table = np.array([[1, 2]], dtype=np.int32)
    codes, scales = _random_pool(rng, 3, heads, hd)
    cache = b.Cache8(_dev(codes), _dev(scales.astype(np.float32)))
    for n in range(1, 66):
        k = _rounded(2.0 ** (n // 9) * rng.standard_normal((1, heads, hd)), "bf16")
        v = _rounded(2.0 ** (n % 5) * rng.standard_normal((1, heads, hd)), "bf16")
        lengths = np.array([n], dtype=np.int32)
        codes, scales, _ = o.append(codes, scales, k, v, [0, 1], table, lengths)
        cache.append(_dev(k, _type("bf16")), _dev(v, _type("bf16")), _i32([0, 1]), _i32(table), _i32(lengths))
    assert np.array_equal(_np(cache.scales), scales)
    got = cache.pages.cpu().numpy()
    assert ((got == codes) | ((got & 127) == 0) & ((codes & 127) == 0)).all()  # no rotation: bit for bit


def test_pages_that_are_not_there_are_not_written(gpu_device):
    b, rng = _b(), np.random.default_rng(10)
    cu, table, lengths, n_pages = _step(rng, [0, 100, 0, 0], [130, 30, 5, 3])
    table[0, 1], table[1, 1] = n_pages, -7  # beyond the pool, negative
    lengths[2] = 64 * table.shape[1] + 3    # tokens behind the table's end
    lengths[3] = -2                         # tokens before the sequence's beginning
    codes, scales = _random_pool(rng, n_pages, 2, 64)
    k, v = (_rounded(rng.standard_normal((168, 2, 64)), "fp16") for _ in range(2))
    want = o.append(codes, scales, k, v, cu, table, lengths)
    cache = b.Cache8(_dev(codes), _dev(scales.astype(np.float32)))
    cache.append(_dev(k, _type("fp16")), _dev(v, _type("fp16")), _i32(cu), _i32(table), _i32(lengths))
    got = cache.pages.cpu().numpy()
    assert np.array_equal(_np(cache.scales), want[1]) and ((got == want[0]) | ((got & 127) == 0) & ((want[0] & 127) == 0)).all()


# ---- read --------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads,hd,rot,layout", [(2, 64, 32, o.HALVES), (3, 128, 128, o.ADJACENT), (1, 256, 256, o.HALVES), (2, 128, 0, o.ADJACENT)])
def test_read(gpu_device, dtype, heads, hd, rot, layout):
    torch, b, rng = _t(), _b(), np.random.default_rng(hd + rot)
    olds, news = [0, 100, 5, 64, 1], [200, 1, 0, 64, 130]
    _, table, lengths, n_pages = _step(rng, olds, news)
    table[0, 2] = n_pages + 3  # a page that is not there reads as 0
    first = np.array([3, 90, 0, 64, -2], dtype=np.int32)  # from before the beginning, and past the end
    cu = np.array([0, 190, 205, 205, 230, 380], dtype=np.int32)
    rows = 383  # three rows behind the last sequence
    codes, scales = _random_pool(rng, n_pages, heads, hd)
    cos, sin = _tables(rng.integers(0, 5000, rows), rot) if rot else (None, None)
    kw64 = (None, None) if cos is None else (cos.astype(np.float64), sin.astype(np.float64))
    wk, wv = o.read(codes, scales, rows, cu, first, table, lengths, *kw64, layout)
    cache = b.Cache8(_dev(codes), _dev(scales.astype(np.float32)))
    out = tuple(torch.full((rows, heads, 2 * hd), 7.0, device="cuda", dtype=_type(dtype))[..., :hd] for _ in range(2))
    kw = dict(cos=None if cos is None else _dev(cos), sin=None if sin is None else _dev(sin), layout=layout)
    args = (_i32(cu), _i32(first), _i32(table), _i32(lengths))
    k, v = cache.read(rows, *args, out=out, **kw)
    gk, gv = _np(k), _np(v)
    assert (gk[380:] == 7.0).all() and (gv[380:] == 7.0).all()
    assert np.all(np.abs(gv - wv)[:380] <= _half(dtype, wv)[:380])
    size = o.read(codes, scales, rows, cu, first, table, lengths)[0]
    err = 3 * 2.0**-24 * 2 * np.abs(size).max(axis=2, keepdims=True) if rot else 0.0
    assert np.all(np.abs(gk - wk)[:380] <= (err + _half(dtype, np.abs(wk) + err))[:380])
    k2, _ = cache.read(rows, *args, dtype=_type(dtype), **kw)
    assert torch.equal(k2[:380], k[:380])


# ---- attention ---------------------------------------------------------------------------------
def _attend_case(rng, dtype, heads, rep, hd, olds, news, extra_rows=0, sharp=1.0):
    cu, table, lengths, n_pages = _step(rng, olds, news)
    codes, scales = _random_pool(rng, n_pages, heads, hd)
    rows = int(cu[-1]) + extra_rows
    q = _rounded(sharp * rng.standard_normal((rows, heads * rep, hd)), dtype)
    return cu, table, lengths, codes, scales, q


def _check_attention(got, want, dtype, hd, tokens, q):
    out, ssize, vsize = want
    dot = (hd + 8) * 2.0**-24
    e = ssize * ((2.0**-21 if dtype == "fp32" else 0.0) + dot + 2.0**-24 * 4)
    # elements below 2^-22 of a row's largest are rounded: at most 2^-25 of it, against |k| <= sum |k|
    e = e + (0.0 if dtype == "fp32" else 2.0**-25 * ssize * hd)
    rel = 2 * np.expm1(e) + 2 * ((2.0**-21 if dtype == "fp32" else 2.0**-11) + 2.0**-22) + (tokens / 32 + 48) * 2.0**-23
    bound = rel[..., None] * vsize + 2.0**-24 * np.fmax.reduce(vsize, axis=2, keepdims=True)  # of the channels that are numbers
    bound = bound + _half(dtype, np.abs(out) + bound)
    fin = np.isfinite(out)
    assert np.array_equal(fin, np.isfinite(got))
    assert np.array_equal(np.isnan(out), np.isnan(got))
    bad = ~(np.abs(got - out) <= bound) & fin
    assert not bad.any(), (int(bad.sum()), float(np.abs(got - out)[fin].max()), np.argwhere(bad)[:4])


def _attend(case, dtype, scale, window=0, sinks=0, **kw):
    b = _b()
    cu, table, lengths, codes, scales, q = case
    cache = b.Cache8(_dev(codes), _dev(scales.astype(np.float32)))
    return cache.attend(_dev(q, _type(dtype)), _i32(cu), _i32(table), _i32(lengths), scale=scale, window=window, sinks=sinks, **kw)


ATTENDS = [  # tokens held, tokens brought, window, sinks
    ([0], [1], 0, 0), ([62], [1], 0, 0), ([63], [1], 0, 0), ([64], [1], 0, 0), ([700], [1], 0, 0), ([700], [1], 100, 0), ([700], [1], 1, 0),
    ([700], [1], 64, 70), ([700], [1], 5000, 4), ([0, 5, 500, 64, 127, 300], [1, 1, 1, 1, 1, 1], 0, 0),
    ([0, 5, 500, 64], [1, 0, 3, 2], 33, 2), ([40], [90], 0, 0), ([0], [130], 0, 0), ([100, 0, 7], [65, 17, 0], 50, 3), ([130], [64], 10, 130),
    ([200] * 66, [1] * 66, 70, 1),
]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads,rep,hd", [(1, 1, 64), (2, 4, 128), (2, 3, 64), (1, 8, 256), (1, 20, 128), (3, 5, 128)])
def test_attention(gpu_device, dtype, heads, rep, hd):
    torch = _t()
    for n, (olds, news, window, sinks) in enumerate(ATTENDS):
        if len(olds) > 8 and (heads, rep) != (2, 4):
            continue
        rng = np.random.default_rng(1000 * n + heads * rep + hd)
        case = _attend_case(rng, dtype, heads, rep, hd, olds, news, extra_rows=2)
        cu, table, lengths, codes, scales, q = case
        out = torch.full((q.shape[0], heads * rep + 2, hd), 5.0, device="cuda", dtype=_type(dtype))[:, 1:-1]
        scale = 0.6 * hd**-0.5
        _attend(case, dtype, scale, window, sinks, out=out)
        want = o.attend(codes, scales, q, cu, table, lengths, scale, window, sinks)
        got, used = _np(out), int(cu[-1])
        assert (got[used:] == 5.0).all()
        _check_attention(got[:used], [x[:used] for x in want], dtype, hd, max(lengths), q)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_attention_over_long_caches(gpu_device, dtype):
    """Split over workgroups and joined; ragged, so that runs begin and end inside sequences."""
    rng = np.random.default_rng(11)
    for olds, news, heads, rep in (([20000], [1], 1, 4), ([9000, 3, 0, 15000, 700], [1, 1, 1, 2, 1], 2, 2), ([12000], [40], 1, 2)):
        case = _attend_case(rng, dtype, heads, rep, 64, olds, news)
        cu, table, lengths, codes, scales, q = case
        got = _np(_attend(case, dtype, 0.08))
        _check_attention(got, o.attend(codes, scales, q, cu, table, lengths, 0.08), dtype, 64, max(lengths), q)


def _attend_heads(case, dtype, scale, window, sinks, heads, rep, hd, picked):
    """All heads on the GPU, some kv heads in the oracle."""
    cu, table, lengths, codes, scales, q = case
    got = _np(_attend(case, dtype, scale, window, sinks))
    for h in picked:
        part = slice(h * rep, (h + 1) * rep)
        want = o.attend(codes[:, h : h + 1], scales[:, h : h + 1], q[:, part], cu, table, lengths, scale, window, sinks)
        _check_attention(got[:, part], want, dtype, hd, int(lengths.max()), q)


@pytest.mark.parametrize("dtype,window,sinks", [("bf16", 0, 0), ("fp16", 200, 5)])
def test_attention_of_long_chunks(gpu_device, dtype, window, sinks):
    """More blocks of columns and heads than the chip takes at once; several sequences, one that brings nothing."""
    rng = np.random.default_rng(18)
    case = _attend_case(rng, dtype, 16, 8, 64, [100, 7, 0, 300], [700, 0, 301, 150])
    _attend_heads(case, dtype, 0.07, window, sinks, 16, 8, 64, (0, 15))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attention_of_many_short_chunks(gpu_device, dtype):
    """More than 256 sequences and blocks of columns, with gaps."""
    rng = np.random.default_rng(19)
    news = [int(n) for n in rng.integers(0, 20, 300)]
    case = _attend_case(rng, dtype, 2, 8, 64, [int(n) for n in rng.integers(0, 90, 300)], news)
    _attend_heads(case, dtype, 0.07, 0, 0, 2, 8, 64, (1,))


@pytest.mark.parametrize("heads,hd,olds,news", [
    (2, 128, [5], [300]), (2, 256, [0], [130]), (2, 64, [4000], [70]), (1, 256, [2500, 0, 60], [40, 0, 9]), (2, 128, [0, 3000], [500, 20])])
def test_attention_of_a_few_chunks(gpu_device, heads, hd, olds, news):
    """Fewer blocks of columns than workgroups: each a workgroup's own where all are short, shared where one is long."""
    rng = np.random.default_rng(hd + len(news))
    case = _attend_case(rng, "bf16", heads, 8, hd, olds, news)
    _attend_heads(case, "bf16", 0.07, 0, 0, heads, 8, hd, (heads - 1,))


def test_attention_of_more_than_a_thousand_chunks(gpu_device):
    rng = np.random.default_rng(20)
    news = [int(n) for n in rng.integers(0, 14, 1100)]
    case = _attend_case(rng, "bf16", 1, 8, 64, [int(n) for n in rng.integers(0, 70, 1100)], news)
    _attend_heads(case, "bf16", 0.07, 0, 0, 1, 8, 64, (0,))


@pytest.mark.parametrize("dtype", ["fp32", "fp16"])
def test_sharp_and_flat_softmax(gpu_device, dtype):
    rng = np.random.default_rng(12)
    for sharp, scale in ((30.0, 0.5), (1.0, 0.0), (1e-3, 1.0), (1.0, -0.3), (1000.0 if dtype == "fp16" else 1e20, 1e-3 if dtype == "fp16" else 1e-21)):
        case = _attend_case(rng, dtype, 1, 4, 128, [900], [1], sharp=sharp)
        cu, table, lengths, codes, scales, q = case
        got = _np(_attend(case, dtype, scale))
        _check_attention(got, o.attend(codes, scales, q, cu, table, lengths, scale), dtype, 128, 901, q)


def test_values_of_very_different_pages(gpu_device):
    """Scales of values far apart, a page of zeros with the smallest scale, and keys' scales far apart."""
    rng = np.random.default_rng(13)
    case = _attend_case(rng, "fp32", 1, 2, 64, [400], [1], sharp=0.1)
    cu, table, lengths, codes, scales, q = case
    for i, e in enumerate((-9, -30, 3, -100, 20, -9, 11)):
        scales[table[0, i], 0, 1] = 2.0**e
    codes[table[0, 3], 0, 1] = 0
    scales[table[0, 4], 0, 0] = 2.0**-60
    got = _np(_attend(case, "fp32", 0.1))
    _check_attention(got, o.attend(codes, scales, q, cu, table, lengths, 0.1), "fp32", 64, 401, q)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_chunks_over_values_of_very_different_pages(gpu_device, dtype):
    """The same for many columns: pages of zeros that hold most of the weight, scales that jump up and down, in whole and in part."""
    rng = np.random.default_rng(23)
    for exps in ((-9, -100, -9, -100, -100, -8), (-100, -9, -30, 3, -9, -10), (-9, -11, -9, -13, -20, -60)):
        case = _attend_case(rng, dtype, 1, 4, 64, [340], [40], sharp=0.1)
        cu, table, lengths, codes, scales, q = case
        for i, e in enumerate(exps):
            scales[table[0, i], 0, 1] = 2.0**e
            if e == -100:
                codes[table[0, i], 0, 1] = 0
        got = _np(_attend(case, dtype, 0.1))
        # contributions of pages 2^-40 below another page's scale may be dropped: of 2^-40 of that page's values
        _check_attention(got, o.attend(codes, scales, q, cu, table, lengths, 0.1), dtype, 64, 380, q)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-30, 3.0])
def test_chunks_with_softmax_scales_of_any_size_and_sign(gpu_device, dtype, scale):
    rng = np.random.default_rng(24)
    case = _attend_case(rng, dtype, 1, 4, 64, [100], [50], sharp=0.3)
    cu, table, lengths, codes, scales, q = case
    scales[:, :, 0] *= 2.0**-20 if scale == 0.0 else 1.0
    got = _np(_attend(case, dtype, scale, 70, 3))
    _check_attention(got, o.attend(codes, scales, q, cu, table, lengths, scale, 70, 3), dtype, 64, 150, q)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("olds,news,window,sinks", [([100], [1], 0, 0), ([100], [1], 20, 3), ([70], [30], 0, 0), ([150], [50], 30, 2), ([0], [200], 64, 0)])
def test_what_is_hidden_does_not_reach_the_result(gpu_device, dtype, olds, news, window, sinks):
    """NaN codes in every slot behind the end, and in some tokens: only queries that see such a token are NaN there."""
    rng = np.random.default_rng(14)
    heads, rep, hd = 2, 4, 128
    case = _attend_case(rng, dtype, heads, rep, hd, olds, news)
    cu, table, lengths, codes, scales, q = case
    length = int(lengths[0])
    last = table[0, (length - 1) // 64]
    codes[last, :, 0].reshape(heads, 64, hd)[:, (length - 1) % 64 + 1 :] = 127
    codes[last, :, 1].reshape(heads, hd, 64)[:, :, (length - 1) % 64 + 1 :] = 255
    free = [p for p in range(codes.shape[0]) if p not in table[0]]
    codes[free], scales[free] = 127, np.nan
    rows_before = []
    for t in (length - 2, length // 2, 5):  # a token's value in one channel of head 0, another's key in head 1
        page = table[0, t // 64]
        codes[page, 0, 1].reshape(hd, 64)[t % 17, t % 64] = 127
        rows_before.append(t)
    page = table[0, (length - 3) // 64]
    codes[page, 1, 0].reshape(64, hd)[(length - 3) % 64, 9] = 255
    want = o.attend(codes, scales, q, cu, table, lengths, 0.05, window, sinks)
    assert np.isnan(want[0]).any() and np.isfinite(want[0]).any()
    got = _np(_attend(case, dtype, 0.05, window, sinks))
    _check_attention(got, want, dtype, hd, length, q)


def test_rows_that_see_nothing_are_zero_and_missing_pages_are_not_seen(gpu_device):
    torch, b, rng = _t(), _b(), np.random.default_rng(15)
    case = _attend_case(rng, "bf16", 2, 2, 64, [0, 200, 300, 0, 128], [2, 1, 3, 1, 1])
    cu, table, lengths, codes, scales, q = case
    lengths[0] = 1                      # row 0 lies before the sequence's beginning
    table[1, :] = -1                    # nothing there
    table[2, 0], table[2, 3] = 1 << 30, codes.shape[0]
    lengths[3] = 0
    lengths[4] = 64 * table.shape[1] + 40  # longer than its table
    table[4, :] = table[2, 1]           # one page many times, shared with another sequence
    for window, sinks in ((0, 0), (100, 3)):
        want = o.attend(codes, scales, q, cu, table, lengths, 0.1, window, sinks)
        assert (want[0][0] == 0).all() and (want[0][2] == 0).all() and (want[0][6] == 0).all()
        got = _np(_attend(case, "bf16", 0.1, window, sinks))
        _check_attention(got, want, "bf16", 64, int(lengths.max()), q)


def _among_empty(cu, table, lengths, front, back, rng):
    """The same step with sequences that bring nothing before and behind."""
    def around(x, a, z):
        return np.concatenate([a, x, z]).astype(np.int32)

    n = table.shape[1]
    some = lambda k: rng.integers(-5, 300, k)  # noqa: E731
    return (around(cu, np.zeros(front), np.full(back, cu[-1])), around(table, rng.integers(-3, 9, (front, n)), rng.integers(-3, 9, (back, n))),
            around(lengths, some(front), some(back)))


@pytest.mark.parametrize("front,back", [(3, 61), (70, 30), (400, 1100)])
@pytest.mark.parametrize("dtype,heads,hd,rot,layout", [("bf16", 3, 64, 32, o.HALVES), ("fp16", 2, 128, 128, o.ADJACENT), ("fp32", 1, 128, 64, o.HALVES),
                                                       ("bf16", 3, 256, 256, o.ADJACENT), ("fp16", 1, 256, 0, o.HALVES), ("fp32", 2, 64, 64, o.ADJACENT)])
def test_sequences_that_bring_nothing_change_nothing(gpu_device, front, back, dtype, heads, hd, rot, layout):
    """Bit for bit, though other kernels and other searches run: append, read and attention of single tokens."""
    torch, b, rng = _t(), _b(), np.random.default_rng(front + hd)
    olds, news = [0, 5, 63, 100, 64, 20, 33], [1, 60, 1, 3, 70, 1, 9]
    cu, table, lengths, codes, scales, k, v, cos, sin = _append_case(rng, dtype, heads, hd, rot, layout, olds, news, big=30.0, extra_rows=1)
    k[0, 0, 5], k[2, -1, 0], v[1, 0, 3] = np.nan, np.inf, -np.inf
    want = o.append(codes, scales, k, v, cu, table, lengths, None if cos is None else cos.astype(np.float64),
                    None if sin is None else sin.astype(np.float64), layout)
    kw = dict(cos=None if cos is None else _dev(cos), sin=None if sin is None else _dev(sin), layout=layout)
    rows, first = k.shape[0], np.maximum(lengths - 20, 0).astype(np.int32)
    wide = _among_empty(cu, table, lengths, front, back, rng)
    results = []
    for arrays, f in (((cu, table, lengths), first), (wide, np.concatenate([np.zeros(front), first, np.zeros(back)]))):
        cache = b.Cache8(_dev(codes), _dev(scales.astype(np.float32)))
        args = tuple(_i32(x) for x in arrays)
        cache.append(_dev(k, _type(dtype)), _dev(v, _type(dtype)), *args, **kw)
        out = tuple(torch.zeros(rows, heads, hd, device="cuda", dtype=_type(dtype)) for _ in range(2))
        cache.read(rows, args[0], _i32(f), *args[1:], out=out, **kw)
        results.append((cache.pages, cache.scales, *(x.view(torch.int32 if dtype == "fp32" else torch.int16) for x in out)))
    for one, other in zip(*results):
        assert torch.equal(one, other)
    _check_append(results[1][0].cpu().numpy(), _np(results[1][1]), want, codes, (cu, table, lengths, codes, scales, k, v, cos, sin))
    case = _attend_case(rng, dtype, heads, 4, hd, [0, 5, 63, 100, 64, 2000, 33] * 3, [1, 1, 0, 1, 1, 1, 1] * 3)
    cu, table, lengths, codes, scales, q = case
    got = _attend(case, dtype, 0.1)
    wide = _among_empty(cu, table, lengths, front, back, rng)
    assert torch.equal(got, _attend((*wide, codes, scales, q), dtype, 0.1))


def test_step_arrays_that_make_no_sense_stay_in_bounds(gpu_device):
    """cu beyond the rows, descending, negative: rows are clamped to the step's, no row is read or written outside."""
    torch, b, rng = _t(), _b(), np.random.default_rng(16)
    case = _attend_case(rng, "fp16", 1, 2, 64, [10, 20, 30], [2, 2, 2])
    _, table, lengths, codes, scales, q = case
    for cu in ([-5, 3, 2, 1000], [0, 6, 6, 6], [4, 2, 1, 0]):
        cu = np.array(cu, dtype=np.int32)
        want = o.attend(codes, scales, q, cu, table, lengths, 0.1)
        out = torch.zeros(6, 2, 64, device="cuda", dtype=torch.float16)
        got = _np(_attend((cu, table, lengths, codes, scales, q), "fp16", 0.1, out=out))
        _check_attention(got, want, "fp16", 64, 40, q)


def test_pages_beyond_four_gigabytes(gpu_device):
    torch, b, rng = _t(), _b(), np.random.default_rng(17)
    heads, hd = 8, 128
    n_pages = (1 << 32) // (heads * 2 * 64 * hd) + 40
    pages = torch.empty((n_pages, heads, 2, 64 * hd), dtype=torch.uint8, device="cuda")
    scales = torch.ones((n_pages, heads, 2), device="cuda")
    cache = b.Cache8(pages, scales)
    table = np.array([[n_pages - 1, 3, n_pages - 30]], dtype=np.int32)
    k, v = (_rounded(rng.standard_normal((150, heads, hd)), "bf16") for _ in range(2))
    q = _rounded(rng.standard_normal((150, heads, hd)), "bf16")
    cu, lengths = np.array([0, 150], dtype=np.int32), np.array([150], dtype=np.int32)
    cache.append(_dev(k, _type("bf16")), _dev(v, _type("bf16")), _i32(cu), _i32(table), _i32(lengths))
    out = _np(cache.attend(_dev(q, _type("bf16")), _i32(cu), _i32(table), _i32(lengths)))
    rk, rv = cache.read(150, _i32(cu), _i32([0]), _i32(table), _i32(lengths), dtype=torch.float32)
    small, ss = np.zeros((3, heads, 2, 64 * hd), dtype=np.uint8), np.ones((3, heads, 2))
    t3 = np.array([[0, 1, 2]], dtype=np.int32)
    codes, sc, _ = o.append(small, ss, k, v, cu, t3, lengths)
    wk, wv = o.read(codes, sc, 150, cu, [0], t3, lengths)
    assert np.array_equal(_np(rk), wk) and np.array_equal(_np(rv), wv)
    _check_attention(out, o.attend(codes, sc, q, cu, t3, lengths, hd**-0.5), "bf16", hd, 150, q)


# ---- together, as a serving loop uses them -----------------------------------------------------
class _Loop:
    """Three sequences that prefill and then decode; the oracle walks along."""

    def __init__(self, seed, dtype="bf16", heads=2, rep=4, hd=128, rot=128, layout=o.ADJACENT, seqs=3, room=6):
        torch, b = _t(), _b()
        self.rng = np.random.default_rng(seed)
        self.dtype, self.heads, self.rep, self.hd, self.rot, self.layout = dtype, heads, rep, hd, rot, layout
        self.table = self.rng.permutation(seqs * room).reshape(seqs, room).astype(np.int32)
        self.codes, self.scales = _random_pool(self.rng, seqs * room, heads, hd)
        self.cache = b.Cache8(_dev(self.codes), _dev(self.scales.astype(np.float32)))
        self.lengths = np.zeros(seqs, dtype=np.int32)
        self.rows = []

    def inputs(self, news):
        rows = int(sum(news))
        self.lengths = self.lengths + np.array(news, dtype=np.int32)
        cu = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        pos = np.concatenate([np.arange(t - n, t) for t, n in zip(self.lengths, news)]).astype(np.int64)
        shape = [(rows, self.heads * self.rep, self.hd), (rows, self.heads, self.hd), (rows, self.heads, self.hd)]
        q, k, v = (_rounded(self.rng.standard_normal(s), self.dtype) for s in shape)
        return cu, pos, q, k, v

    def device(self, step):
        cu, pos, q, k, v = step
        t = _type(self.dtype)
        return dict(cu=_i32(cu), pos=_dev(pos), q=_dev(q, t), k=_dev(k, t), v=_dev(v, t), lengths=_i32(self.lengths), table=_i32(self.table))

    def run(self, d, **kw):
        b = _b()
        cos, sin = b.rope_tables(d["pos"], self.rot)
        q = b.rope(d["q"], cos, sin, layout=self.layout)
        self.cache.append(d["k"], d["v"], d["cu"], d["table"], d["lengths"], cos=cos, sin=sin, layout=self.layout)
        return q, self.cache.attend(q, d["cu"], d["table"], d["lengths"], window=150, sinks=2, **kw)

    def check(self, step, q, out):
        """The oracle's step from the codes that the GPU wrote (its own keys' codes may differ by a tie)."""
        cu, pos, _, k, v = step
        cos, sin = o.tables(pos, self.rot)
        want = o.append(self.codes, self.scales, k, v, cu, self.table, self.lengths, cos, sin, self.layout)
        got = self.cache.pages.cpu().numpy(), _np(self.cache.scales)
        assert np.array_equal(got[1], want[1])
        assert ((got[0] == want[0]) | ((got[0] & 127) == 0)).mean() > 0.999
        self.codes, self.scales = got
        _check_attention(_np(out), o.attend(*got, _np(q), cu, self.table, self.lengths, self.hd**-0.5, 150, 2), self.dtype, self.hd,
                         int(self.lengths.max()), None)


@pytest.mark.parametrize("dtype,layout,rot", [("bf16", o.ADJACENT, 128), ("fp16", o.HALVES, 64), ("fp32", o.HALVES, 128)])
def test_a_serving_loop(gpu_device, dtype, layout, rot):
    loop = _Loop(20, dtype=dtype, layout=layout, rot=rot)
    for news in ([100, 63, 1], [1, 1, 1], [1, 0, 1], [2, 3, 1], [150, 1, 40], [1, 1, 1]):
        step = loop.inputs(news)
        q, out = loop.run(loop.device(step))
        loop.check(step, q, out)


def test_tokens_that_leave_the_cache_are_encoded(gpu_device):
    """Keys read back un-rotated, values as they are, through the quantizer of the framework: the codes of what the cache holds."""
    torch, b = _t(), _b()
    loop = _Loop(21, dtype="fp16")
    step = loop.inputs([120, 90, 64])
    loop.run(loop.device(step))
    d = loop.device(step)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    quant = b.Quantizer(d=128, dhat=32, depth=4, K=256, grouping=b.STRIDED, in_dtype=b.F16)
    quant.set_codebooks(torch.randn(4, 256, 32, device="cuda", generator=gen))
    cu, first, n = _i32([0, 50, 100, 150]), _i32([0, 0, 0]), 150
    pos = np.concatenate([np.arange(50)] * 3)
    cos, sin = b.rope_tables(_dev(pos.astype(np.int64)), 128)
    k, v = loop.cache.read(n, cu, first, d["table"], d["lengths"], dtype=torch.float16, cos=cos, sin=sin)
    # an e4m3 rounding of a rotated pair is off by at most 2^-4 of each, so is the pair turned back
    held = np.concatenate([step[3][c : c + 50] for c in (0, 120, 210)])
    pair = np.hypot(held[..., 0::2], held[..., 1::2]).repeat(2, axis=2)
    assert np.all(np.abs(_np(k) - held) <= 2.0**-4 * pair * 1.01 + 2.0**-8 * loop.scales.max())
    codes, std, _ = quant.encode(k.reshape(n * 2, 128))
    back = quant.decode(codes, std)
    plain, pstd, _ = quant.encode(_dev(_np(k)).half().reshape(n * 2, 128))
    assert torch.equal(codes, plain) and torch.equal(std, pstd) and torch.isfinite(back).all()
    quant.close()


def test_captured_steps_are_replayed_with_other_lengths_and_pages(gpu_device):
    """Two captured graphs of a decoding step with a workspace each, on two loops, replayed in turn with eager work in between."""
    torch, b = _t(), _b()
    loops = [_Loop(30, seqs=3), _Loop(31, seqs=3, dtype="fp16", layout=o.HALVES)]
    graphs = []
    for loop in loops:
        step = loop.inputs([70, 130, 5])
        q, out = loop.run(loop.device(step))
        loop.check(step, q, out)
        step = loop.inputs([1, 1, 1])
        d = loop.device(step)
        ws = torch.empty(loop.cache.workspace_bytes(d["q"], 3), dtype=torch.uint8, device="cuda")
        q, out = loop.run(d, workspace=ws)
        loop.check(step, q, out)
        pages, scales = loop.cache.pages.clone(), loop.cache.scales.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            q, out = loop.run(d, workspace=ws)
        loop.cache.pages.copy_(pages)
        loop.cache.scales.copy_(scales)
        graphs.append((g, d, q, out))
    for turn in range(4):
        todo = []
        for loop, (g, d, q, out) in zip(loops, graphs):
            step = loop.inputs([1, 1, 1])
            for name, x in loop.device(step).items():
                d[name].copy_(x)
            if turn == 2:  # another order of the pages: the table is read by the replay
                order = loop.rng.permutation(len(loop.codes))
                loop.codes, loop.scales = loop.codes[order], loop.scales[order]
                loop.table = np.argsort(order)[loop.table].astype(np.int32)
                loop.cache.pages.copy_(_dev(loop.codes))
                loop.cache.scales.copy_(_dev(loop.scales.astype(np.float32)))
                d["table"].copy_(_i32(loop.table))
            todo.append((loop, step, q, out))
        for g, *_ in graphs:
            g.replay()
        for loop, step, q, out in todo:
            loop.check(step, q, out)
        torch.cuda.synchronize()


def test_calls_on_another_stream(gpu_device):
    """The work goes to the current stream: behind queued work of a side stream, and two caches on two streams at once."""
    torch = _t()
    loops = [_Loop(40), _Loop(41, dtype="fp32")]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for news in ([200, 3, 64], [1, 1, 1]):
        todo = []
        for loop, s in zip(loops, streams):
            step = loop.inputs(news)
            d = loop.device(step)
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                torch.cuda._sleep(2_000_000)
                q, out = loop.run(d)
            todo.append((loop, step, q, out, d))
        for s in streams:
            s.synchronize()
        for loop, step, q, out, _ in todo:
            loop.check(step, q, out)


def test_results_do_not_depend_on_the_run(gpu_device):
    """No atomics: the same bits every time."""
    torch = _t()
    rng = np.random.default_rng(50)
    case = _attend_case(rng, "bf16", 2, 4, 128, [3000, 700, 5], [1, 1, 1])
    first = _attend(case, "bf16", 0.05)
    for _ in range(3):
        assert torch.equal(_attend(case, "bf16", 0.05), first)


@pytest.mark.parametrize("dtype,rep", [("fp32", 2), ("bf16", 2), ("fp16", 60)])
def test_windows_and_sinks_of_the_largest_sizes(gpu_device, dtype, rep):
    """Beyond every length, alone and together, they hide nothing; a window of the length and no sinks likewise."""
    rng, most = np.random.default_rng(60), 2**31 - 1
    case = _attend_case(rng, dtype, 1, rep, 64, [300, 0, 70], [3, 1, 1])
    cu, table, lengths, codes, scales, q = case
    full = _np(_attend(case, dtype, 0.1))
    _check_attention(full, o.attend(codes, scales, q, cu, table, lengths, 0.1), dtype, 64, 303, q)
    for window, sinks in ((most, 0), (most, most), (1, most), (303, 0), (0, most)):
        want = o.attend(codes, scales, q, cu, table, lengths, 0.1, window, sinks)
        _check_attention(_np(_attend(case, dtype, 0.1, window=window, sinks=sinks)), want, dtype, 64, 303, q)
        assert np.allclose(want[0], o.attend(codes, scales, q, cu, table, lengths, 0.1)[0], atol=1e-12)


@pytest.mark.parametrize("dtype,rep", [("fp32", 1), ("bf16", 3), ("bf16", 50), ("fp16", 40)])
def test_tokens_behind_the_table_and_shared_pages(gpu_device, dtype, rep):
    """Lengths beyond the table's room: queries out there see what the table holds.  Pages named twice and by two sequences."""
    rng = np.random.default_rng(61)
    case = _attend_case(rng, dtype, 2, rep, 128, [100, 190, 64, 200], [2, 1, 3, 4])
    cu, table, lengths, codes, scales, q = case
    table[0, :2] = table[1, [2, 2]]
    table[2, :2] = table[1, :2]
    lengths = lengths.copy()
    lengths[1] = 64 * table.shape[1] + 1000   # its query has no page
    lengths[3] = 64 * table.shape[1] + 2      # two of its queries have none
    case = cu, table, lengths, codes, scales, q
    for window, sinks in ((0, 0), (90, 3), (5, 0)):
        want = o.attend(codes, scales, q, cu, table, lengths, 0.06, window, sinks)
        _check_attention(_np(_attend(case, dtype, 0.06, window=window, sinks=sinks)), want, dtype, 128, int(lengths.max()), q)


@pytest.mark.parametrize("dtype,rep", [("fp32", 3), ("bf16", 3), ("fp16", 50)])
def test_strided_and_broadcast_queries_and_strided_results(gpu_device, dtype, rep):
    torch, rng = _t(), np.random.default_rng(62)
    case = _attend_case(rng, dtype, 2, rep, 64, [100, 3], [2, 1])
    cu, table, lengths, codes, scales, q = case
    q[:] = q[:, :1]
    cache = _b().Cache8(_dev(codes), _dev(scales.astype(np.float32)))
    args = (_i32(cu), _i32(table), _i32(lengths))
    want = o.attend(codes, scales, q, cu, table, lengths, 0.1)
    one = torch.zeros(3, 5, 64, device="cuda", dtype=_type(dtype))
    one[:, 2] = _dev(q[:, 0], _type(dtype))
    out = torch.full((4, 2 * rep, 3, 64), 9.0, device="cuda", dtype=_type(dtype))
    got = cache.attend(one[:, 2:3].expand(3, 2 * rep, 64), *args, scale=0.1, out=out[:3, :, 1])
    _check_attention(_np(got), want, dtype, 64, 102, q)
    assert (out[:, :, 0] == 9.0).all() and (out[:, :, 2] == 9.0).all() and (out[3] == 9.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("sharp", [4.0, 12.0])
def test_scores_of_chunks_are_sums_of_full_length(gpu_device, dtype, sharp):
    """Large products of either sign that cancel: what a short sum loses of them would show in the weights."""
    rng = np.random.default_rng(65)
    case = _attend_case(rng, dtype, 1, 40, 128, [191, 400], [15, 9], sharp=sharp)
    cu, table, lengths, codes, scales, q = case
    _check_attention(_np(_attend(case, dtype, 0.1)), o.attend(codes, scales, q, cu, table, lengths, 0.1), dtype, 128, 409, q)


def test_a_thousand_kv_heads_and_hundreds_of_queries_of_one(gpu_device):
    rng = np.random.default_rng(63)
    case = _attend_case(rng, "bf16", 1024, 1, 64, [70, 2], [1, 1])
    _attend_heads(case, "bf16", 0.1, 0, 0, 1024, 1, 64, (0, 511, 1023))
    case = _attend_case(rng, "fp16", 1, 300, 128, [900], [1])
    _attend_heads(case, "fp16", 0.1, 0, 0, 1, 300, 128, (0,))
    case = _append_case(rng, "bf16", 1023, 64, 16, o.HALVES, [5, 63], [1, 2])
    cu, table, lengths, codes, scales, k, v, cos, sin = case
    want = o.append(codes, scales, k, v, cu, table, lengths, cos.astype(np.float64), sin.astype(np.float64), o.HALVES)
    cache = _b().Cache8(_dev(codes), _dev(scales.astype(np.float32)))
    cache.append(_dev(k, _type("bf16")), _dev(v, _type("bf16")), _i32(cu), _i32(table), _i32(lengths), _dev(cos), _dev(sin), layout=o.HALVES)
    _check_append(cache.pages.cpu().numpy(), _np(cache.scales), want, codes, case)


def test_a_captured_chunk_is_replayed_behind_caches_of_other_lengths(gpu_device):
    """The same rows alone, behind many tokens and behind few: blocks go by whole items or by runs as the lengths say."""
    torch, b, rng = _t(), _b(), np.random.default_rng(64)
    heads, rep, hd, n = 2, 8, 128, 200
    cu, table, lengths, codes, scales, q = _attend_case(rng, "bf16", heads, rep, hd, [5000], [n])
    cache = b.Cache8(_dev(codes), _dev(scales.astype(np.float32)))
    dq, dcu, dtable, dlen = _dev(q, _type("bf16")), _i32(cu), _i32(table), _i32(lengths)
    ws = torch.empty(cache.workspace_bytes(dq, 1), dtype=torch.uint8, device="cuda")
    out = cache.attend(dq, dcu, dtable, dlen, scale=0.05, workspace=ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        cache.attend(dq, dcu, dtable, dlen, scale=0.05, workspace=ws, out=out)
    for length in (n, 5000 + n, 700, n + 3, 3000):
        dlen.fill_(length)
        out.fill_(9.0)
        g.replay()
        got = out.clone()
        eager = cache.attend(dq, dcu, dtable, dlen, scale=0.05)
        assert torch.equal(got, eager)
        part = slice(rep, 2 * rep)
        want = o.attend(codes[:, 1:], scales[:, 1:], q[:, part], cu, table, np.array([length]), 0.05)
        _check_attention(_np(got)[:, part], want, "bf16", hd, length, q)


def test_a_workspace_that_is_too_small_is_refused(gpu_device):
    torch, b = _t(), _b()
    case = _attend_case(np.random.default_rng(51), "bf16", 1, 1, 64, [10], [1])
    cu, table, lengths, codes, scales, q = case
    cache = b.Cache8(_dev(codes), _dev(scales.astype(np.float32)))
    dq = _dev(q, _type("bf16"))
    need = cache.workspace_bytes(dq, 1)
    out = torch.full_like(dq, 3.0)
    with pytest.raises(b.RvqError) as e:
        cache.attend(dq, _i32(cu), _i32(table), _i32(lengths), out=out, workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == b.RVQ_EWORKSPACE
    torch.cuda.synchronize()
    assert (out == 3.0).all()
    with pytest.raises(b.RvqError):
        cache.attend(dq, _i32(cu), _i32(table), _i32(lengths), out=dq)
