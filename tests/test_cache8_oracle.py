"""The fp64 oracle of the 8-bit cache against torch and SciPy, and the refusals of the entry points (no GPU work: every
refusal is decided by the host before anything is enqueued)."""
import ctypes

import numpy as np
import pytest
import torch
from scipy.special import softmax

from oracle import cache8 as o
from paper_2410_15704_amd import binding as b

FAKE = 1 << 20  # an aligned address that a refused call never reads


# ---- the oracle --------------------------------------------------------------------------------
def test_codes_are_those_of_torchs_e4m3():
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, o.VALUES, equal_nan=True)
    rng = np.random.default_rng(0)
    x = rng.standard_normal(50000) * 2.0 ** rng.integers(-12, 7, 50000)
    x = np.concatenate([np.clip(x, -448, 448), (o.VALUES[:126] + o.VALUES[1:127]) / 2]).astype(np.float32)  # ties too
    assert np.array_equal(torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), o.encode(x))
    assert o.encode(np.array([np.inf, -np.inf, np.nan])).tolist() == [127, 127, 127]


def test_scale_is_the_smallest_power_of_two_in_range():
    for amax in (448.0, 448.0 * (1 + 1e-9), 1.0, 3e-30, 1e30, 0.0, 7.0 * 2**-9):
        s = o.scale_of(amax)
        assert amax <= 448 * s and (s == 2.0**-100 or amax > 448 * s / 2) and np.frexp(s)[0] == 0.5


@pytest.mark.parametrize("layout", [o.ADJACENT, o.HALVES])
def test_rotation_is_a_product_of_complex_numbers(layout):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 3, 32))
    cos, sin = o.tables([0, 1, 17, 4000, 131071], 16)
    y = o.rotate(x, cos, sin, layout)
    part = x[..., :16].reshape(5, 3, 8, 2) if layout == o.ADJACENT else x[..., :16].reshape(5, 3, 2, 8).swapaxes(2, 3)
    z = (part[..., 0] + 1j * part[..., 1]) * np.exp(1j * np.arctan2(sin, cos))[:, None]
    got = y[..., :16].reshape(5, 3, 8, 2) if layout == o.ADJACENT else y[..., :16].reshape(5, 3, 2, 8).swapaxes(2, 3)
    assert np.allclose(got[..., 0] + 1j * got[..., 1], z, atol=1e-13)
    assert np.array_equal(y[..., 16:], x[..., 16:])
    assert np.allclose(o.rotate(y, cos, -sin, layout), x, atol=1e-13)


def test_tables_stretch_by_parts():
    pos = np.arange(7)
    plain, linear = o.tables(pos, 32), o.tables(pos * 8, 32, factor=8.0)
    assert np.allclose(plain, linear, atol=1e-14)  # everything divided
    parts = o.tables(pos, 32, factor=8.0, orig_len=4096, alpha=1, beta=32)
    assert np.allclose(parts[0][:, 0], plain[0][:, 0])  # a fast frequency stays
    slow = o.tables(pos, 32, factor=8.0)
    assert np.allclose(parts[0][:, -1], slow[0][:, -1])  # a slow one is divided (0.1 turns in 4096 tokens)


def test_append_in_two_steps_then_read_gives_the_tokens_back():
    rng = np.random.default_rng(2)
    hd, heads = 64, 2
    codes, scales = rng.integers(0, 256, (5, heads, 2, 64 * hd)).astype(np.uint8), np.ones((5, heads, 2))
    table, k, v = np.array([[3, 1, 4]]), rng.standard_normal((100, heads, hd)), 1e-3 * rng.standard_normal((100, heads, hd))
    k[60:] *= 50  # the second step's keys are larger: page 3's earlier codes are rounded again
    c1, s1, _ = o.append(codes, scales, k[:50], v[:50], [0, 50], table, [50])
    c2, s2, _ = o.append(c1, s1, k[50:], v[50:], [0, 50], table, [100])
    assert (s2[3, :, 0] > s1[3, :, 0]).all()
    assert np.array_equal(c2[[0, 2, 4]], codes[[0, 2, 4]])  # other pages
    rk, rv = o.read(c2, s2, 100, [0, 100], [0], table, [100])
    # a half step of e4m3 is 2^-4 of the value; the first 50 keys were rounded twice; below 2^-6 scales, steps of 2^-9
    assert np.all(np.abs(rv - v) <= 2.0**-4 * np.abs(v) + 2.0**-10 * s2[[3, 1]].max())
    assert np.all(np.abs(rk - k) <= 2 * 2.0**-4 * 1.07 * np.abs(k) + 2.0**-9 * s2[[3, 1]].max())


def test_attention_of_the_oracle_is_a_softmax_over_what_is_seen():
    rng = np.random.default_rng(3)
    hd, heads, n = 64, 2, 150
    codes = rng.integers(0, 120, (4, heads, 2, 64 * hd)).astype(np.uint8)
    scales, table = np.full((4, heads, 2), 2.0**-6), np.array([[2, 0, 3]])
    q = rng.standard_normal((3, 4, hd)) * 0.1
    out, _, _ = o.attend(codes, scales, q, [0, 3], table, [n], 0.1, window=40, sinks=2)
    k, v = o.read(codes, scales, n, [0, n], [0], table, [n])
    for i in range(3):
        p = n - 3 + i
        t = np.array([x for x in range(n) if x <= p and (x > p - 40 or x < 2)])
        for a in range(4):
            w = softmax(k[t, a // 2] @ q[i, a] * 0.1)
            assert np.allclose(out[i, a], w @ v[t, a // 2], rtol=1e-12)


# ---- refusals ----------------------------------------------------------------------------------
def _view(**kw):
    d = dict(pages=FAKE, scales=FAKE, n_pages=4, n_kv_heads=2, head_dim=64, table=FAKE, table_pages=3, n_seqs=1, lengths=FAKE)
    d.update(kw)
    return b.rvq_cache8(*[d[n] for n, _ in b.rvq_cache8._fields_])


BAD_VIEWS = [dict(pages=None), dict(pages=FAKE + 8), dict(scales=None), dict(scales=FAKE + 4), dict(n_pages=0), dict(n_pages=1 << 60),
             dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=96), dict(head_dim=0), dict(table=None), dict(table=FAKE + 2),
             dict(table_pages=0), dict(table_pages=1 << 30), dict(n_seqs=0), dict(n_seqs=65536), dict(lengths=None)]


def _append(view, **kw):
    d = dict(k=FAKE, v=FAKE, dtype=b.BF16, rows=3, ldk=128, hsk=64, ldv=128, hsv=64, cu=FAKE, cos=FAKE, sin=FAKE, rot=32,
             layout=b.ROPE_ADJACENT)
    d.update(kw)
    return b.lib.rvq_cache8_append(view and ctypes.byref(view), *d.values(), None)


def _read(view, **kw):
    d = dict(cu=FAKE, first=FAKE, rows=3, cos=FAKE, sin=FAKE, rot=32, layout=b.ROPE_ADJACENT, dtype=b.BF16, k=FAKE, ldk=128, hsk=64,
             v=FAKE, ldv=128, hsv=64)
    d.update(kw)
    return b.lib.rvq_cache8_read(view and ctypes.byref(view), *d.values(), None)


def _attn(view, **kw):
    d = dict(q=FAKE, dtype=b.BF16, rows=3, heads=4, ldq=256, hsq=64, cu=FAKE, scale=0.1, window=0, sinks=0, out=2 * FAKE, ldo=256,
             hso=64, ws=FAKE, ws_bytes=1 << 40)
    d.update(kw)
    return b.lib.rvq_cache8_attn(view and ctypes.byref(view), *d.values(), None)


@pytest.mark.parametrize("call", [_append, _read, _attn])
def test_bad_caches_are_refused(call):
    assert call(None) == b.RVQ_EINVAL
    for bad in BAD_VIEWS:
        assert call(_view(**bad)) == b.RVQ_EINVAL, bad
    assert call(_view(pages=None), rows=0) == b.RVQ_OK  # nothing to do


@pytest.mark.parametrize("bad", [
    dict(k=None), dict(v=None), dict(k=FAKE + 2), dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 31), dict(ldk=129),
    dict(hsk=68), dict(ldv=-128), dict(ldv=1 << 62), dict(cu=None), dict(cu=FAKE + 1), dict(cos=None), dict(sin=None), dict(cos=FAKE + 4), dict(rot=0), dict(rot=8),
    dict(rot=80), dict(rot=-16), dict(layout=2), dict(cos=None, sin=None)])
def test_append_refuses(bad):
    assert _append(_view(), **bad) == b.RVQ_EINVAL


@pytest.mark.parametrize("bad", [
    dict(first=None), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(dtype=9), dict(rows=-5), dict(ldk=64), dict(hsk=32), dict(ldv=0), dict(hsv=0),
    dict(cos=None), dict(rot=40), dict(layout=-1), dict(cu=None)])
def test_read_refuses(bad):
    assert _read(_view(), **bad) == b.RVQ_EINVAL
    assert _read(_view(), k=None, v=None) == b.RVQ_OK


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(q=FAKE + 8), dict(out=None), dict(out=FAKE), dict(dtype=4), dict(rows=-1), dict(heads=3), dict(heads=1), dict(heads=0),
    dict(heads=1 << 20), dict(ldq=100), dict(hsq=60), dict(ldo=128), dict(hso=32), dict(ldo=0), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(window=-1), dict(sinks=-1), dict(ws=None), dict(ws=FAKE + 4), dict(cu=None), dict(rows=(1 << 31) - 1)])
def test_attention_refuses(bad):
    assert _attn(_view(), **bad) == b.RVQ_EINVAL


def test_rope_refuses():
    def tables(pos=FAKE, N=4, rot=32, base=1e4, factor=1.0, orig=0.0, alpha=1.0, beta=32.0, amp=1.0, cos=FAKE, sin=FAKE):
        return b.lib.rvq_rope_tables(pos, N, rot, base, factor, orig, alpha, beta, amp, cos, sin, None)

    nan, inf = float("nan"), float("inf")
    for bad in (dict(pos=None), dict(pos=FAKE + 4), dict(N=-1), dict(rot=0), dict(rot=7), dict(base=0.0), dict(base=nan), dict(base=inf),
                dict(factor=0.0), dict(factor=nan), dict(orig=-1.0), dict(orig=8.0, alpha=3.0, beta=3.0), dict(orig=8.0, alpha=nan),
                dict(amp=inf), dict(cos=None), dict(sin=FAKE + 2), dict(N=1 << 62)):
        assert tables(**bad) == b.RVQ_EINVAL, bad
    assert tables(N=0, pos=None) == b.RVQ_OK

    def rope(x=FAKE, dtype=b.BF16, N=4, heads=2, hd=64, rot=32, layout=0, ldx=128, hsx=64, cos=FAKE, sin=FAKE, out=2 * FAKE, ldo=128, hso=64):
        return b.lib.rvq_rope(x, dtype, N, heads, hd, rot, layout, ldx, hsx, cos, sin, out, ldo, hso, None)

    for bad in (dict(x=None), dict(x=FAKE + 1), dict(dtype=3), dict(N=-1), dict(heads=0), dict(hd=1), dict(rot=0), dict(rot=66), dict(rot=3),
                dict(layout=2), dict(ldx=-1), dict(cos=None), dict(sin=None), dict(out=None), dict(ldo=0), dict(hso=32), dict(ldo=100),
                dict(out=FAKE, ldo=256), dict(N=1 << 60), dict(ldo=1 << 62)):
        assert rope(**bad) == b.RVQ_EINVAL, bad
    assert rope(N=0, x=None) == b.RVQ_OK


def test_the_binding_refuses_what_the_entry_points_cannot_see():
    q = torch.zeros(3, 4, 64)
    with pytest.raises(ValueError):
        b.Cache8(torch.zeros(2, 2, 64 * 64, dtype=torch.uint8), torch.zeros(2, 2))
    with pytest.raises(ValueError):
        b.Cache8(torch.zeros(2, 2, 2, 64 * 64), torch.zeros(2, 2, 2))  # type of the codes
    with pytest.raises(ValueError):
        b.Cache8(torch.zeros(2, 2, 2, 64 * 64, dtype=torch.uint8), torch.zeros(2, 2))
    c = b.Cache8.empty(2, 2, 64, device="cpu")
    i = dict(dtype=torch.int32)
    cu, table, lengths = torch.tensor([0, 3], **i), torch.zeros(1, 2, **i), torch.tensor([3], **i)
    k = torch.zeros(3, 2, 64)
    with pytest.raises(TypeError):
        c.append(k.double(), k.double(), cu, table, lengths)
    for kk, vv, args in ((k, k.half(), (cu, table, lengths)), (k, k[:2], (cu, table, lengths)), (k[:, :1], k, (cu, table, lengths)),
                         (k.transpose(1, 2).contiguous().transpose(1, 2), k, (cu, table, lengths)), (k, k, (cu.long(), table, lengths)),
                         (k, k, (cu[:1], table, lengths)), (k, k, (cu, table[0], lengths)), (k, k, (cu, table, lengths[None]))):
        with pytest.raises(ValueError):
            c.append(kk, vv, *args)
    with pytest.raises(ValueError):
        c.append(k, k, cu, table, lengths, cos=torch.zeros(3, 32))
    with pytest.raises(ValueError):
        c.append(k, k, cu, table, lengths, cos=torch.zeros(2, 32), sin=torch.zeros(2, 32))
    for call in (lambda: c.append(k, k, cu, table, lengths), lambda: c.attend(q, cu, table, lengths), lambda: c.attend(q[..., :32], cu, table, lengths),
                 lambda: b.rope(q, torch.zeros(3, 32), torch.zeros(3, 32)), lambda: b.rope_tables(torch.zeros(3, dtype=torch.int64), 32)):
        with pytest.raises(ValueError):  # not on a GPU
            call()


def test_numbers_that_pass_fp32_on_the_way_are_refused():
    assert _attn(_view(), scale=3e38) == b.RVQ_EINVAL
    assert b.lib.rvq_rope_tables(FAKE, 4, 32, 1e4, 1.0, 0.0, 1.0, 32.0, 1e300, FAKE, FAKE, None) == b.RVQ_EINVAL
