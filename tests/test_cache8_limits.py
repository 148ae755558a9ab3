"""What the paged 8-bit cache promises at the ends of its range, as far as no GPU is needed for it."""
import numpy as np
import pytest

from oracle import cache8 as o
from paper_2410_15704_amd import binding as b
from paper_2410_15704_amd import build


def test_attention_is_compiled_with_nan():
    """A NaN code reaches the result of the rows that see it: nothing that handles one may be compiled as if there were none."""
    for name in ("rvq_cache8.hip", "rvq_cache8_attn.hip", "rvq_cache8_chunk.hip", "rvq_rope.hip"):
        flags = build.FLAGS + build.EXTRA.get(name, [])
        assert not [f for f in flags if f in ("-fno-honor-nans", "-ffast-math", "-ffinite-math-only", "-fno-honor-infinities")], name


@pytest.mark.parametrize("layout", [o.ADJACENT, o.HALVES])
@pytest.mark.parametrize("amplitude", [1.0, 1.2, 0.3, 40.0])
def test_keys_come_back_from_tables_of_any_amplitude(layout, amplitude):
    """The oracle: appended and read with the same tables, keys are what they were, but for their codes' rounding."""
    rng = np.random.default_rng(80)
    hd, heads, n, rot = 64, 2, 100, 32
    codes, scales = np.zeros((3, heads, 2, 64 * hd), dtype=np.uint8), np.ones((3, heads, 2))
    table, k, v = np.array([[2, 0]]), rng.standard_normal((n, heads, hd)), rng.standard_normal((n, heads, hd))
    cos, sin = o.tables(np.arange(n), rot, amplitude=amplitude)
    c1, s1, exact = o.append(codes, scales, k, v, [0, n], table, [n], cos, sin, layout)
    rk, rv = o.read(c1, s1, n, [0, n], [0], table, [n], cos, sin, layout)
    for t in range(n):
        page, slot = table[0, t // 64], t % 64
        for h in range(heads):
            s, x = s1[page, h, 0], exact[page, h, 0, slot]
            # half a step of each code, 2^-4 of it or 2^-10 of the scale; a pair turned back mixes its two errors
            half = np.maximum(2.0**-4 * np.abs(x), 2.0**-10 * s)
            a, b = (slice(0, rot, 2), slice(1, rot, 2)) if layout == o.ADJACENT else (slice(0, rot // 2), slice(rot // 2, rot))
            pair = np.hypot(half[a], half[b]) / amplitude
            for part in (a, b):
                assert np.all(np.abs(rk[t, h][part] - k[t, h][part]) <= pair * (1 + 1e-12))
            assert np.all(np.abs(rk[t, h][rot:] - k[t, h][rot:]) <= half[rot:])


@pytest.mark.parametrize("dtype", [b.BF16, b.F32])
@pytest.mark.parametrize("heads,rep,hd,seqs", [(8, 4, 128, 1), (8, 4, 128, 64), (32, 1, 64, 3), (1, 40, 256, 600), (8, 8, 128, 1025), (16, 8, 64, 1)])
def test_a_workspace_for_the_largest_step_serves_smaller_ones(dtype, heads, rep, hd, seqs):
    """The bytes that are asked for do not fall as the rows of a step grow: a loop may keep one workspace."""
    view = b.rvq_cache8(n_pages=100, n_kv_heads=heads, head_dim=hd, table_pages=4, n_seqs=seqs)
    last = 0
    for rows in [*range(1, 70), *range(70, 9000, 53), *range(9000, 300000, 9001)]:
        size = b.lib.rvq_cache8_attn_workspace_bytes(view, dtype, rows, heads * rep)
        assert size >= last > -1 and size % 4 == 0, rows
        last = size
    assert last >= 1 << 15
