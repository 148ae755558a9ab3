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
