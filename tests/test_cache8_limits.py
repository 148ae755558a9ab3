"""What the paged 8-bit cache promises at the ends of its range, as far as no GPU is needed for it."""
from paper_2410_15704_amd import build


def test_attention_is_compiled_with_nan():
    """A NaN code reaches the result of the rows that see it: nothing that handles one may be compiled as if there were none."""
    for name in ("rvq_cache8.hip", "rvq_cache8_attn.hip", "rvq_cache8_chunk.hip", "rvq_rope.hip"):
        flags = build.FLAGS + build.EXTRA.get(name, [])
        assert not [f for f in flags if f in ("-fno-honor-nans", "-ffast-math", "-ffinite-math-only", "-fno-honor-infinities")], name
