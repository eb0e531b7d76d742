"""The roundings that a sum of exponentials over the vocabulary passes, counted as
lm_ref's bound of 600 u for them has it (CPU only)."""
import pytest

import test_gpu_vocab as V


def roundings(words, bf, grown=None):
    """In u: additions of the slot, of the join's lane (every 64th slot) and of its
    64 lanes; exponentials of 9 u beyond the term's own, of which `grown` (None:
    all) where the largest z grows between groups of eight of a lane's slots."""
    slots = -(-words // (128 if bf else 64))
    lane = -(-slots // 64)
    groups = -(-lane // 8)
    additions = (32 if bf else 16) + 2 + lane + 64
    factors = 3 + (groups if grown is None else min(grown, groups))
    return additions + 9 * factors


@pytest.mark.parametrize("bf", [False, True])
def test_sums_over_the_vocabulary_are_within_the_bound(bf):
    sizes = [c for _, c, _ in V.SHAPES] + [128000, 262444, 450000, 600001, 900000]
    assert max(roundings(c, bf) for c in sizes) <= 600
    assert roundings(1 << 20, bf, grown=25) <= 600
