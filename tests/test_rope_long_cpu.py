"""Rotary positions stretched by parts (YaRN) where the original context is long for the base: even the last pair turns more than once in
it, so none is stretched in full.  Against the definition pair by pair: a pair's share of the stretch rises linearly in its number, from the
last that turns 32 times to the first that turns once."""
import math

import numpy as np
import pytest

from paper_2509_01229_amd import api
from oracle import attention_oracle as A


def _pair_frequencies(table):
    row = table[1].astype(np.float64)
    half = row.size // 2
    return np.arctan2(row[half:], row[:half])  # (position 1; below pi)


@pytest.mark.parametrize("rot,original", [(64, 65536), (128, 65536), (128, 131072), (16, 32768), (128, 1 << 20), (64, 4096), (128, 2048)])
@pytest.mark.parametrize("factor", [4.0, 16.0])
def test_yarn_ramp(rot, original, factor, base=10000.0):
    got = _pair_frequencies(api.attn_rope_table(2, rot, base, "yarn", factor, original))
    i = np.arange(rot // 2)
    plain = base ** (-2.0 * i / rot)
    turns = original * plain / (2 * math.pi)
    number = lambda t: rot * math.log(original / (2 * math.pi * t)) / (2 * math.log(base))  # of the pair that turns t times
    first, last = math.floor(number(32)), math.ceil(number(1))
    assert 0 <= first < last <= rot - 1
    share = np.clip((i - first) / (last - first), 0, 1)
    want = plain * (1 - share + share / factor)
    # (sines and cosines rounded to 2^-24 of themselves)
    assert np.abs(got / want - 1).max() < 2.0 ** -22
    # said without the ramp: all of the stretch where a pair turns once or less, none of it where 32 times (one pair's step of the ramp less)
    stretched = (1 - got / plain) / (1 - 1 / factor)
    assert (stretched[turns > base ** (2 / rot)] < 0.999).all() and np.allclose(stretched[turns <= 1], 1, atol=1e-5)
    assert np.allclose(stretched[turns >= 32 * base ** (2 / rot)], 0, atol=1e-5)


@pytest.mark.parametrize("rot,original", [(64, 65536), (128, 131072)])
def test_yarn_table_against_the_oracle(rot, original):
    got = api.attn_rope_table(500, rot, 10000.0, "yarn", 4.0, original)
    assert np.abs(got - A.rope_table(500, rot, 10000.0, "yarn", 4.0, original)).max() <= 2.0 ** -23 + 1e-12  # (below 1.2)


def test_last_pair_of_a_long_context():
    # the pairs that turn 32 times and once have the numbers 20.1 and 32.1: pair 31 (1.39 turns) has 11/13 of the stretch
    f = 1e4 ** (-62 / 64)
    assert 65536 * f / (2 * math.pi) > 1
    got = _pair_frequencies(api.attn_rope_table(2, 64, 1e4, "yarn", 4.0, 65536))[-1]
    assert abs(got / f - (1 - 11 / 13 * 0.75)) < 2.0 ** -22
