"""Host side of the operators around the 8-bit paged cache at the ends of what their documentation allows (no GPU is touched)."""
import math

import numpy as np
import pytest

from paper_2506_23431_b200 import binding as B


@pytest.mark.parametrize("original,fast,slow", [(4, 32.0, 1.0), (6, 32.0, 1.0), (100, 64.0, 16.5), (1, 1e-3, 1e-4), (7, 32.0, 1.0), (4096, 32.0, 1.0), (4096, 1.0, 1.0), (4, 1.0, 1.0), (1 << 20, 1e9, 1e8)])
def test_frequencies_by_parts_at_the_first_pair(original, fast, slow):
    """Every pair that makes at most `slow` turns over the original context is divided, the first one too; every one that makes at least `fast` is not."""
    factor = 8.0
    turns, _ = B.rotary_turns(64, 10000.0, B.PD_ROTARY_BY_PARTS, factor, original, fast, slow)
    base = 10000.0 ** (-np.arange(32) / 32) / (2 * math.pi)
    made = base * original
    few, many = (made <= slow) & (made < fast), made >= fast
    assert np.allclose(turns[few], base[few] / factor, rtol=1e-14) and np.allclose(turns[many], base[many], rtol=1e-14)
    assert ((turns <= base * (1 + 1e-14)) & (turns >= base / factor * (1 - 1e-14))).all()


def test_binding_refuses_sizes_beyond_32_bits():
    """A size that the C call would take modulo 2^32 (and silently do something else) is refused before anything else is looked at."""
    import torch
    q, k, i32 = torch.zeros(1, 2, 128), torch.zeros(4, 2, 64), torch.zeros(1, dtype=torch.int32)
    codes, scales, table = torch.zeros(3, 2, 2, 4096, dtype=torch.uint8), torch.ones(3, 2, 2), torch.zeros(1, 3, dtype=torch.int32)
    for wide in ((1 << 32) + 100, 1 << 32, 1 << 31, -(1 << 32) + 100):
        with pytest.raises(ValueError, match="32 bits"):
            B.cache_attention(q, codes, scales, table, i32, i32, 0.125, max_len=wide)
        with pytest.raises(ValueError, match="32 bits"):
            B.cache_append(k, k, i32, i32, i32, table, codes, scales, wide)
        with pytest.raises(ValueError, match="32 bits"):
            B.cache_attention_scratch_bytes(1, 1, 2, 2, 2, wide)
        with pytest.raises(ValueError, match="32 bits"):
            B.rotary_turns(64, 10000.0, B.PD_ROTARY_BY_PARTS, 4.0, wide)


def test_append_of_nothing_looks_at_nothing_else():
    """No rows, or no tokens allowed: strides, alignment and missing tensors are no error, with and without a status word (whose call checks counts only)."""
    P = 1 << 20            # an address that is never followed: every call here returns before its launch
    for rows, most in ((0, 5), (5, 0)):
        for status in (None, P):
            assert B._lib.pd_cache_append(1, 2, 3, 8, 4, rows, most, P + 2, 0, None, 1, None, P, P, None, P + 1, None, status, None) == 0
        assert B._lib.pd_cache_append(1, 2, 3, 8, 4, rows, most, P + 2, 0, None, 1, P, P, P, None, P + 1, None, P + 2, None) == -1
