"""The operators around the 8-bit paged cache at the ends of what their documentation allows: caps, biases, scores and values of any
size, bad blocks between good ones, walks of many blocks, counts of zero, launches that fail."""
import ctypes as C
import math

import numpy as np
import pytest

from tests import cache_reference as R
from tests.test_gpu_cache_ops import HALF, Cache, _attend, _check, _dev, _dt, _filled, _host, _i32

pytestmark = pytest.mark.gpu


# ---- append ----------------------------------------------------------------------------------------------------
def _same_rows_everywhere(batch, heads, n, bad, seed, plant=None):
    """Sequences that all receive the same rows, for more (sequence, head) pairs than one CTA each per block; blocks j of a sequence with
    bad(j) have no valid id.  Compares every sequence with the plain form of one; returns the status word."""
    import torch
    from paper_2506_23431_b200 import binding as B
    g = np.random.default_rng(seed)
    per = -(-n // 64)
    # every block has a size of its own, so that a maximum taken from another block gives another scale
    size = 2.0 ** g.integers(-8, 9, per).repeat(64)[:n, None, None]
    k, v = g.standard_normal((n, heads, 64)) * size, g.standard_normal((n, heads, 64)) / size
    if plant is not None:
        plant(k, v)
    kd, vd = _dev(k, torch.bfloat16), _dev(v, torch.bfloat16)
    codes = torch.full((batch * per, heads, 2, 4096), 0x33, dtype=torch.uint8, device="cuda")
    scales = torch.full((batch * per, heads, 2), 0.25, device="cuda")
    table = g.permutation(batch * per).reshape(batch, per)
    given = table.copy()
    given[:, [j for j in range(per) if bad(j)]] = -1
    given[1::2, [j for j in range(per) if bad(j)]] = batch * per
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.cache_append(kd, vd, _i32([0] * batch), _i32([n] * batch), _i32([0] * batch), _i32(given), codes, scales, n, status=status)
    w_codes, w_scales = np.full((per, heads, 2, 4096), 0x33, np.uint8), np.full((per, heads, 2), 0.25)
    R.append(w_codes, w_scales, np.arange(per)[None], _host(kd), _host(vd), [0], [n], [0])
    for j in range(per):
        if bad(j):
            w_codes[j], w_scales[j] = 0x33, 0.25
    at = torch.from_numpy(table.reshape(-1)).cuda()
    got_c, got_s = codes[at].view(batch, per, heads, 2, 4096), scales[at].view(batch, per, heads, 2)
    assert torch.equal(got_s, _dev(w_scales.astype(np.float32)).expand_as(got_s))
    assert torch.equal(got_c, _dev(w_codes).expand_as(got_c))
    return status.item()


@pytest.mark.parametrize("every", [2, 3])
def test_append_bad_blocks_between_good_ones(every):
    """600 (sequence, head) pairs of 79 blocks, 15 CTAs a pair: a CTA walks five or six blocks, some of them out of range."""
    for seed in range(3):
        assert _same_rows_everywhere(75, 8, 5000, lambda j: j % every == 1, seed) == -1
    assert _same_rows_everywhere(75, 8, 5000, lambda j: j // 15 % every == 1, 3) == -1


def test_append_many_blocks_per_cta():
    """3200 (sequence, head) pairs: two CTAs walk the seven blocks of a pair, one of them with an infinity."""
    def plant(k, v):
        k[200, 3, 7], v[260, 5, 9] = math.inf, -math.inf
        k[64 * 6, :, :] = 0.0
    assert _same_rows_everywhere(200, 16, 64 * 6 + 40, lambda j: False, 5, plant) == 0


# ---- attention: walks of many blocks --------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,batch,kv,blocks", [("bf16", 131, 2, 20), ("bf16", 131, 2, 36), ("bf16", 65, 4, 70), ("fp32", 97, 2, 36), ("fp32", 49, 4, 70)])
def test_attention_of_many_blocks_per_warp(dtype, batch, kv, blocks):
    """So many segments that each is one CTA's: its four warps take the blocks in turn, some tens each, in runs of 16 with tails of every kind.  The sequences
    share the blocks of one (what an entry of the table names is read afresh by every warp) and differ in length."""
    import torch
    from paper_2506_23431_b200 import binding as B
    most = 4 * blocks * 64
    g = np.random.default_rng(blocks)
    c = _filled(53, [64 * 40], kv)                                 # forty blocks, named again and again in another order
    named = np.concatenate([g.permutation(c.table[0, :40]) for _ in range(-(-4 * blocks // 40))])[:4 * blocks]
    table = np.repeat(named[None], batch, axis=0)
    lens = most - (np.arange(batch) * 97) % (most // 2)
    lens[:5] = most, most - 63, most - 64, most - 64 * 4, 64 * 4 * (blocks - 1) + 1
    q = _dev(g.standard_normal((batch, 1, kv * 64)) * 0.7, _dt(dtype))
    out = B.cache_attention(q, c.d_codes, c.d_scales, _i32(table), _i32(np.ones(batch)), _i32(lens), 0.125)
    some = [0, 1, 2, 3, 4, batch // 2, batch - 1]
    _check(out[some], R.attend(_host(q[some]), c.codes, c.scales, table[some], [1] * len(some), lens[some], 0.125), dtype)
    # a window far into the walk
    spans = np.stack([lens - 1000, lens - 3], -1)[:, None]
    out = B.cache_attention(q, c.d_codes, c.d_scales, _i32(table), _i32(np.ones(batch)), _i32(lens), 0.125, spans=_i32(spans))
    _check(out[some], R.attend(_host(q[some]), c.codes, c.scales, table[some], [1] * len(some), lens[some], 0.125, spans[some]), dtype)


# ---- attention: caps of any size -------------------------------------------------------------------------------
def _dense(c, n, kv):
    """Keys and values of the one sequence of a cache, float64 [kv heads, n, 64]."""
    at = c.table[0, :-(-n // 64)]
    val = R.VALUES[c.codes[at]] * np.asarray(c.scales, np.float64)[at][..., None]
    k = val[:, :, 0].reshape(-1, kv, 64, 64).transpose(1, 0, 2, 3).reshape(kv, -1, 64)[:, :n]
    v = val[:, :, 1].reshape(-1, kv, 64, 64).transpose(1, 0, 3, 2).reshape(kv, -1, 64)[:, :n]
    return k, v


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cap", [65.0, 1e3, 1e5, 1e8, 1e20, 9e29])
def test_large_caps(dtype, cap):
    """A cap far above the scores is as good as none: a score's error goes by the score, not by the cap.

    The bound is that of the plain form with 2^-21 |score| in the cap's place: a sum of 64 products (2^-17 + 2^-22 of the summed
    magnitudes), scaling 2^-24 twice, tanh 2^-22 and its product 2^-24, all below 2^-20 |score|."""
    lens, rows, heads, kv = [300], 4, 4, 2
    c = _filled(61, lens, kv)
    q = _dev(np.random.default_rng(62).standard_normal((1, rows, heads * 64)) * 2, _dt(dtype))
    got = _host(_attend(c, q, [rows], lens, None, None, cap)).reshape(rows, heads, 64)
    K, V = _dense(c, 300, kv)
    for r in range(rows):
        for h in range(heads):
            qq, k, v = _host(q)[0, r, h * 64:h * 64 + 64], K[h * kv // heads], V[h * kv // heads]
            s = 0.125 * (k @ qq)
            err = 0.125 * ((2.0 ** -17 + 2.0 ** -22) * (np.abs(k) @ np.abs(qq)) + 2.0 ** -24 * np.abs(qq).max() * np.abs(k).sum(-1)) + 2.0 ** -20 * np.abs(s)
            s = cap * np.tanh(s / cap)
            w = np.exp(s - s.max())
            w /= w.sum()
            ref, mean = w @ v, w @ np.abs(v)
            bound = HALF[dtype] * np.abs(ref) * 1.01 + mean * (2 * err.max() + 2.0 ** -16 + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -22)) + 2.0 ** -40 * np.abs(v).sum(0)
            assert (np.abs(got[r, h] - ref) <= bound).all(), f"{(np.abs(got[r, h] - ref) / bound).max():.1f} times the bound"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_small_caps_and_scores(dtype):
    """A cap at which every score saturates, and scores of nothing."""
    lens = [200]
    c = _filled(63, lens, 2)
    q = _dev(np.random.default_rng(64).standard_normal((1, 3, 128)) * 2, _dt(dtype))
    for cap in (1e-3, 1e-30, 1e-44):
        _check(_attend(c, q, [3], lens, None, None, cap), R.attend(_host(q), c.codes, c.scales, c.table, [3], lens, 0.125, cap=cap), dtype)
        zero = q * 0
        _check(_attend(c, zero, [3], lens, None, None, cap), R.attend(_host(zero), c.codes, c.scales, c.table, [3], lens, 0.125, cap=cap), dtype)


# ---- attention: values, biases and scores of any size ----------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sizes", [[1e-35], [1e-30], [1e33], [1e35], [2e36], [1, 1e30, 1e-20, 1e36, 1], [1e19, 1e20, 1e25, 1e18, 1e22], [1e36, 1e-25, 1e-10, 1e-25, 1e-25]])
def test_values_of_any_size(dtype, sizes):
    """Sums of values are held relative to the row's largest weight: no size of values overflows whose sum over the tokens is a number, and small ones lose nothing.
    One row sees all blocks, the others one block each, of a size of its own.

    The bound is the plain form's, and what underflow adds: the factor of a block's values is off by half of 2^-149 where it is no normal number, its sums of
    64 weights up to 2^15 times codes up to 448 turn that into 2^-120, and the lift of 2^15 goes again: 2^-135, sixteen blocks and the sum's roundings 2^-130; a result
    below the normal range is off by half its spacing, 2^-134 in bf16.  Where a warp has met large values the lift has gone before: 2^-115 for the small blocks' rows."""
    from paper_2506_23431_b200 import binding as B
    n, rows = 1000, 6
    g = np.random.default_rng(67)
    c = Cache(67, 1, 16, 2)
    v = g.standard_normal((n, 2, 64)) * np.resize(sizes, 16).repeat(64)[:n, None, None]
    c.append(g.standard_normal((n, 2, 64)), v, [0], [n], [0], "fp32")
    q = _dev(g.standard_normal((1, rows, 128)), _dt(dtype))
    sp = np.array([[[0, n], [0, 64], [64, 128], [128, 192], [192, 256], [256, 300]]])
    ref, mean, slack = R.attend(_host(q), c.codes, c.scales, c.table, [rows], [n], 0.125, sp)
    bound = HALF[dtype] * np.abs(ref) * 1.01 + slack + mean * (2.0 ** -11 if dtype == "bf16" else 2.0 ** -22) + (2.0 ** -115 if max(sizes) > 1e18 else 2.0 ** -130)
    for batch in (1, 300):                                         # a block for each warp, or four
        got = _host(B.cache_attention(q.expand(batch, -1, -1).contiguous(), c.d_codes, c.d_scales, c.d_table.expand(batch, -1).contiguous(), _i32([rows] * batch), _i32([n] * batch), 0.125,
                                      spans=_i32(np.repeat(sp, batch, 0))))
        for b in (0, batch - 1):
            assert np.isfinite(got[b]).all() and (np.abs(got[b] - ref[0]) <= bound[0]).all(), f"{np.nanmax(np.abs(got[b] - ref[0]) / bound[0]):.1f} times the bound"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bias_on_either_side_of_minus_infinity(dtype):
    """Below -2e38 a bias removes the position; at and above it is a number like others: a row that has the same everywhere takes the values' mean (its scores are
    far below the bias's last place)."""
    lens, rows = [200], 2
    c = _filled(71, lens, 2)
    q = _dev(np.random.default_rng(72).standard_normal((1, rows, 128)), _dt(dtype))
    _, V = _dense(c, 200, 2)
    for low, gone in ((-2.2e38, True), (-2.01e38, True), (-2e38, False), (-1.9e38, False)):
        bias = np.zeros((2, 3), np.float32)
        bias[0] = low
        got = _host(_attend(c, q, [rows], lens, None, bias, 0.0))
        every = R.attend(_host(q), c.codes, c.scales, c.table, [rows], lens, 0.125)
        _check(_dev(got[..., 64:]), tuple(w[..., 64:] for w in every), dtype)
        if gone:
            assert not got[..., :64].any()
        else:
            ref, mean = V[0].mean(0), np.abs(V[0]).mean(0)
            assert (np.abs(got[..., :64] - ref) <= HALF[dtype] * np.abs(ref) * 1.01 + 2.0 ** -16 * mean).all()
        bias[0] = [0.0, low, 0.0]                                  # one position removed: it weighs nothing either way
        got = _host(_attend(c, q, [rows], lens, None, bias, 0.0))
        K, _ = _dense(c, 200, 2)
        s = 0.125 * np.einsum("rd,kd->rk", _host(q)[0, :, :64], K[0])
        s[:, 198] = -math.inf
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        assert np.abs(got[0, :, :64] - w @ V[0]).max() <= 2.0 ** -6 * np.abs(V[0]).max()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [1e5, 4e6, 1.3e7, 3e7, 1e8, 7e9, 1e15, 1e25, 1e35])
@pytest.mark.parametrize("mod", ["plain", "bias", "cap"])
def test_scores_of_any_size(dtype, size, mod):
    """Scores so large that neighbouring numbers lie further apart than a weight's range: the largest takes all, equal ones share.

    Key p is a multiple of one direction: the chosen positions have the largest score, all others at most 0.9 of it (or, below zero, 1.1), which is a weight of nothing
    at these sizes; equal keys have equal codes, so equal scores.  The result is the mean of the chosen values: the output's rounding and 2^-16 for its sums."""
    from paper_2506_23431_b200 import binding as B
    g = np.random.default_rng(int(math.log2(size)))
    n, rows = 700, 3
    for sign in (1, -1):
        for chosen in ([5], [650], [3, 64, 200, 699]):
            k = np.empty((n, 1, 64))
            k[:] = (np.round(g.random((n, 1, 1)) * 8) / 16 if sign > 0 else 1.25 + np.round(g.random((n, 1, 1)) * 4) / 8)      # codes hold these exactly
            k[chosen] = 1.0
            c = Cache(73, 1, 11, 1)
            c.append(k, g.standard_normal((n, 1, 64)), [0], [n], [0], "fp32")
            q = _dev(np.full((1, rows, 64), sign * size / 64 * 8 * (1 + g.random())), _dt(dtype))
            bias = np.zeros((1, 4), np.float32) if mod == "bias" else None
            got = _host(B.cache_attention(q, c.d_codes, c.d_scales, c.d_table, _i32([rows]), _i32([n]), 0.125, bias=None if bias is None else _dev(bias),
                                          softcap=9e29 if mod == "cap" and size < 1e28 else 0.0))
            K, V = _dense(c, n, 1)
            assert (K[0][chosen] == 1).all() and (np.delete(K[0], chosen, 0).max() <= 0.9 if sign > 0 else np.delete(K[0], chosen, 0).min() >= 1.1)
            ref, mean = V[0][chosen].mean(0), np.abs(V[0][chosen]).mean(0)
            assert (np.abs(got - ref) <= HALF[dtype] * np.abs(ref) * 1.01 + 2.0 ** -16 * mean).all(), (sign, chosen, got[0, 0, :4], ref[:4])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_queries_with_a_large_scale(dtype):
    """Queries near the end of the range over keys near the other, and a scale above one: the scores are ordinary numbers."""
    from paper_2506_23431_b200 import binding as B
    g = np.random.default_rng(79)
    lens, rows = [200], 3
    for size, scale in ((1e38, 4.0), (1e37, 30.0), (1e30, 1e4), (1e-30, 1e4)):
        c = Cache(79, 1, 5, 2)
        c.append(g.standard_normal((200, 2, 64)) / size / scale * 0.2, g.standard_normal((200, 2, 64)), [0], lens, [0], "fp32")
        q = _dev(np.clip(g.standard_normal((1, rows, 128)), -3, 3) * size, _dt(dtype))
        for cap, bias in ((0.0, None), (0.0, np.zeros((2, 3), np.float32)), (20.0, None)):
            got = B.cache_attention(q, c.d_codes, c.d_scales, c.d_table, _i32([rows]), _i32(lens), scale, softcap=cap, bias=None if bias is None else _dev(bias))
            _check(got, R.attend(_host(q), c.codes, c.scales, c.table, [rows], lens, scale, bias=bias, cap=cap), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size,scale,cap", [(1e20, 1e-30, 9e29), (1e30, 1e-25, 1e25), (1e-30, 1e25, 1e-30), (1e-20, 1e29, 1e29), (1.0, 1e-38, 100.0), (1.0, 1e-38, 50.0)])
def test_scales_far_from_their_caps(dtype, size, scale, cap):
    """The quotient of scale and cap may be no number of 32 bits: the scores are.  Large caps are as good as none (the plain form without one, whose own term of the bound, 2^-21 of
    a score, is doubled by tanh); a tiny one leaves scores of nothing, and every position weighs the same."""
    from paper_2506_23431_b200 import binding as B
    g = np.random.default_rng(97)
    lens, rows = [200], 3
    c = Cache(97, 1, 5, 2)
    c.append(np.clip(g.standard_normal((200, 2, 64)) / size / scale * 0.2, -3e38, 3e38), g.standard_normal((200, 2, 64)), [0], lens, [0], "fp32")
    q = _dev(np.clip(g.standard_normal((1, rows, 128)), -3, 3) * size, _dt(dtype))
    got = B.cache_attention(q, c.d_codes, c.d_scales, c.d_table, _i32([rows]), _i32(lens), scale, softcap=cap)
    if cap < 1e-20:
        ref = np.concatenate([v.mean(0) for v in _dense(c, 200, 2)[1]])
        assert (np.abs(_host(got)[0] - ref) <= HALF[dtype] * np.abs(ref) * 1.01 + 2.0 ** -16 * np.abs(_dense(c, 200, 2)[1]).mean((0, 1)).max()).all()
    elif cap <= 1e3:
        _check(got, R.attend(_host(q), c.codes, c.scales, c.table, [rows], lens, scale, cap=cap), dtype)
    else:
        s = scale * np.einsum("rhd,hkd->rhk", _host(q)[0].reshape(rows, 2, 64), _dense(c, 200, 2)[0])
        assert np.abs(s).max() ** 3 / cap ** 2 < 2.0 ** -20
        out, mean, slack = R.attend(_host(q), c.codes, c.scales, c.table, [rows], lens, scale)
        _check(got, (out, mean, 2 * slack), dtype)


# ---- counts of zero, sizes at the end of 32 bits, launches that fail -------------------------------------------
def test_append_counts_that_its_sizes_do_not_allow():
    """No rows, or no new tokens allowed: a sequence that has some all the same is reported, as with any other bound."""
    import torch
    from paper_2506_23431_b200 import binding as B
    c = _filled(83, [70], 2)
    before = c.d_codes.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for rows, n, most, want in ((5, 0, 0, 0), (0, 0, 0, 0), (0, 0, 7, 0), (5, 3, 0, -1), (0, 3, 7, -1), (0, 3, 0, -1)):
        status.zero_()
        k = torch.ones(rows, 2, 64, dtype=torch.bfloat16, device="cuda")
        B.cache_append(k, k, _i32([0]), _i32([n]), _i32([70]), c.d_table, c.d_codes, c.d_scales, most, status=status)
        assert status.item() == want, (rows, n, most)
    assert torch.equal(c.d_codes, before)


def test_rotary_of_the_most_tokens():
    """2^31 - 1 tokens of one head of two dims: the same as a call on a few of them."""
    import torch
    from paper_2506_23431_b200 import binding as B
    n = (1 << 31) - 1
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 18 GB")
    x = torch.randn(1, 1, 2, device="cuda").bfloat16().expand(n, 1, 2)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    turns = _dev(np.array([0.0123456789]))
    out = torch.empty(n, 1, 2, dtype=torch.bfloat16, device="cuda")
    B.rotary(x, pos, turns, out=out)
    for at in (0, 1 << 20, (1 << 30) - 500, n - 1000):
        few = slice(at, at + 1000)
        assert torch.equal(out[few], B.rotary(x[few], pos[few], turns))


def test_rotary_refuses_more_tokens_than_32_bits_hold():
    """Not the remainder modulo 2^32: nothing is written."""
    import torch
    from paper_2506_23431_b200 import binding as B
    n = (1 << 32) + 3
    x = torch.ones(1, 1, 2, device="cuda").bfloat16().expand(n, 1, 2)
    out = torch.zeros(1, 1, 2, device="cuda").bfloat16()
    with pytest.raises(ValueError, match="32 bits"):
        B.rotary(x, torch.zeros(1, dtype=torch.int32, device="cuda").expand(n), _dev(np.array([0.1])), out=out.expand(n, 1, 2))
    assert not out.any()


def test_a_failed_launch_leaves_no_error_behind():
    """A launch on the default stream while a stream that waits for it is captured is refused by CUDA; the caller's next check of its own must not see that."""
    import torch
    from paper_2506_23431_b200 import binding as B
    x = torch.randn(4, 3, 64, device="cuda").bfloat16()
    pos, turns, out = _i32([1, 2, 3, 4]), _dev(B.rotary_turns(64)[0]), torch.zeros(4, 3, 64, device="cuda").bfloat16()
    c = _filled(89, [70], 2)
    q, n, le, one, zero = torch.randn(1, 2, 128, device="cuda").bfloat16(), _i32([2]), _i32([70]), _i32([1]), _i32([0])
    kv = torch.randn(1, 2, 64, device="cuda").bfloat16()
    res = torch.empty_like(q)
    want = B.cache_attention(q, c.d_codes, c.d_scales, c.d_table, n, le, 0.125)
    torch.cuda.synchronize()
    rt = C.CDLL("libcudart.so.12")
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    calls = [lambda: B._lib.pd_rotary(1, 4, 3, 64, 64, 0, 0, p(x), 192, 64, p(pos), p(turns), 1.0, p(out), 192, 64, None),
             lambda: B._lib.pd_cache_append(1, 1, 2, c.codes.shape[0], c.d_table.shape[1], 1, 1, p(kv), 128, p(kv), 128, p(zero), p(one), p(le), p(c.d_table), p(c.d_codes), p(c.d_scales),
                                            None, None),
             lambda: B._lib.pd_cache_attention(1, 1, 2, 2, 2, c.codes.shape[0], c.d_table.shape[1], 70, 0.125, 0.0, p(q), 128, p(c.d_codes), p(c.d_scales), p(c.d_table), p(n), p(le), None,
                                               None, 0, p(res), None, 0, None, None)]
    for call in calls:
        s, graph = C.c_void_p(), C.c_void_p()
        assert rt.cudaStreamCreate(C.byref(s)) == 0
        assert rt.cudaStreamBeginCapture(s, 2) == 0                          # 2: relaxed
        status, left = call(), rt.cudaPeekAtLastError()
        rt.cudaStreamEndCapture(s, C.byref(graph))
        rt.cudaGetLastError()
        assert rt.cudaStreamDestroy(s) == 0
        assert status == -5 and left == 0
    assert torch.equal(B.cache_attention(q, c.d_codes, c.d_scales, c.d_table, n, le, 0.125), want)
