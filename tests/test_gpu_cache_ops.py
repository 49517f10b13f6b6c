"""The operators around the 8-bit paged cache on the GPU, against their plain 64-bit forms: rotary positions, the append of keys
and values, attention over the cache, and the three one after the other."""
import math

import numpy as np
import pytest

from tests import cache_reference as R

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}          # half a step of the type, relative


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.array(a, order="C")).cuda()
    return t if dtype is None else t.to(dtype)


def _i32(a):
    return _dev(np.asarray(a, np.int32))


def _host(t):
    return t.detach().double().cpu().numpy()


# ---- rotary ----------------------------------------------------------------------------------------------------
ROTARY = [
    # dtype, tokens, heads, d_head, rot, interleaved, inverse, far
    ("bf16", 1, 1, 64, 64, False, False, 100), ("bf16", 7, 24, 64, 64, False, False, 4096), ("bf16", 5000, 6, 64, 64, True, False, 1 << 20),
    ("bf16", 33, 5, 64, 48, False, True, 1 << 20), ("bf16", 33, 5, 64, 40, True, True, 4096), ("bf16", 9, 3, 64, 2, False, False, 4096), ("bf16", 9, 3, 64, 20, False, False, 4096),
    ("bf16", 17, 2, 128, 32, True, False, 1 << 22), ("bf16", 3, 2, 256, 256, False, False, 4096), ("bf16", 11, 3, 10, 6, True, False, 50),
    ("bf16", 4801, 24, 64, 20, False, False, 4096), ("fp32", 4801, 20, 64, 10, True, True, 4096), ("bf16", 700, 3, 64, 56, False, False, 4096), ("bf16", 6000, 5, 72, 18, True, False, 4096),
    ("bf16", 900, 33, 64, 56, False, True, 4096), ("bf16", 40, 3, 68, 24, True, False, 4096), ("fp32", 700, 9, 64, 60, False, False, 4096), ("fp32", 50, 7, 62, 20, True, False, 4096),
    ("fp32", 1, 12, 64, 64, True, False, 100), ("fp32", 1201, 7, 64, 64, False, True, 1 << 30), ("fp32", 77, 5, 64, 40, True, False, 1 << 20), ("fp32", 13, 4, 80, 22, False, False, 4096),
]


def _rotary_inputs(dtype, tokens, heads, dh, rot, far, seed=0):
    from paper_2506_23431_b200 import binding as B
    g = np.random.default_rng(seed + tokens)
    x = _dev(g.standard_normal((tokens, heads, dh)), _dt(dtype))
    pos = g.integers(-far // 2, far, tokens)
    pos[0] = far
    turns, amp = B.rotary_turns(rot, 10000.0, B.PD_ROTARY_BY_PARTS, 8.0, 512)
    return x, pos.astype(np.int32), turns, amp


def _rotary_bound(x, pos, turns, amp, rot, interleaved, dtype, ref):
    """Half a step of the result, and fp32 inside: the angle off by pi 2^-24 (its fraction rounded to fp32) and 2 pi 2^-53 of the turns made, sine and cosine by
    2^-23, three roundings by 2^-24 each - 2^-21 and the far positions' share of |x_a| + |x_b| in all."""
    ax = np.abs(x)
    pair = ax.copy()
    ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    both = amp * (ax[..., ia] + ax[..., ib]) * (2.0 ** -21 + 2 * math.pi * 2.0 ** -52 * np.abs(pos.astype(np.float64)[:, None] * turns)[:, None])
    pair[:] = 0
    pair[..., ia] = pair[..., ib] = both
    return HALF[dtype] * np.abs(ref) * 1.001 + pair


@pytest.mark.parametrize("dtype,tokens,heads,dh,rot,interleaved,inverse,far", ROTARY)
def test_rotary_against_plain_form(dtype, tokens, heads, dh, rot, interleaved, inverse, far):
    from paper_2506_23431_b200 import binding as B
    x, pos, turns, amp = _rotary_inputs(dtype, tokens, heads, dh, rot, far)
    kept = x.clone()
    y = B.rotary(x, _i32(pos), _dev(turns), amp, interleaved=interleaved, inverse=inverse)
    ref = R.rotate(_host(x), pos, turns, amp, interleaved, inverse)
    assert (np.abs(_host(y) - ref) <= _rotary_bound(_host(x), pos, turns, amp, rot, interleaved, dtype, ref)).all()
    assert (x == kept).all() and (y[..., rot:] == x[..., rot:]).all()
    # in place, the same bits
    z = B.rotary(x, _i32(pos), _dev(turns), amp, interleaved=interleaved, inverse=inverse, out=x)
    assert z.data_ptr() == x.data_ptr() and (z == y).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("offset,width,pad", [(0, 3 * 64 * 4, 0), (64, 64 * 9, 0), (3, 64 * 9 + 5, 0), (8, 64 * 9 + 16, 1)])
def test_rotary_strides_and_alignment(dtype, offset, width, pad):
    """Heads inside fused rows, at any offset and row length; an output whose heads lie apart, whose gaps stay as they were."""
    import torch
    from paper_2506_23431_b200 import binding as B
    tokens, heads = 19, 4
    g = np.random.default_rng(5)
    rows = _dev(g.standard_normal((tokens, width)), _dt(dtype))
    x = rows[:, offset:offset + heads * 64].unflatten(1, (heads, 64))
    pos = g.integers(0, 1000, tokens).astype(np.int32)
    turns, _ = B.rotary_turns(64)
    want = B.rotary(x.contiguous(), _i32(pos), _dev(turns))
    room = torch.full((tokens, heads, 64 + 8 * pad), -7.0, dtype=x.dtype, device="cuda")
    out = B.rotary(x, _i32(pos), _dev(turns), out=room[..., :64])
    assert (out == want).all() and (room[..., 64:] == -7).all()
    # [heads, tokens, dims] in memory: tokens inside heads
    t = torch.empty(heads, tokens, 64, dtype=x.dtype, device="cuda").transpose(0, 1)
    assert (B.rotary(x, _i32(pos), _dev(turns), out=t) == want).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_backward(interleaved):
    """The inverse is the gradient: against autograd of the formula in 64 bits, and against differences of the map itself."""
    import torch
    from paper_2506_23431_b200 import binding as B
    x, pos, turns, amp = _rotary_inputs("fp32", 9, 3, 64, 40, 5000, seed=3)
    gy = torch.randn(9, 3, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    gx = B.rotary(gy, _i32(pos), _dev(turns), amp, interleaved=interleaved, inverse=True)
    xd = x.double().requires_grad_()
    ang = 2 * math.pi * (torch.from_numpy(pos).double()[:, None] * torch.from_numpy(turns)).cuda()
    c, s = (ang.cos() * amp)[:, None], (ang.sin() * amp)[:, None]
    a, b = (xd[..., 0:40:2], xd[..., 1:40:2]) if interleaved else (xd[..., :20], xd[..., 20:40])
    ya, yb = a * c - b * s, a * s + b * c
    y = torch.cat([torch.stack([ya, yb], -1).flatten(-2) if interleaved else torch.cat([ya, yb], -1), xd[..., 40:]], -1)
    (y * gy.double()).sum().backward()
    assert (gx.double() - xd.grad).abs().max() <= 2.0 ** -20 * amp * 2 * gy.abs().max().double()
    f = lambda v: (B.rotary(v, _i32(pos), _dev(turns), amp, interleaved=interleaved).double() * gy.double()).sum()  # noqa: E731
    step = torch.randn(9, 3, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    # a linear map: no error of a difference but rounding, 2^-20 of the summed magnitudes
    assert abs((f(x + step) - f(x - step)) / 2 - (gx.double() * step.double()).sum()) <= 2.0 ** -20 * 4 * 2 * amp * (gy.abs() * (x.abs() + step.abs())).sum().item() * 2


# ---- append ----------------------------------------------------------------------------------------------------
class Cache:
    """A cache on the device and its plain copy, filled with stale bytes; blocks of a sequence in mixed order."""

    def __init__(self, seed, batch, per_seq, heads, spare=3):
        g = np.random.default_rng(seed)
        n = batch * per_seq + spare
        self.heads, self.per_seq = heads, per_seq
        self.codes = g.integers(0, 256, (n, heads, 2, 4096)).astype(np.uint8)
        self.scales = 2.0 ** g.integers(-5, 5, (n, heads, 2))
        self.table = g.permutation(n)[:batch * per_seq].reshape(batch, per_seq)
        self.d_codes, self.d_scales, self.d_table = _dev(self.codes), _dev(self.scales.astype(np.float32)), _i32(self.table)

    def append(self, k, v, row_start, n_new, pos_start, dtype, max_new=None, fused=False, status=None):
        import torch
        from paper_2506_23431_b200 import binding as B
        kd, vd = _dev(k, _dt(dtype)), _dev(v, _dt(dtype))
        R.append(self.codes, self.scales, self.table, _host(kd), _host(vd), row_start, n_new, pos_start)
        if fused:
            rows = torch.cat([torch.zeros_like(kd), kd, vd], 1)
            kd, vd = rows[:, self.heads:2 * self.heads], rows[:, 2 * self.heads:]
        B.cache_append(kd, vd, _i32(row_start), _i32(n_new), _i32(pos_start), self.d_table, self.d_codes, self.d_scales, int(max(n_new)) if max_new is None else max_new, status=status)

    def same(self):
        got = self.d_codes.cpu().numpy()
        nan = (got & 0x7F == 0x7F) & (self.codes & 0x7F == 0x7F)            # a code of no number may carry either sign
        bad = (got != self.codes) & ~nan
        assert not bad.any(), f"{bad.sum()} codes differ, first at {np.argwhere(bad)[0]}"
        assert (self.d_scales.cpu().numpy() == self.scales).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("counts,starts", [([1], [0]), ([1, 1, 1], [0, 63, 64]), ([2, 0, 5], [63, 7, 60]), ([64, 65, 128], [0, 0, 64]), ([200, 3, 0, 77], [13, 126, 0, 1]), ([63, 130], [1, 62])])
def test_append_against_plain_form(dtype, fused, counts, starts):
    g = np.random.default_rng(sum(counts))
    c = Cache(1, len(counts), -(-max(n + s for n, s in zip(counts, starts)) // 64) + 1, 3)
    rows = sum(counts) + 4
    k, v = g.standard_normal((rows, 3, 64)) * 3, g.standard_normal((rows, 3, 64)) * 2.0 ** g.integers(-6, 9, (rows, 1, 1))
    order = g.permutation(len(counts))                       # sequences' rows in another order than the sequences
    row_start = np.zeros(len(counts), int)
    at = 2
    for b in order:
        row_start[b], at = at, at + counts[b]
    # valid codes where older tokens are, else the blocks' stale bytes
    for b, s in enumerate(starts):
        if s:
            c.append(g.standard_normal((s, 3, 64)), g.standard_normal((s, 3, 64)), [0] * len(counts), [s if i == b else 0 for i in range(len(counts))], [0] * len(counts), dtype)
    c.append(k, v, row_start, counts, starts, dtype, max_new=max(counts) + 100, fused=fused)
    c.same()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_token_by_token_with_growing_scales(dtype):
    """Every token larger than the ones before: the block's codes move to a new scale again and again, down into the format's subnormals."""
    g = np.random.default_rng(7)
    c = Cache(2, 2, 3, 2)
    for p in range(140):
        size = 2.0 ** (p % 64 / 3)
        c.append(g.standard_normal((2, 2, 64)) * size, g.standard_normal((2, 2, 64)) * (size if p % 5 else size * 1e4), [0, 1], [1, 1 if p < 100 else 0], [p, p], dtype)
    c.same()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_of_extremes(dtype):
    g = np.random.default_rng(8)
    c = Cache(3, 6, 2, 2)
    big = 3.3e38
    k, v = g.standard_normal((6, 70, 2, 64)), g.standard_normal((6, 70, 2, 64))
    k[0], v[0] = 0.0, -0.0                                       # nothing but zeros
    k[1, 3, 0, 5], v[1, 66, 1, 9] = np.nan, np.nan
    k[2, 0, 0, 0], v[2, 5, 1, 63], k[2, 69, 1, 1] = np.inf, -np.inf, np.inf
    k[3] *= 1e-39                                                # below the smallest normal number
    v[3] *= 1e-36
    k[4], v[4, 7] = big, -big
    k[5, :, 0], v[5, :, 0], v[5, :, 1] = 448.0, 450.0, 224.0     # on the border of a power of two, and just over it
    for _ in range(2):                                           # the second time over older tokens, from position 40 on
        p = 0 if _ == 0 else 40
        n = 70 - p if _ else 70
        rows = np.concatenate([a[70 - n:] for a in k]), np.concatenate([a[70 - n:] for a in v])
        c.append(*rows, np.arange(6) * n, [n] * 6, [p] * 6, dtype)
        c.same()


def test_append_bad_input_touches_nothing_else():
    import torch
    g = np.random.default_rng(9)
    c = Cache(4, 7, 2, 2)
    c.append(g.standard_normal((70, 2, 64)), g.standard_normal((70, 2, 64)), [0] * 7, [10, 0, 0, 0, 0, 0, 0], [0] * 7, "bf16")
    k, v = g.standard_normal((40, 2, 64)), g.standard_normal((40, 2, 64))
    good_row, good_n, good_pos = [0, 3, 0, 0, 0, 0, 0], [5, 30, 0, 0, 0, 0, 0], [10, 50, 0, 0, 0, 0, 0]
    R.append(c.codes, c.scales, c.table, _host(_dev(k, torch.bfloat16)), _host(_dev(v, torch.bfloat16)), good_row, good_n, good_pos)
    # rows before the first, rows behind the last, a negative position, more than max_new; a table entry out of range
    row, n, pos = list(good_row), list(good_n), list(good_pos)
    row[2], n[2] = -1, 3
    row[3], n[3] = 38, 3
    n[4], pos[4] = 4, -2
    n[5] = 31
    n[6] = 3
    table = c.table.copy()
    table[6] = [-1, 1 << 30]
    from paper_2506_23431_b200 import binding as B
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.cache_append(_dev(k, torch.bfloat16), _dev(v, torch.bfloat16), _i32(row), _i32(n), _i32(pos), _i32(table), c.d_codes, c.d_scales, 30, status=status)
    c.same()
    assert status.item() == -1
    # the tokens behind the end of the table are dropped, those before it are written
    status.zero_()
    R.append(c.codes, c.scales, c.table, _host(_dev(k, torch.bfloat16)), _host(_dev(v, torch.bfloat16)), [0] * 7, [8, 0, 0, 0, 0, 0, 0], [120, 0, 0, 0, 0, 0, 0])
    B.cache_append(_dev(k, torch.bfloat16), _dev(v, torch.bfloat16), _i32([0] * 7), _i32([20, 0, 0, 0, 0, 0, 0]), _i32([120, 0, 0, 0, 0, 0, 0]), c.d_table, c.d_codes, c.d_scales, 30,
                   status=status)
    c.same()
    assert status.item() == -1


# ---- attention -------------------------------------------------------------------------------------------------
def _filled(seed, lens, kv_heads, extra_blocks=1):
    """A cache of these lengths; what stands behind a sequence's last token is no number."""
    g = np.random.default_rng(seed)
    c = Cache(seed, len(lens), max(1, -(-max(lens) // 64)) + extra_blocks, kv_heads)
    rows = sum(lens) + 1
    k = g.standard_normal((rows, kv_heads, 64)) * (0.5 + 2 * g.random((1, kv_heads, 64)))
    v = g.standard_normal((rows, kv_heads, 64)) * 2.0 ** g.integers(-3, 4, (rows, 1, 1))
    c.codes[:], c.d_codes[:] = 0x7F, 0x7F
    c.append(k, v, np.concatenate([[0], np.cumsum(lens)])[:-1], lens, [0] * len(lens), "fp32")
    return c


def _check(out, want, dtype):
    ref, mean, slack = want
    got = _host(out)
    # a weight in f16 (10 bits behind the point: spacing 2^-10, at most half of it off) is off by 2^-11, in two parts by 2^-11 of 2^-11
    w_eps = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22
    bound = HALF[dtype] * np.abs(ref) * 1.01 + slack + mean * w_eps + 2.0 ** -120
    assert (np.isnan(got) == np.isnan(ref)).all()
    bad = np.abs(got - ref) > bound
    assert not bad.any(), f"{bad.sum()} of {bad.size} beyond the bound, worst {np.nanmax(np.abs(got - ref) / bound):.2f} times, first at {np.argwhere(bad)[0]}"


def _spans(kind, g, lens, n_rows, rows):
    if kind == "none":
        return None
    sp = np.zeros((len(lens), rows, 2), np.int64)
    for b, n in enumerate(lens):
        for r in range(rows):
            end = n - n_rows[b] + 1 + r
            sp[b, r] = {"causal": (0, end), "window": (end - 70, end), "document": sorted(g.integers(-5, n + 6, 2)), "beyond": (-100, 1 << 30), "empty": (n // 2, n // 2) if r % 3 else (0, n),
                        "one": (max(end - 1, 0), end)}[kind]
    return sp


ATTEND = [
    # dtype, heads, kv heads, rows, lens, spans, distances of the bias (0: none), cap
    ("bf16", 1, 1, 1, [1], "none", 0, 0.0),
    ("bf16", 2, 2, 3, [64, 0, 65, 1, 63, 128], "none", 0, 0.0),
    ("bf16", 12, 12, 8, [777], "none", 0, 0.0),
    ("bf16", 3, 1, 5, [200, 300], "causal", 0, 0.0),
    ("bf16", 8, 2, 9, [130, 7, 700], "window", 0, 30.0),
    ("bf16", 4, 4, 16, [260, 31], "document", 32, 0.0),
    ("bf16", 2, 1, 64, [190, 77], "causal", 512, 0.0),
    ("bf16", 4, 2, 17, [500, 100], "empty", 5, 5.0),
    ("bf16", 16, 1, 4, [333], "one", 1, 0.0),
    ("bf16", 2, 2, 33, [129, 64, 1000], "beyond", 0, 2.0),
    ("bf16", 1, 1, 1, [5000], "none", 0, 0.0),
    ("bf16", 6, 2, 2, [9001, 40], "window", 200, 0.0),
    ("fp32", 1, 1, 1, [1], "none", 0, 0.0),
    ("fp32", 4, 4, 5, [64, 0, 190, 1], "none", 0, 20.0),
    ("fp32", 4, 2, 9, [200, 300], "causal", 64, 0.0),
    ("fp32", 3, 1, 30, [150, 500], "document", 0, 0.0),
    ("fp32", 2, 2, 3, [4000], "window", 100, 50.0),
]


def _attend_inputs(dtype, heads, kv, rows, lens, spans, n_bias, cap, seed=11):
    g = np.random.default_rng(seed)
    c = _filled(seed, lens, kv)
    n_rows = [rows if b != 1 else max(rows - 2, 0) for b in range(len(lens))]
    q = _dev(g.standard_normal((len(lens), rows, heads * 64)) * 2, _dt(dtype))
    sp = _spans(spans, g, lens, n_rows, rows)
    bias = g.standard_normal((heads, n_bias)).astype(np.float32) if n_bias else None
    for b, n in enumerate(n_rows):
        q[b, n:] = math.nan                                       # rows that are not there are not read
    return c, q, n_rows, sp, bias


def _attend(c, q, n_rows, lens, sp, bias, cap, **kw):
    from paper_2506_23431_b200 import binding as B
    return B.cache_attention(q, c.d_codes, c.d_scales, c.d_table, _i32(n_rows), _i32(lens), 0.125, spans=None if sp is None else _i32(sp), bias=None if bias is None else _dev(bias),
                             softcap=cap, **kw)


@pytest.mark.parametrize("dtype,heads,kv,rows,lens,spans,n_bias,cap", ATTEND)
def test_attention_against_plain_form(dtype, heads, kv, rows, lens, spans, n_bias, cap):
    import torch
    c, q, n_rows, sp, bias = _attend_inputs(dtype, heads, kv, rows, lens, spans, n_bias, cap)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = _attend(c, q, n_rows, lens, sp, bias, cap, status=status)
    want = R.attend(_host(torch.nan_to_num(q)), c.codes, c.scales, c.table, n_rows, lens, 0.125, sp, bias, cap)
    _check(out, want, dtype)
    assert status.item() == 0
    for b, n in enumerate(n_rows):
        assert not out[b, n:].any()
    # the same bits again; with a scratch full of no numbers; with a bound on the lengths (other splits: within the bounds again)
    assert torch.equal(_attend(c, q, n_rows, lens, sp, bias, cap), out)
    from paper_2506_23431_b200 import binding as B
    need = B.cache_attention_scratch_bytes(1 if dtype == "bf16" else 0, len(lens), rows, heads, kv, c.table.shape[1] * 64)
    assert torch.equal(_attend(c, q, n_rows, lens, sp, bias, cap, scratch=torch.full((need // 4,), math.nan, device="cuda")), out)
    _check(_attend(c, q, n_rows, lens, sp, bias, cap, max_len=max(lens)), want, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [1e-37, 1e-30, 1e-6, 1e4, 1e20, 1e37])
def test_attention_over_blocks_of_any_size(dtype, size):
    """Keys and queries of any magnitude (the product in range), blocks of values 2^40 apart: what a block of small weights and large values adds is not lost."""
    import torch
    g = np.random.default_rng(13)
    lens = [300]
    c = Cache(13, 1, 5, 2)
    k = g.standard_normal((300, 2, 64)) / size
    v = g.standard_normal((300, 2, 64)) * 2.0 ** (np.arange(300) // 64 * 10 - 20)[:, None, None]
    k[:64] -= 3 / size * np.sign(k[:64])
    c.append(k, v, [0], lens, [0], "fp32")
    q = _dev(g.standard_normal((1, 4, 128)) * size, _dt(dtype))
    _check(_attend(c, q, [4], lens, None, None, 0.0), R.attend(_host(q), c.codes, c.scales, c.table, [4], lens, 0.125), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_numbers_reach_the_rows_that_see_them_and_no_others(dtype):
    import torch
    lens, rows = [150], 6
    for where, which in ((140, 0), (140, 1), (146, 1), (20, 1), (20, 0)):
        c = _filled(17, lens, 2)
        at = c.table[0, where // 64]
        t = where % 64
        if which == 0:
            c.codes[at, 1, 0].reshape(64, 64)[t, 3] = 0x7F
        else:
            c.codes[at, 1, 1].reshape(64, 64)[5, t] = 0xFF
        c.d_codes.copy_(_dev(c.codes))
        q = _dev(np.random.default_rng(3).standard_normal((1, rows, 256)), _dt(dtype))
        sp = np.array([[[0, 138], [0, 141], [141, 147], [30, 150], [0, 150], [0, 20]]])
        with np.errstate(invalid="ignore"):
            want = R.attend(_host(q), c.codes, c.scales, c.table, [rows], lens, 0.125, sp)
        sees = (sp[0, :, 0] <= where) & (where < sp[0, :, 1])
        ref = want[0].reshape(rows, 4, 64)
        got = _host(_attend(c, q, [rows], lens, sp, None, 0.0)).reshape(rows, 4, 64)
        assert (np.isnan(got) == np.isnan(ref)).all()
        assert (np.isnan(ref).any((1, 2)) == sees).all() and not np.isnan(ref[:, :2]).any()
        fine = ~np.isnan(ref)
        assert np.abs(got - ref)[fine].max() < 0.02 * np.abs(ref[fine]).max()
    # a query that is no number: its row alone
    c = _filled(17, lens, 2)
    q[0, 2, 70] = math.nan
    got = _host(_attend(c, q, [rows], lens, None, None, 0.0)).reshape(rows, 4, 64)
    assert np.isnan(got[2, 1]).all() and np.isnan(got).sum() == 64


def test_attention_bad_blocks_and_counts():
    """Table entries out of range count as positions that are not there; counts out of range are clamped; both stay inside the tensors."""
    import torch
    lens = [200, 130]
    c, q, n_rows, _, _ = _attend_inputs("bf16", 4, 2, 5, lens, "none", 0, 0.0)
    q = torch.nan_to_num(q)
    table = c.table.copy()
    table[0, 1], table[1, 2] = -3, c.codes.shape[0]
    d_table = c.d_table
    c.d_table = _i32(table)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = _attend(c, q, [9, -1], [200, 130], None, None, 0.0, status=status)
    assert status.item() == -1 and not out[1].any()
    sp = np.array([[[0, 64]] * 5, [[0, 0]] * 5])
    # positions 64..127 are missing: the first block and the ones behind, as a dense softmax over two spans
    near, far = R.attend(_host(q), c.codes, c.scales, c.table, [5, 0], lens, 0.125, sp), None
    whole = R.attend(_host(q), np.concatenate([c.codes[[c.table[0, 0]]], c.codes[[c.table[0, 2]]], c.codes[[c.table[0, 3]]]]),
                     np.concatenate([c.scales[[c.table[0, 0]]], c.scales[[c.table[0, 2]]], c.scales[[c.table[0, 3]]]]), np.array([[0, 1, 2], [0, 1, 2]]), [5, 0], [136, 0], 0.125)
    assert near[0].any() and far is None
    _check(out, whole, "bf16")
    # lengths beyond the table and below zero
    c.d_table = d_table
    c2 = _filled(19, [256], 2, extra_blocks=0)
    q2 = q[:1].contiguous()
    out = _attend(c2, q2, [5], [1 << 30], None, None, 0.0)
    _check(out, R.attend(_host(q2), c2.codes, c2.scales, c2.table, [5], [256], 0.125), "bf16")
    assert not _attend(c2, q2, [5], [-4], None, None, 0.0).any()
    assert not _attend(c2, q2, [0], [256], None, None, 0.0).any()
    _check(_attend(c2, q2, [5], [256], None, None, 0.0, max_len=100), R.attend(_host(q2), c2.codes, c2.scales, c2.table, [5], [100], 0.125), "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bias_of_the_lowest_value_removes_positions(dtype):
    """The type's lowest value, or minus infinity, as a mask by distance: the positions weigh nothing, a row with no others is zero."""
    import torch
    lens = [200]
    c = _filled(37, lens, 2)
    q = _dev(np.random.default_rng(4).standard_normal((1, 3, 128)), _dt(dtype))
    for low in (-math.inf, float(np.finfo(np.float32).min)):
        bias = np.zeros((2, 100), np.float32)
        bias[0, 70:] = low                                        # head 0 sees the last 70 positions only, head 1 all
        got = _attend(c, q, [3], lens, None, bias, 0.0)
        near = R.attend(_host(q), c.codes, c.scales, c.table, [3], lens, 0.125, np.array([[[130, 200]] * 3]))
        every = R.attend(_host(q), c.codes, c.scales, c.table, [3], lens, 0.125)
        for h, want in ((0, near), (1, every)):
            _check(got[..., h * 64:h * 64 + 64], tuple(w[..., h * 64:h * 64 + 64] for w in want), dtype)
        bias[0] = low
        assert not _attend(c, q, [3], lens, None, bias, 0.0)[..., :64].any()


def test_operators_after_copies_and_joined_streams_in_a_graph():
    """Each operator as the first node behind copies, a fill, and a join of two captured streams: it waits for all of them."""
    import torch
    from paper_2506_23431_b200 import binding as B
    g = np.random.default_rng(41)
    heads, n = 4, 3000
    c = Cache(41, 1, 60, heads)
    src = _dev(g.standard_normal((n, 3 * heads, 64)), torch.bfloat16)
    x, kv, q, out = torch.empty_like(src), torch.empty_like(src), torch.empty(1, 8, heads * 64, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 8, heads * 64, dtype=torch.bfloat16, device="cuda")
    pos, turns = torch.zeros(n, dtype=torch.int32, device="cuda"), _dev(B.rotary_turns(64)[0])
    want_pos = torch.arange(n, dtype=torch.int32, device="cuda")
    zero, cnt, lens, rows = _i32([0]), _i32([n]), _i32([0]), _i32([8])
    le = _i32([n])
    scratch = torch.empty(B.cache_attention_scratch_bytes(1, 1, 8, heads, heads, 60 * 64), dtype=torch.uint8, device="cuda")

    def chain(fork):
        s, s2 = torch.cuda.current_stream(), torch.cuda.Stream()
        if fork:
            s2.wait_stream(s)
            with torch.cuda.stream(s2):
                kv.copy_(src)
                lens.copy_(le)
        else:
            kv.copy_(src)
            lens.copy_(le)
        x.copy_(src)
        pos.copy_(want_pos)
        B.rotary(x, pos, turns, out=x)
        if fork:
            s.wait_stream(s2)
        B.cache_append(kv[:, heads:2 * heads], kv[:, 2 * heads:], zero, cnt, zero, c.d_table, c.d_codes, c.d_scales, n)
        q.zero_()
        q.copy_(x[-8:, :heads].reshape(1, 8, heads * 64))
        B.cache_attention(q, c.d_codes, c.d_scales, c.d_table, rows, lens, 0.125, out=out, scratch=scratch)

    chain(False)
    torch.cuda.synchronize()
    want, codes = out.clone(), c.d_codes.clone()
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        chain(True)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            chain(True)
    for _ in range(4):
        for t in (x, kv, q, out, pos, lens):
            t.zero_()
        c.d_codes[c.d_table.long()[0, :47]] = 0x7F
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.isfinite(out).all() and torch.equal(out, want)
        at = c.d_table.long()[0, :46]
        assert torch.equal(c.d_codes[at], codes[at])


def test_attention_strided_queries_and_batch_independence():
    import torch
    lens = [300, 64, 5, 129]
    c, q, n_rows, _, _ = _attend_inputs("bf16", 6, 3, 7, lens, "none", 0, 0.0)
    fused = torch.full((4, 7, 3 * 384), math.nan, dtype=q.dtype, device="cuda")
    fused[..., 384:768] = q
    out = _attend(c, fused[..., 384:768], n_rows, lens, None, None, 0.0)
    assert torch.equal(out, _attend(c, q, n_rows, lens, None, None, 0.0))
    want = R.attend(_host(torch.nan_to_num(q)), c.codes, c.scales, c.table, n_rows, lens, 0.125)
    _check(out, want, "bf16")
    # queries in an order that has no single row stride are refused
    with pytest.raises(ValueError):
        _attend(c, fused.transpose(0, 1).contiguous().transpose(0, 1)[..., :384], n_rows, lens, None, None, 0.0)


def test_attention_far_into_a_large_cache():
    """Blocks whose codes lie beyond 2^32 bytes of the cache's start."""
    import torch
    from paper_2506_23431_b200 import binding as B
    heads, lens = 8, [150]
    small = _filled(23, lens, heads)
    n = (5 << 30) // (heads * 8192)
    codes = torch.empty((n, heads, 2, 4096), dtype=torch.uint8, device="cuda")
    scales = torch.ones((n, heads, 2), device="cuda")
    far = np.array([[n - 1, n - 7000, n - 3]])
    assert (far * heads * 8192 > 1 << 32).all()
    g = np.random.default_rng(23)
    k, v = g.standard_normal((150, heads, 64)), g.standard_normal((150, heads, 64))
    B.cache_append(_dev(k, torch.bfloat16), _dev(v, torch.bfloat16), _i32([0]), _i32([150]), _i32([0]), _i32(far), codes, scales, 150)
    small.append(k, v, [0], [150], [0], "bf16")
    for i in range(3):
        assert torch.equal(codes[far[0, i], :, 0].view(heads, 64, 64)[:, :min(64, 150 - i * 64)], small.d_codes[small.table[0, i], :, 0].view(heads, 64, 64)[:, :min(64, 150 - i * 64)])
    q = torch.randn(1, 3, heads * 64, device="cuda").bfloat16()
    got = B.cache_attention(q, codes, scales, _i32(far), _i32([3]), _i32(lens), 0.125)
    assert torch.equal(got, B.cache_attention(q, small.d_codes, small.d_scales, small.d_table[:, :3].contiguous(), _i32([3]), _i32(lens), 0.125))


# ---- the three together ----------------------------------------------------------------------------------------
def test_decode_steps_rotate_append_attend():
    """A prompt and then single tokens of a batch, as a decode runs them: rotate queries and keys of the fused projection's rows, append, attend causally.
    Every step against the plain forms fed with the kernels' rotated rows (so that a step's rounding does not decide a code)."""
    import torch
    from paper_2506_23431_b200 import binding as B
    g = np.random.default_rng(29)
    heads, kv, batch = 4, 2, 3
    prompt = [70, 1, 33]
    c = Cache(29, batch, 3, kv)
    turns, amp = B.rotary_turns(64, 10000.0, B.PD_ROTARY_BY_PARTS, 4.0, 64)
    d_turns = _dev(turns)
    held = [0] * batch
    for step in range(6):
        n = prompt if step == 0 else [1, 1, 1 if step < 3 else 0]
        rows = sum(n)
        start = np.concatenate([[0], np.cumsum(n)])[:-1]
        qkv = _dev(g.standard_normal((rows, (heads + 2 * kv) * 64)), torch.bfloat16).view(rows, heads + 2 * kv, 64)
        pos = np.concatenate([held[b] + np.arange(n[b]) for b in range(batch)]).astype(np.int32)
        turn = qkv[:, :heads + kv]
        ref = R.rotate(_host(turn), pos, turns, amp, False, False)
        bound = _rotary_bound(_host(turn), pos, turns, amp, 64, False, "bf16", ref)
        B.rotary(turn, _i32(pos), d_turns, amp, out=turn)
        assert (np.abs(_host(turn) - ref) <= bound).all()
        k, v = qkv[:, heads:heads + kv], qkv[:, heads + kv:]
        B.cache_append(k, v, _i32(start), _i32(n), _i32(held), c.d_table, c.d_codes, c.d_scales, max(n))
        R.append(c.codes, c.scales, c.table, _host(k), _host(v), start, n, held)
        c.same()
        held = [h + x for h, x in zip(held, n)]
        most = min(8, max(n))
        q = torch.zeros(batch, most, heads * 64, dtype=torch.bfloat16, device="cuda")
        n_q = [min(most, x) for x in n]
        sp = np.zeros((batch, most, 2), np.int64)
        for b in range(batch):
            last = qkv[start[b]:start[b] + n[b], :heads].reshape(n[b], heads * 64)[n[b] - n_q[b]:]
            q[b, :n_q[b]] = last
            sp[b, :n_q[b], 1] = held[b] - n_q[b] + 1 + np.arange(n_q[b])
        out = _attend(c, q, n_q, held, sp, None, 0.0)
        _check(out, R.attend(_host(q), c.codes, c.scales, c.table, n_q, held, 0.125, sp), "bf16")


def test_captured_steps_follow_their_tensors():
    """Rotate, append and attend in one graph on a stream of its own; replayed with other rows, positions and lengths it gives what eager calls give."""
    import torch
    from paper_2506_23431_b200 import binding as B
    heads, batch = 2, 2
    g = np.random.default_rng(31)
    c, e = Cache(31, batch, 40, heads), Cache(31, batch, 40, heads)
    qkv = torch.zeros(batch, 3 * heads, 64, dtype=torch.bfloat16, device="cuda")
    pos, one, row, lens, ones = _i32([0, 0]), _i32([1, 1]), _i32([0, 1]), _i32([1, 1]), _i32([1, 1])
    turns, out = _dev(B.rotary_turns(64)[0]), torch.zeros(batch, 1, heads * 64, dtype=torch.bfloat16, device="cuda")
    scratch = torch.empty(B.cache_attention_scratch_bytes(1, batch, 1, heads, heads, 40 * 64), dtype=torch.uint8, device="cuda")

    def step(cache, x, to, sc):
        B.rotary(x[:, :2 * heads], pos, turns, out=x[:, :2 * heads])
        B.cache_append(x[:, heads:2 * heads], x[:, 2 * heads:], row, one, pos, cache.d_table, cache.d_codes, cache.d_scales, 1)
        return B.cache_attention(x[:, :heads].reshape(batch, 1, heads * 64), cache.d_codes, cache.d_scales, cache.d_table, ones, lens, 0.125, out=to, scratch=sc)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        step(c, qkv, out, scratch)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            step(c, qkv, out, scratch)
    held = 0
    for p in (0, 1, 2, 63, 64, 65, 900):
        x = _dev(g.standard_normal((batch, 3 * heads, 64)), torch.bfloat16)
        if p > held:                                              # a jump: fill both caches alike
            n = p - held
            kk, vv = _dev(g.standard_normal((2 * n, heads, 64)), torch.bfloat16), _dev(g.standard_normal((2 * n, heads, 64)), torch.bfloat16)
            for cache in (c, e):
                B.cache_append(kk, vv, _i32([0, n]), _i32([n, n]), _i32([held, held]), cache.d_table, cache.d_codes, cache.d_scales, n)
        held = p + 1
        pos.copy_(_i32([p, p]))
        lens.copy_(_i32([p + 1, p + 1]))
        qkv.copy_(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = step(e, x.clone(), torch.empty_like(out), torch.empty_like(scratch))
        assert torch.isfinite(out).all() and torch.equal(out, want) and torch.equal(c.d_scales[c.d_table.long()[:, p // 64]], e.d_scales[e.d_table.long()[:, p // 64]])


def test_sequences_that_share_blocks_and_many_short_ones():
    """A prefix held once for several sequences; a batch far larger than the GPU has places for, lengths from none."""
    import torch
    from paper_2506_23431_b200 import binding as B
    c = _filled(43, [200], 2)
    table = np.repeat(c.table, 3, axis=0)
    q = _dev(np.random.default_rng(6).standard_normal((3, 2, 256)), torch.bfloat16)
    lens = [200, 130, 64]
    out = B.cache_attention(q, c.d_codes, c.d_scales, _i32(table), _i32([2, 2, 2]), _i32(lens), 0.125)
    _check(out, R.attend(_host(q), c.codes, c.scales, table, [2, 2, 2], lens, 0.125), "bf16")
    n = 3000
    table = np.repeat(c.table, n, axis=0)
    lens = np.arange(n) % 201
    q = _dev(np.random.default_rng(7).standard_normal((n, 1, 128)), torch.bfloat16)
    out = B.cache_attention(q, c.d_codes, c.d_scales, _i32(table), _i32(np.ones(n)), _i32(lens), 0.125)
    some = list(range(0, n, 97))
    _check(out[some], R.attend(_host(q[some]), c.codes, c.scales, table[some], [1] * len(some), lens[some], 0.125), "bf16")


def test_no_tokens():
    import torch
    from paper_2506_23431_b200 import binding as B
    x = torch.zeros(0, 3, 64, dtype=torch.bfloat16, device="cuda")
    assert B.rotary(x, _i32(np.zeros(0)), _dev(B.rotary_turns(64)[0])).shape == (0, 3, 64)
    c = _filled(47, [70], 2)
    before = c.d_codes.clone()
    k = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    B.cache_append(k, k, _i32([0]), _i32([0]), _i32([70]), c.d_table, c.d_codes, c.d_scales, 0)
    B.cache_append(torch.ones(5, 2, 64, device="cuda"), torch.ones(5, 2, 64, device="cuda"), _i32([0]), _i32([0]), _i32([70]), c.d_table, c.d_codes, c.d_scales, 5)
    assert torch.equal(c.d_codes, before)
    out = B.cache_attention(torch.ones(1, 2, 128, dtype=torch.bfloat16, device="cuda"), c.d_codes, c.d_scales, c.d_table, _i32([2]), _i32([0]), 0.125, 0)
    assert not out.any()


def test_calls_on_two_streams_at_once():
    import torch
    lens = [5000]
    c, q, n_rows, _, _ = _attend_inputs("bf16", 4, 4, 3, lens, "none", 0, 0.0)
    want = _attend(c, q, n_rows, lens, None, None, 0.0)
    n, le = _i32(n_rows), _i32(lens)
    torch.cuda.synchronize()
    from paper_2506_23431_b200 import binding as B
    streams, outs = [torch.cuda.Stream() for _ in range(3)], []
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(B.cache_attention(q, c.d_codes, c.d_scales, c.d_table, n, le, 0.125))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
