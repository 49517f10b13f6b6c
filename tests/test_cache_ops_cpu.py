"""Host side of the operators around the 8-bit paged cache: frequencies, scratch sizes, refusals (no GPU is touched: a call with a bad
argument returns before its first CUDA call), and the pins of the plain forms that the GPU tests compare with."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2506_23431_b200 import binding as B
from tests import cache_reference as R

LIB = B._lib


def test_plain_form_of_the_format():
    import torch
    assert np.isnan(R.VALUES[[0x7F, 0xFF]]).all() and R.VALUES[126] == 448 and R.VALUES[1] == 2.0 ** -9
    every = np.array([c for c in range(256) if c & 0x7F != 0x7F], np.uint8)
    assert (R.to_code(R.VALUES[every]) == every).all()
    x = np.concatenate([np.random.default_rng(0).standard_normal(20000) * 50, (R.VALUES[:126] + R.VALUES[1:127]) / 2])
    x = np.clip(x, -448, 448).astype(np.float32)
    assert (R.to_code(x) == torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()).all()
    assert R.fresh_scale([448.0]) == 1 and R.fresh_scale([448.5]) == 2 and R.fresh_scale([0.0]) == 2.0 ** -126
    assert R.fresh_scale([math.inf, math.nan, 3.5]) == 2.0 ** -7


def test_plain_form_of_the_attention_against_a_dense_softmax():
    g = np.random.default_rng(1)
    k, v = g.standard_normal((70, 2, 64)), g.standard_normal((70, 2, 64))
    codes, scales = np.zeros((4, 2, 2, 4096), np.uint8), np.zeros((4, 2, 2))
    table = np.array([[3, 1]])
    R.append(codes, scales, table, k, v, [0], [70], [0])
    q = g.standard_normal((1, 1, 256))
    out, _, _ = R.attend(q, codes, scales, table, [1], [70], 0.125)
    for h in range(4):
        s = 0.125 * k[:, h // 2] @ q[0, 0, h * 64:h * 64 + 64]
        w = np.exp(s) / np.exp(s).sum()
        assert np.abs(out[0, 0, h * 64:h * 64 + 64] - w @ v[:, h // 2]).max() < 0.06      # quantisation alone: half a step is 2^-4 of a value
    # token by token the codes are the same here: later scales are never larger than the first token's times a power that the format holds
    c2, s2 = np.zeros_like(codes), np.zeros_like(scales)
    for p in range(70):
        R.append(c2, s2, table, k[p:p + 1], v[p:p + 1], [0], [1], [p])
    assert (s2 == scales).all()


def test_rotary_frequencies():
    plain, amp = B.rotary_turns(64)
    assert amp == 1.0 and np.allclose(plain, 10000.0 ** (-np.arange(32) / 32) / (2 * math.pi), rtol=1e-14)
    lin, amp = B.rotary_turns(20, 500.0, B.PD_ROTARY_LINEAR, 4.0)
    assert amp == 1.0 and np.allclose(lin, 500.0 ** (-np.arange(10) / 10) / (8 * math.pi), rtol=1e-14)
    parts, amp = B.rotary_turns(64, 10000.0, B.PD_ROTARY_BY_PARTS, 16.0, 4096)
    base = 10000.0 ** (-np.arange(32) / 32) / (2 * math.pi)
    turns = base * 4096                                                   # over the original context
    assert amp == pytest.approx(0.1 * math.log(16.0) + 1)
    assert np.allclose(parts[turns >= 40], base[turns >= 40], rtol=1e-14) and np.allclose(parts[turns <= 0.8], base[turns <= 0.8] / 16, rtol=1e-14)
    between = parts[(turns < 32) & (turns > 1)] / base[(turns < 32) & (turns > 1)]
    assert (np.diff(between) < 0).all() and between.max() < 1 and between.min() > 1 / 16
    assert (B.rotary_turns(64, 10000.0, B.PD_ROTARY_BY_PARTS, 1.0, 4096)[0] == base).all() or np.allclose(B.rotary_turns(64, 10000.0, B.PD_ROTARY_BY_PARTS, 1.0, 4096)[0], base)


@pytest.mark.parametrize("args", [(3, 10000.0), (0, 10000.0), (258, 10000.0), (64, 1.0), (64, math.inf), (64, math.nan), (64, 10000.0, 7), (64, 10000.0, 1, 0.5),
                                  (64, 10000.0, 1, math.nan), (64, 10000.0, 2, 4.0, 0), (64, 10000.0, 2, 4.0, 4096, 1.0, 2.0), (64, 10000.0, 2, 4.0, 4096, 32.0, 0.0)])
def test_rotary_frequencies_refuse(args):
    with pytest.raises(B.PdError) as e:
        B.rotary_turns(*args)
    assert e.value.status == -1


def _call(name, good, **bad):
    """The entry point's status with some of the arguments of a call that would be taken replaced."""
    args = dict(good)
    assert set(bad) <= set(args)
    args.update(bad)
    return getattr(LIB, name)(*args.values())


P = 1 << 20            # an address that is never followed: every call here is refused
ROTARY = dict(dtype=1, tokens=4, n_heads=3, d_head=64, rot_dim=64, interleaved=0, inverse=0, x=P, xt=192, xh=64, pos=P, turns=P, amp=1.0, out=2 * P, ot=192, oh=64, stream=None)
APPEND = dict(dtype=1, batch=2, heads=3, n_blocks=8, max_blocks=4, rows=10, max_new=5, k=P, ks=192, v=P, vs=192, row_start=P, n_new=P, pos=P, table=P, codes=P, scales=P,
              status=None, stream=None)
ATTEND = dict(dtype=1, batch=2, rows=5, heads=6, kv=3, n_blocks=8, max_blocks=4, max_len=200, scale=0.125, cap=0.0, q=P, qs=384, codes=P, scales=P, table=P, n_rows=P, lens=P,
              spans=None, bias=None, n_bias=0, out=P, scratch=P, bytes=1 << 30, status=None, stream=None)


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(tokens=-1), dict(n_heads=0), dict(d_head=257), dict(rot_dim=63), dict(rot_dim=66), dict(rot_dim=0), dict(x=None), dict(out=None),
                                 dict(pos=None), dict(turns=None), dict(x=P + 1), dict(pos=P + 2), dict(turns=P + 4), dict(xt=-1), dict(oh=32), dict(ot=128), dict(oh=0), dict(ot=0),
                                 dict(out=P, ot=256), dict(ot=64, oh=128)])
def test_rotary_refuses(bad):
    assert _call("pd_rotary", ROTARY, **bad) == -1


def test_nothing_to_do_is_no_error():
    assert _call("pd_rotary", ROTARY, tokens=0, x=None, out=None, pos=None, turns=None) == 0
    assert _call("pd_cache_append", APPEND, max_new=0) == 0 and _call("pd_cache_append", APPEND, rows=0, k=None, v=None) == 0


@pytest.mark.parametrize("bad", [dict(dtype=-1), dict(batch=0), dict(batch=65536), dict(heads=0), dict(n_blocks=0), dict(max_blocks=0), dict(rows=-1), dict(max_new=-1), dict(k=None),
                                 dict(v=None), dict(table=None), dict(codes=None), dict(scales=None), dict(n_new=None), dict(pos=None), dict(row_start=None), dict(k=P + 8), dict(codes=P + 4),
                                 dict(ks=128), dict(vs=196), dict(scales=P + 4), dict(table=P + 2), dict(n_new=P + 1), dict(row_start=P + 2), dict(pos=P + 2), dict(status=P + 2)])
def test_append_refuses(bad):
    assert _call("pd_cache_append", APPEND, **bad) == -1


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(batch=0), dict(rows=0), dict(rows=65), dict(heads=7), dict(heads=2), dict(kv=0), dict(n_blocks=0), dict(max_blocks=0), dict(max_len=-1),
                                 dict(scale=0.0), dict(scale=math.nan), dict(scale=math.inf), dict(cap=-1.0), dict(cap=math.nan), dict(q=None), dict(codes=None), dict(table=None),
                                 dict(n_rows=None), dict(lens=None), dict(out=None), dict(q=P + 8), dict(out=P + 8), dict(qs=320), dict(qs=388), dict(spans=P + 4), dict(bias=P, n_bias=0),
                                 dict(scales=P + 4), dict(scratch=P + 8), dict(table=P + 2), dict(lens=P + 2), dict(n_rows=P + 1), dict(bias=P + 2, n_bias=4), dict(status=P + 2)])
def test_attention_refuses(bad):
    assert _call("pd_cache_attention", ATTEND, **bad) == -1


def test_attention_scratch():
    need = LIB.pd_cache_attention_scratch_bytes(1, 1, 8, 12, 12, 100000)
    assert need > 256
    big = dict(batch=1, rows=8, heads=12, kv=12, qs=768, max_blocks=2000, max_len=100000)
    assert _call("pd_cache_attention", ATTEND, bytes=need - 1, **big) == -3
    assert _call("pd_cache_attention", ATTEND, scratch=None, **big) == -1
    for args in [(2, 1, 8, 12, 12, 10), (1, 0, 8, 12, 12, 10), (1, 1, 65, 12, 12, 10), (1, 1, 8, 12, 5, 10), (1, 1, 8, 12, 12, -1)]:
        assert LIB.pd_cache_attention_scratch_bytes(*args) == 0


def test_binding_checks_its_tensors():
    import torch
    x = torch.zeros(4, 3, 64)
    with pytest.raises(ValueError):
        B.rotary(x.to(torch.float16), torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64))
    with pytest.raises(ValueError):
        B.rotary(x, torch.zeros(4, dtype=torch.int64), torch.zeros(32, dtype=torch.float64))
    with pytest.raises(ValueError, match="CUDA"):
        B.rotary(x, torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64))
    assert C.sizeof(C.c_int32) == 4 and B.PD_CACHE_BLOCK == R.BLOCK
