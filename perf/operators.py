"""What a decode step asks of a cache held in 8 bits, as cases that can be timed and compared.

Three operators, used one after the other on a step's projected rows: rotary positions on the queries and keys, the
append of keys and values to a paged cache of E4M3 codes (64-token blocks, a power-of-two scale for each block, head and
keys | values), and the attention of the step's rows over that cache.

Every pass comes in two forms: the framework's kernels (`own`), and elementary torch operations in 32 bits (64 for
angles).  The cache's layout is the framework's: codes [blocks, kv heads, 2, 4096], keys of a block as [token][dim],
values as [dim][token]; scales [blocks, kv heads, 2]; a table [batch, blocks of a sequence] of block ids.
"""
import math

import numpy as np
import torch

own = False

DH, BLOCK = 64, 64
_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _rotary(name, tokens, q_heads, kv_heads, **kw):
    c = {"name": name, "kind": "rotary", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "rot": DH, "interleaved": False, "factor": 1.0,
         "far": 4096, "inverse": False, "dtype": "bf16"}
    c.update(kw)
    return c


def _append(name, batch, kv_heads, ctx, new, **kw):
    c = {"name": name, "kind": "append", "batch": batch, "kv_heads": kv_heads, "ctx": ctx, "new": new, "ragged": True, "dtype": "bf16"}
    c.update(kw)
    return c


def _attend(name, batch, rows, heads, kv_heads, ctx, **kw):
    c = {"name": name, "kind": "attend", "batch": batch, "rows": rows, "heads": heads, "kv_heads": kv_heads, "ctx": ctx, "ragged": False, "spans": "none",
         "window": 0, "bias": False, "cap": 0.0, "dtype": "bf16"}
    c.update(kw)
    return c


def listed():
    return [
        # queries and keys of the open subsequences of one request: one small launch
        _rotary("rotary_step", 8, 12, 12),
        # queries and keys of a batch of long prompts
        _rotary("rotary_prompt", 32 * 2048, 16, 16),
        # part of the head, neighbouring dims paired, frequencies scaled by parts, far positions, 32 bits; the backward direction
        _rotary("rotary_far", 5003, 5, 5, rot=40, interleaved=True, factor=32.0, far=1 << 20, inverse=True, dtype="fp32"),
        # one new token for each of a batch of running sequences
        _append("append_token", 64, 12, 1024, 1),
        # documents of different lengths written in one call
        _append("append_prompt", 32, 16, 0, 2048),
        # a few hundred more tokens behind older ones, in 32 bits
        _append("append_chunk", 7, 5, 700, 333, dtype="fp32"),
        # one request over a document of odd length
        _attend("attend_one", 1, 8, 12, 12, 777),
        # a batch of documents: the step of the summarisation workload
        _attend("attend_step", 32, 12, 16, 16, 2048),
        # two sequences over a very long cache, four query heads to a key head, one row each
        _attend("attend_long", 2, 1, 16, 4, 131072),
        # a step's own tokens at the end of sequences of different lengths: causal, with a bias that depends on the distance
        _attend("attend_causal_bias", 16, 8, 16, 16, 1024, ragged=True, spans="causal", bias=True),
        # many rows for shared key heads, a window of positions for each row, capped scores
        _attend("attend_window_cap", 8, 33, 8, 2, 4096, ragged=True, spans="window", window=1500, cap=30.0),
        # the same in 32 bits, few sequences
        _attend("attend_fp32", 3, 5, 4, 4, 1500, ragged=True, dtype="fp32", cap=20.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "append", "attend", "attend", "attend"])
    if kind == "rotary":
        q, kv = rng.randint(1, 16), rng.randint(1, 16)
        c = _rotary("", _log_int(rng, 1, 32 * 2048 * 32 // (q + kv)), q, kv, rot=rng.choice([2, 10, 20, 32, 48, 56, 64, 64, 64]), interleaved=rng.random() < 0.5,
                    factor=rng.choice([1.0, 1.0, 4.0, 32.0]), far=_log_int(rng, 64, 1 << 22), inverse=rng.random() < 0.25, dtype=rng.choice(["bf16", "bf16", "fp32"]))
        if c["dtype"] == "fp32":
            c["tokens"] = max(1, c["tokens"] // 2)
    elif kind == "append":
        batch, kv = _log_int(rng, 1, 64), rng.randint(1, 16)
        most = max(1, 32 * 2048 * 16 // (batch * kv))
        new = 1 if rng.random() < 0.3 else _log_int(rng, 1, min(8192, most))
        c = _append("", batch, kv, rng.choice([0, _log_int(rng, 1, 2000)]), new, ragged=rng.random() < 0.6, dtype=rng.choice(["bf16", "bf16", "fp32"]))
        if c["dtype"] == "fp32":
            c["new"] = max(1, c["new"] // 2)
    else:
        kv, group = rng.choice([1, 2, 3, 4, 8, 12, 16]), rng.choice([1, 1, 1, 2, 4, 8])
        batch = _log_int(rng, 1, 64)
        rows = rng.choice([1, _log_int(rng, 1, 16), _log_int(rng, 1, 64)])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        keys = 32 * 2048 * 16 // (batch * kv)                     # no more cache, and no more scores, than the largest listed ones
        keys = min(keys, 32 * 2048 * 16 * 12 // (batch * kv * group * rows), 131072)
        ctx = _log_int(rng, 1, max(1, keys if dtype == "bf16" else keys // 4))
        spans = rng.choice(["none", "none", "causal", "window"])
        c = _attend("", batch, rows, kv * group, kv, ctx, ragged=rng.random() < 0.6, spans=spans, window=_log_int(rng, 1, ctx) if spans == "window" else 0,
                    bias=rng.random() < 0.3, cap=rng.choice([0.0, 0.0, 15.0, 50.0]), dtype=dtype)
    del c["name"]
    return c


# ---- shapes: functions of the case alone -------------------------------------------------------------------
def _ragged(n, most, on):
    """n lengths up to `most`: all of it, or spread from none to all of it with the longest first."""
    if not on or n == 1:
        return np.full(n, most, np.int64)
    return np.round(most * (1.0 - (np.arange(n) * 0.61803398875) % 1.0)).astype(np.int64)


def _shape(c):
    if c["kind"] == "append":
        return _ragged(c["batch"], c["ctx"], c["ragged"])[::-1].copy(), _ragged(c["batch"], c["new"], c["ragged"] and c["new"] > 1)
    lens = _ragged(c["batch"], c["ctx"], c["ragged"])
    n_rows = np.minimum(c["rows"], np.maximum(1, lens)) if c["spans"] != "none" else np.full(c["batch"], c["rows"])
    return lens, n_rows


def _spans(c, lens, n_rows):
    """[batch, rows, 2] first visible position and the one behind the last; rows that are not there: nothing."""
    r = np.arange(c["rows"])[None, :]
    end = np.where(r < n_rows[:, None], np.maximum(lens[:, None] - n_rows[:, None] + 1 + r, 0), 0)
    end = np.minimum(end, lens[:, None])
    begin = np.maximum(end - c["window"], 0) if c["spans"] == "window" else np.zeros_like(end)
    return np.stack([begin, end], -1).astype(np.int32)


def _turns(rot, theta, factor, original):
    """Turns per position of every rotated pair; by parts: slow pairs' positions divided by `factor`, fast ones' not."""
    i = np.arange(rot // 2, dtype=np.float64)
    f = theta ** (-2.0 * i / rot)
    if factor == 1.0:
        return f / (2 * math.pi), 1.0
    place = lambda turns: rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    lo, hi = max(math.floor(place(32.0)), 0), min(math.ceil(place(1.0)), rot - 1)
    ramp = np.clip((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
    return (f / factor * ramp + f * (1 - ramp)) / (2 * math.pi), 0.1 * math.log(factor) + 1.0


def _quantise(x):
    """[..., 4096] in 32 bits -> codes and a power-of-two scale for each block."""
    e = _exponent(x.abs().amax(-1))
    s = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)
    return (x / s[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), s


def _exponent(amax):
    """The least e >= -126 with amax <= 448 * 2^e."""
    m, e = torch.frexp(amax)
    return torch.where(amax == 0, torch.full_like(e, -126), torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126))


def _cache(g, n_blocks, kv_heads):
    """A cache in use: channels of different size among the keys, blocks of different size among the values."""
    dev = torch.device("cuda")
    dim = 0.5 + 2 * torch.rand(kv_heads, 1, DH, device=dev, generator=g)
    k = torch.randn(n_blocks, kv_heads, BLOCK, DH, device=dev, generator=g) * dim
    v = torch.randn(n_blocks, kv_heads, DH, BLOCK, device=dev, generator=g) * torch.exp2(torch.randint(-2, 3, (n_blocks, kv_heads, 1, 1), device=dev, generator=g).float())
    return _quantise(torch.stack([k.flatten(2), v.flatten(2)], 2))


# ---- inputs ------------------------------------------------------------------------------------------------
def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    dt = _DT[c["dtype"]]
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev, torch.int32)  # noqa: E731
    if c["kind"] == "rotary":
        n, heads = c["tokens"], c["q_heads"] + c["kv_heads"]
        qkv = torch.randn(n, (heads + c["kv_heads"]) * DH, device=dev, generator=g).to(dt)      # a fused projection's rows
        turns, amplitude = _turns(c["rot"], 10000.0, c["factor"], 4096)
        return {"c": c, "x": qkv[:, :heads * DH].view(n, heads, DH), "pos": torch.randint(0, c["far"], (n,), device=dev, generator=g, dtype=torch.int32),
                "turns": torch.from_numpy(turns).to(dev), "amplitude": amplitude}
    B, H = c["batch"], c["kv_heads"]
    if c["kind"] == "append":
        pos0, n_new = _shape(c)
        per_seq = max(1, int(-(-(pos0 + n_new).max() // BLOCK)))
        codes, scales = _cache(g, B * per_seq, H)
        table = torch.randperm(B * per_seq, device=dev, generator=g).view(B, per_seq).to(torch.int32)
        row0 = np.concatenate([[0], np.cumsum(n_new)])[:-1]
        total = max(1, int(n_new.sum()))
        kv = torch.randn(total, 2 * H * DH, device=dev, generator=g)
        kv[:, H * DH:] *= torch.exp2(torch.randint(-2, 3, (total, 1), device=dev, generator=g).float())
        kv = kv.to(dt)                                                                          # a fused projection's rows
        # the blocks that receive tokens, for the plain form: sequence, block, first and last new position in it
        first = pos0 // BLOCK
        count = np.where(n_new > 0, -(-(pos0 + n_new) // BLOCK) - first, 0)
        seq = np.repeat(np.arange(B), count)
        blk = np.concatenate([first[b] + np.arange(count[b]) for b in range(B)])
        lo = np.maximum(pos0[seq] - blk * BLOCK, 0)
        hi = np.minimum((pos0 + n_new)[seq] - blk * BLOCK, BLOCK)
        return {"c": c, "k": kv[:, :H * DH].view(total, H, DH), "v": kv[:, H * DH:].view(total, H, DH), "row0": i32(row0), "n_new": i32(n_new), "pos0": i32(pos0),
                "table": table, "codes": codes, "scales": scales, "max_new": int(n_new.max()),
                "plan": torch.from_numpy(np.stack([seq, blk, lo, hi, row0[seq] + blk * BLOCK - pos0[seq]]).astype(np.int64)).to(dev)}
    lens, n_rows = _shape(c)
    per_seq = max(1, -(-c["ctx"] // BLOCK))
    codes, scales = _cache(g, B * per_seq, H)
    table = torch.randperm(B * per_seq, device=dev, generator=g).view(B, per_seq).to(torch.int32)
    # what stands behind a sequence's last token is whatever the block held before: here no numbers at all
    pos = torch.arange(per_seq * BLOCK, device=dev).view(per_seq, BLOCK)
    stale = (pos[None] >= torch.from_numpy(lens).to(dev)[:, None, None]).nonzero()
    view = codes.view(B * per_seq, H, 2, BLOCK, DH)
    at = table.long()[stale[:, 0], stale[:, 1]]
    view[at, :, 0, stale[:, 2]] = 0x7F
    view[at, :, 1, :, stale[:, 2]] = 0x7F
    qkv = torch.randn(B, c["rows"], 3, c["heads"] * DH, device=dev, generator=g).to(dt)
    bias = None
    if c["bias"]:
        # one value for each bucket of distances (exact up to 15, logarithmic up to 127), drawn anew for each head
        d = torch.arange(512, device=dev)
        far = 16 + (torch.log(d.clamp(min=1).float() / 16) / math.log(8.0) * 16).long()
        bucket = torch.where(d < 16, d, far.clamp(max=31))
        bias = (torch.randn(c["heads"], 32, device=dev, generator=g) * 0.5)[:, bucket].contiguous()
    return {"c": c, "q": qkv[:, :, 0], "codes": codes, "scales": scales, "table": table, "n_rows": i32(n_rows), "lens": i32(lens),
            "spans": None if c["spans"] == "none" else i32(_spans(c, lens, n_rows)), "bias": bias, "scale": DH ** -0.5}


# ---- the pass ----------------------------------------------------------------------------------------------
def run(s):
    c = s["c"]
    if own:
        from paper_2506_23431_b200 import binding as B
        if c["kind"] == "rotary":
            return B.rotary(s["x"], s["pos"], s["turns"], s["amplitude"], interleaved=c["interleaved"], inverse=c["inverse"])
        if c["kind"] == "append":
            B.cache_append(s["k"], s["v"], s["row0"], s["n_new"], s["pos0"], s["table"], s["codes"], s["scales"], s["max_new"])
            return {"codes": s["codes"].view(torch.float8_e4m3fn), "scales": s["scales"]}
        return B.cache_attention(s["q"], s["codes"], s["scales"], s["table"], s["n_rows"], s["lens"], s["scale"], c["ctx"], spans=s["spans"], bias=s["bias"],
                                 softcap=c["cap"])
    return {"rotary": _run_rotary, "append": _run_append, "attend": _run_attend}[c["kind"]](s)


def _run_rotary(s):
    c, x = s["c"], s["x"].float()
    n, r = x.shape[0], c["rot"]
    t = s["pos"].double()[:, None] * s["turns"][None, :]
    t = (t - torch.round(t)) * (2 * math.pi)
    cos, sin = (torch.cos(t) * s["amplitude"]).float()[:, None], (torch.sin(t) * s["amplitude"]).float()[:, None]
    if c["inverse"]:
        sin = -sin
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([y, x[..., r:]], -1).to(s["x"].dtype)


def _run_append(s):
    seq, blk, lo, hi, row = s["plan"]
    codes, scales, H = s["codes"], s["scales"], s["c"]["kv_heads"]
    at = s["table"].long()[seq, blk]
    t = torch.arange(BLOCK, device=at.device)
    new = (t >= lo[:, None]) & (t < hi[:, None])                                  # [touched, 64]
    old = t < lo[:, None]
    rows = (row[:, None] + t).clamp(0, s["k"].shape[0] - 1)
    for w, x in ((0, s["k"]), (1, s["v"])):
        x = torch.where(new[:, :, None, None], x[rows].float(), 0.0).transpose(1, 2)          # [touched, heads, tokens, dims]
        was = codes[at, :, w].view(-1, H, BLOCK, DH)
        was = was if w == 0 else was.transpose(2, 3)
        had = scales[at, :, w]
        fresh = torch.ldexp(torch.ones_like(had), _exponent(x.abs().amax((2, 3))))
        now = torch.where(lo[:, None] > 0, torch.maximum(had, fresh), fresh)[:, :, None, None]
        moved = (was.contiguous().view(torch.float8_e4m3fn).float() * (had[:, :, None, None] / now)).to(torch.float8_e4m3fn).view(torch.uint8)
        put = (x / now).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        got = torch.where(new[:, None, :, None], put, torch.where(old[:, None, :, None], moved, was))
        codes[at, :, w] = (got if w == 0 else got.transpose(2, 3)).flatten(2)
        scales[at, :, w] = now[:, :, 0, 0]
    return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales}


def _run_attend(s):
    c, q = s["c"], s["q"].float()
    B, R, Hq, H = c["batch"], c["rows"], c["heads"], c["kv_heads"]
    at = s["table"].long()
    L = at.shape[1] * BLOCK
    kv = s["codes"][at].view(torch.float8_e4m3fn).float() * s["scales"][at][..., None]         # [batch, blocks, heads, 2, 4096]
    k = kv[:, :, :, 0].unflatten(-1, (BLOCK, DH)).permute(0, 2, 1, 3, 4).reshape(B, H, L, DH)
    v = kv[:, :, :, 1].unflatten(-1, (DH, BLOCK)).permute(0, 2, 1, 4, 3).reshape(B, H, L, DH)
    pos = torch.arange(L, device=q.device)
    held = (pos < s["lens"][:, None])[:, None, :, None]
    k, v = torch.where(held, k, 0.0), torch.where(held, v, 0.0)
    if s["spans"] is None:
        begin, end = torch.zeros(B, R, 1, device=q.device, dtype=torch.int64), s["lens"].long()[:, None, None].expand(B, R, 1)
    else:
        begin, end = s["spans"].long()[..., 0:1], s["spans"].long()[..., 1:2]
    there = (torch.arange(R, device=q.device) < s["n_rows"][:, None])[..., None]
    seen = (pos >= begin) & (pos < end) & (pos < s["lens"][:, None, None]) & there             # [batch, rows, positions]
    q = q.view(B, R, H, Hq // H, DH).permute(0, 2, 3, 1, 4)                                    # [batch, kv heads, group, rows, 64]
    score = torch.matmul(q.reshape(B, H, -1, DH), k.transpose(2, 3)).view(B, H, Hq // H, R, L) * s["scale"]
    if c["cap"] > 0:
        score = c["cap"] * torch.tanh(score / c["cap"])
    if s["bias"] is not None:
        near = (end - 1 - pos).clamp(0, s["bias"].shape[1] - 1)
        score = score + s["bias"][:, near].permute(1, 0, 2, 3).reshape(B, H, Hq // H, R, L)
    score = torch.where(seen[:, None, None], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    out = torch.matmul(p.reshape(B, H, -1, L), v).view(B, H, Hq // H, R, DH) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    return out.permute(0, 3, 1, 2, 4).reshape(B, R, Hq * DH).to(s["q"].dtype)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------
def _round_e4m3(x):
    """Nearest E4M3 value, ties to even, in 64 bits."""
    e = torch.frexp(x)[1].clamp(min=-5).double()                  # x = m 2^e with m in [0.5, 1): four bits behind the point
    step = torch.exp2(e - 4)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] == "rotary":
        x = s["x"].double()
        a = 2 * math.pi * torch.remainder(s["pos"].double()[:, None] * s["turns"], 1.0)
        z = torch.polar(torch.full_like(a, s["amplitude"]), -a if c["inverse"] else a)[:, None]
        r = c["rot"]
        if c["interleaved"]:
            y = torch.view_as_real(torch.view_as_complex(x[..., :r].unflatten(-1, (r // 2, 2)).contiguous()) * z).flatten(-2)
        else:
            w = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * z
            y = torch.cat([w.real, w.imag], -1)
        x = x.contiguous()
        x[..., :r] = y
        return x
    if c["kind"] == "append":
        codes = s["codes"].view(torch.float8_e4m3fn).float().double().view(-1, c["kv_heads"], 2, BLOCK, DH)
        scales = s["scales"].double()
        table = s["table"].cpu().numpy()
        for seq, blk, lo, hi, row in s["plan"].cpu().numpy().T:
            at = int(table[seq, blk])
            for w, x in ((0, s["k"]), (1, s["v"])):
                x = x[row + lo:row + hi].double().transpose(0, 1)                 # [heads, new tokens, dims]
                body = codes[at, :, w] if w == 0 else codes[at, :, w].transpose(1, 2)
                need = torch.log2(x.abs().amax((1, 2)).clamp(min=448 * 2.0 ** -126) / 448).ceil()
                to = torch.exp2(need)
                if lo > 0:
                    to = torch.maximum(to, scales[at, :, w])
                    body[:, :lo] = _round_e4m3(body[:, :lo] * (scales[at, :, w] / to)[:, None, None])
                body[:, lo:hi] = _round_e4m3(x / to[:, None, None])
                scales[at, :, w] = to
        return {"codes": codes.view(-1, c["kv_heads"], 2, BLOCK * DH), "scales": scales}
    B, R, Hq, H = c["batch"], c["rows"], c["heads"], c["kv_heads"]
    lens, n_rows = _shape(c)
    spans = _spans(c, lens, n_rows) if c["spans"] != "none" else np.stack([np.zeros((B, R), np.int64), np.where(np.arange(R) < n_rows[:, None], lens[:, None], 0)], -1)
    out = torch.zeros(B, R, Hq, DH, dtype=torch.float64, device="cuda")
    for b in range(B):
        n = int(lens[b])
        if n == 0:
            continue
        at = s["table"][b, :-(-n // BLOCK)].long()
        kv = s["codes"][at].view(torch.float8_e4m3fn).double() * s["scales"][at].double()[..., None]
        k = kv[:, :, 0].view(-1, H, BLOCK, DH).transpose(0, 1).reshape(H, -1, DH)[:, :n].repeat_interleave(Hq // H, 0)
        v = kv[:, :, 1].view(-1, H, DH, BLOCK).permute(1, 0, 3, 2).reshape(H, -1, DH)[:, :n].repeat_interleave(Hq // H, 0)
        for r in range(int(n_rows[b])):
            lo, hi = int(spans[b, r, 0]), int(spans[b, r, 1])
            if hi <= lo:
                continue
            score = torch.einsum("hd,hkd->hk", s["q"][b, r].double().view(Hq, DH), k[:, lo:hi]) * s["scale"]
            if c["cap"] > 0:
                score = c["cap"] * torch.tanh(score / c["cap"])
            if s["bias"] is not None:
                score = score + s["bias"].double()[:, (hi - 1 - torch.arange(lo, hi, device="cuda")).clamp(max=s["bias"].shape[1] - 1)]
            out[b, r] = torch.einsum("hk,hkd->hd", torch.softmax(score, -1), v[:, lo:hi])
    return out.view(B, R, Hq * DH)


# ---- what a pass cannot do without -----------------------------------------------------------------------------
def work(case):
    c = dict(case)
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rotary":
        n = c["tokens"] * (c["q_heads"] + c["kv_heads"])
        return {"bytes": float(2 * n * DH * e + c["tokens"] * 4 + c["rot"] // 2 * 8), "flops": float(3 * n * c["rot"])}
    H = c["kv_heads"]
    if c["kind"] == "append":
        pos0, n_new = _shape(c)
        blocks = int(np.where(n_new > 0, -(-(pos0 + n_new) // BLOCK) - pos0 // BLOCK, 0).sum())
        n = int(n_new.sum())
        return {"bytes": float(2 * n * H * DH * (e + 1) + blocks * (4 + H * 8)), "flops": float(2 * 2 * n * H * DH)}
    lens, n_rows = _shape(c)
    rows = int(n_rows.sum())
    if c["spans"] == "none":
        seen, pairs = int(lens.sum()), int((lens * n_rows).sum())
    else:
        sp = _spans(c, lens, n_rows).astype(np.int64)
        there = np.arange(c["rows"])[None, :] < n_rows[:, None]
        first = np.where(there, sp[..., 0], 1 << 40).min(1)
        seen = int(np.maximum(np.where(there, sp[..., 1], 0).max(1) - np.minimum(first, lens), 0).sum())
        pairs = int(np.maximum(sp[..., 1] - sp[..., 0], 0).sum())
    return {"bytes": float(seen * H * 2 * DH + seen // BLOCK * (4 + H * 8) + 2 * rows * c["heads"] * DH * e), "flops": float(4 * DH * c["heads"] * pairs)}
