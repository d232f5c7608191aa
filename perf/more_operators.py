"""Rotary positions, the rotated append and the 4-bit cache's attention, as cases that can be timed and checked.

  rotate  rows of queries or keys turned to their positions, forwards, back again, or all by one shift (laser_rotate);
  append  new keys rotated into the paged cache, values beside them, queries rotated into rows of their own
          (laser_kv_write_rotated), and the written positions read back as the values the cache now stands for;
  attend  attention of new tokens, one or a chunk of them per sequence, over a cache held in 4 bits (laser_attend).

A case names its heads (hq query heads, hkv key/value heads of hd dimensions: those of the shapes in configs.py), the
cache's element type (mxfp4: blocks of 32 dims with a power of two as their scale; int8, fp8, bf16, f32), the type `io` of the
caller's rows, and `batch` sequences that hold `lo` to `hi` positions before `n` new ones come.  Rotations are of the first
`rot` dims, as pairs (i, i + rot/2) ("half") or (2i, 2i + 1) ("interleaved"), with plain or scaled frequencies.

With `own` false the operators run in their plain form: pages of the values that a cache stands for, gathered, and elementary
operations in float32; rotations in float64, since the values that are kept in 4 bits lie next to borders and angles are large.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
PAGE = 16
Q15, Q7, L8, TINY = HEADS = [(12, 2, 128), (28, 4, 128), (32, 8, 128), (4, 2, 64)]
THETA = {Q15: 1.0e4, Q7: 1.0e4, L8: 5.0e5, TINY: 1.0e4}
IO = {"bf16": torch.bfloat16, "f32": torch.float32}
SCALED = {"plain": {}, "linear": {"factor": 4.0}, "base": {"factor": 4.0},
          "bands": {"factor": 8.0, "old_positions": 8192.0, "low": 1.0, "high": 4.0},
          "ramp": {"factor": 4.0, "old_positions": 4096.0, "low": 1.0, "high": 32.0}}


def _case(name, op, heads, io, batch, lo, hi, n, kv="mxfp4", rot=0, layout="half", scaling="plain", turn="on", window=0):
    c = {"op": op, "hq": heads[0], "hkv": heads[1], "hd": heads[2], "io": io, "batch": batch, "lo": lo, "hi": hi, "n": n}
    if op != "rotate":
        c["kv"] = kv
    if op == "attend":
        c["window"] = window
    else:
        c.update(rot=rot or heads[2], layout=layout, scaling=scaling)
    if op == "rotate":
        c["turn"] = turn
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one decoded token's queries, at the end of a long chain of thought: latency counts
        _case("rotate-1", "rotate", Q7, "bf16", 1, 14335, 14335, 1),
        # a busy server's step in fp32: half of each head rotated, pairs side by side, positions interpolated
        _case("rotate-b33-part", "rotate", Q15, "f32", 33, 100, 60000, 1, rot=64, layout="interleaved", scaling="linear"),
        # the queries of a whole long prompt, frequencies in bands
        _case("rotate-16384", "rotate", L8, "bf16", 1, 0, 0, 16384, scaling="bands"),
        # one decoded token of one request goes into the 4-bit cache of a layer
        _case("append-1", "append", Q7, "bf16", 1, 14335, 14335, 1),
        # the same for a full server
        _case("append-b64", "append", L8, "bf16", 64, 3000, 14000, 1, scaling="bands"),
        # answers' prompts of a few hundred tokens in fp32 rows into a 16-bit cache, part of the head rotated
        _case("append-b5-part", "append", Q15, "f32", 5, 50, 275, 203, kv="bf16", rot=96, layout="interleaved", scaling="ramp"),
        # a whole chain of thought arrives from another engine
        _case("append-14336", "append", L8, "bf16", 1, 0, 0, 14336, scaling="bands"),
        # a token of a toy model; of one request at the end of a long chain of thought; of a full server
        _case("attend-tiny", "attend", TINY, "f32", 1, 130, 130, 1),
        _case("attend-1", "attend", Q7, "bf16", 1, 14335, 14335, 1),
        _case("attend-b64", "attend", L8, "bf16", 64, 3000, 14000, 1),
        # the probe's answer-inducing suffix behind a long chain of thought
        _case("attend-suffix-8", "attend", Q7, "bf16", 1, 14001, 14001, 8),
        # a chunk of a long prompt: the matrix cores' work
        _case("attend-chunk-4096", "attend", L8, "bf16", 1, 12288, 12288, 4096),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotate", "append", "attend", "attend"])
    heads = rng.choice(HEADS)
    io = "f32" if rng.random() < 0.25 else "bf16"
    batch = 1 if rng.random() < 0.4 else _log_int(rng, 2, 64)
    turned = {"rot": heads[2] if rng.random() < 0.6 else 2 * rng.randint(1, heads[2] // 2),
              "layout": rng.choice(["half", "half", "interleaved"]), "scaling": rng.choice(sorted(SCALED))}
    if op == "rotate":
        n = 1 if rng.random() < 0.3 else _log_int(rng, 1, 16384 // batch)
        hi = _log_int(rng, 1, 200000)
        return _case(None, op, heads, io, batch, rng.randint(0, hi), hi, n, turn=rng.choice(["on", "on", "back", "shift"]), **turned)
    if op == "append":
        kv = rng.choice(["mxfp4", "mxfp4", "bf16", "int8", "fp8"]) if io == "bf16" else rng.choice(["mxfp4", "bf16", "fp8"])
        n = 1 if rng.random() < 0.3 else _log_int(rng, 1, min(14336, 30000 // batch))
        hi = _log_int(rng, 1, 14336)
        return _case(None, op, heads, io, batch, rng.randint(0, hi), hi, n, kv=kv, **turned)
    kind = rng.choice(["decode", "decode", "suffix", "chunk"])
    window = _log_int(rng, 16, 4096) if rng.random() < 0.15 else 0
    if kind == "decode":
        hi = _log_int(rng, 1, min(65000, 600000 // batch))
        return _case(None, op, heads, io, batch, rng.randint(0, hi), hi, 1, window=window)
    if kind == "suffix":
        batch = min(batch, 16)
        hi = _log_int(rng, 1, 14336)
        return _case(None, op, heads, io, batch, rng.randint(0, hi), hi, rng.randint(2, 40), window=window)
    batch = rng.choice([1, 1, 2, 3])
    n = _log_int(rng, 41, 4096 // batch)
    hi = _log_int(rng, 1, 12288)
    return _case(None, op, heads, io, batch, rng.randint(0, hi), hi, n, window=window)


# ------------------------------------------------------------------------------ inputs

def _contexts(case):
    """Positions each sequence holds before the new ones: the two ends of the range, the rest between."""
    b, lo, hi = case["batch"], case["lo"], case["hi"]
    g = torch.Generator().manual_seed(4000 + 31 * lo + hi + b)
    mid = [int(x) for x in torch.randint(lo, hi + 1, (b,), generator=g)]
    return [hi] if b == 1 else [lo, hi] + mid[2:]


def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + 7919 * what) % (1 << 62))


def _rows(case, rows, seed, what, dtype):
    """Rows of keys or values: normal, with channels of different size (a few much larger, as keys have them)."""
    g = _gen(seed, what)
    shape = (rows, case["hkv"], case["hd"])
    size = torch.exp(0.6 * torch.randn((1,) + shape[1:], generator=g, device=DEV))
    return (torch.randn(shape, generator=g, device=DEV) * size).to(dtype)


def _queries(case, rows, seed):
    return torch.randn((rows, case["hq"], case["hd"]), generator=_gen(seed, 5), device=DEV).to(IO[case["io"]])


def _inputs(case, seed):
    """Positions held, the cached rows (sequence after sequence), the new rows, the queries."""
    ctx = _contexts(case)
    n, b, io = case["n"], case["batch"], IO[case["io"]]
    held = new = None
    if case["op"] == "attend":
        total = sum(ctx) + b * n
        held = tuple(_rows(case, total, seed, i, torch.bfloat16) for i in (1, 2))
    if case["op"] == "append":
        new = tuple(_rows(case, b * n, seed, i, io) for i in (3, 4))
    return ctx, held, new, _queries(case, b * n, seed)


# ------------------------------------------------------------------------------ the plain form

def _theta(case):
    return THETA[(case["hq"], case["hkv"], case["hd"])]


def _frequencies(case):
    """Angle per position of each pair, and what sines and cosines are multiplied by."""
    r, theta, p = case["rot"], _theta(case), SCALED[case["scaling"]]
    f = theta ** (-torch.arange(0, r, 2, dtype=torch.float64, device=DEV) / r)
    if case["scaling"] == "linear":  # positions interpolated
        return f / p["factor"], 1.0
    if case["scaling"] == "base":  # a larger base: the slowest pair `factor` times slower
        wide = theta * p["factor"] ** (r / max(r - 2, 1))
        return wide ** (-torch.arange(0, r, 2, dtype=torch.float64, device=DEV) / r), 1.0
    if case["scaling"] == "bands":  # by a pair's turns over the old context: many stay, few are interpolated
        turns = p["old_positions"] * f / (2.0 * math.pi)
        keep = ((turns - p["low"]) / (p["high"] - p["low"])).clamp(0.0, 1.0)
        return f * (keep + (1.0 - keep) / p["factor"]), 1.0
    if case["scaling"] == "ramp":  # along the pairs, between those that make `high` and `low` turns there
        at = [r * math.log(p["old_positions"] / (2.0 * math.pi * t)) / (2.0 * math.log(theta)) for t in (p["high"], p["low"])]
        first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
        slow = ((torch.arange(r // 2, dtype=torch.float64, device=DEV) - first) / max(last - first, 1.0e-3)).clamp(0.0, 1.0)
        return f * (1.0 - slow + slow / p["factor"]), 1.0 + 0.1 * math.log(p["factor"])
    return f, 1.0


def _turned(case, x, pos):
    """Rows x [rows, heads, hd] at positions pos [rows], in float64."""
    r, x = case["rot"], x.double()
    f, amplitude = _frequencies(case)
    angle = (pos.double()[:, None] * f)[:, None, :]
    c, s = torch.cos(angle) * amplitude, torch.sin(angle) * amplitude
    if case["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * c - b * s, b * c + a * s, x[..., r:]], -1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., r:]], -1)


def _stored(kv, x):
    """The values that a cache of type `kv` keeps of rows x [..., hd], in float32."""
    if kv == "mxfp4":
        blocks = x.reshape(x.shape[:-1] + (-1, 32))
        m, e = torch.frexp(blocks.abs().amax(-1, keepdim=True))  # the largest is m 2^e, m in [1/2, 1)
        e = (e - 3 + (m > 0.875).to(e.dtype)).clamp(-100, 125)   # at most 7 2^e
        scale = torch.ldexp(torch.ones_like(m), e)
        y = blocks / scale
        step = torch.where(y.abs() < 2.0, 0.5, torch.where(y.abs() < 4.0, 1.0, 2.0))
        return ((torch.round(y / step) * step).clamp(-6.0, 6.0) * scale).reshape(x.shape).float()
    if kv == "fp8":
        scale = torch.ldexp(torch.ones_like(x), (torch.frexp(x)[1] - 4).clamp_min(-9))
        return (torch.round(x / scale) * scale).clamp(-448.0, 448.0).float()
    if kv == "int8":
        x = x.float()
        top = x.abs().amax(-1, keepdim=True)
        q = torch.where(top > 0, torch.round(127.0 * x / top), torch.zeros((), device=x.device))
        return q * (top / 127.0)
    scale = torch.ldexp(torch.ones_like(x), torch.frexp(x)[1] - 8)  # bf16, rounded once: eight significant bits
    return (torch.round(x / scale) * scale).float()


class _PlainCache:
    """Pages [page, position in the page, kv head, hd] of the values kept; `at`: where each sequence's pages start."""

    def __init__(self, case, lengths):
        pages = [-(-n // PAGE) for n in lengths]
        self.kv = case["kv"]
        self.pools = [torch.zeros((max(1, sum(pages)), PAGE, case["hkv"], case["hd"]), device=DEV) for _ in range(2)]
        starts = [sum(pages[:i]) for i in range(len(pages))]
        self.table = torch.arange(0, max(1, max(pages)), device=DEV)[None, :] + torch.tensor(starts, device=DEV)[:, None]

    def write(self, seq, pos, k, v):
        page, slot = self.table[seq, pos // PAGE], pos % PAGE
        for pool, x in zip(self.pools, (k, v)):
            pool[page, slot] = _stored(self.kv, x)

    def read(self, seq, pos):
        page, slot = self.table[seq, pos // PAGE], pos % PAGE
        return [pool[page, slot] for pool in self.pools]


def _places(starts, lengths):
    """Sequence and position of rows that lie sequence after sequence."""
    n = torch.tensor(lengths, device=DEV)
    seq = torch.repeat_interleave(torch.arange(len(lengths), device=DEV), n)
    first = torch.cumsum(n, 0) - n
    return seq, torch.arange(sum(lengths), device=DEV) - first[seq] + torch.tensor(starts, device=DEV)[seq]


# ------------------------------------------------------------------------------ the framework's handles

_models = {}


def _model(case):
    """A model handle with the case's heads (one layer, everything else as small as it goes)."""
    from paper_2606_31580_amd import laser as L, synth
    from paper_2606_31580_amd.configs import ModelShape

    key = (case["hq"], case["hkv"], case["hd"], case["kv"])
    if key not in _models:
        shape = ModelShape("heads-%d-%d-%d" % key[:3], 1, 64, key[0], key[1], key[2], 64, 64, True, False, "bf16", 1.0e4,
                           1.0e-6, kv_dtype="" if case["kv"] == "bf16" else case["kv"])
        _models[key] = L.Model(shape, synth.make_weights(shape, device=DEV), max_rows=1, max_positions=65536, tiles=False)
    return _models[key]


def _cache(case, lengths):
    from paper_2606_31580_amd import laser as L

    pages = [-(-n // PAGE) for n in lengths]
    kv = L.KVCache(_model(case), max(1, sum(pages)), len(lengths), max(1, max(pages)))
    for i, n in enumerate(lengths):
        kv.add_seq(i, n)
    return kv


def _rope(case):
    from paper_2606_31580_amd import laser as L

    return L.rope(case["hd"], _theta(case), rot_dim=case["rot"], layout=case["layout"], scaling=case["scaling"], **SCALED[case["scaling"]])


# ------------------------------------------------------------------------------ the interface

def _turn(case, c):
    """First position and step of the n rows of a sequence that holds c positions."""
    return {"on": (c, 1), "back": (-c, -1), "shift": (-c, 0)}[case.get("turn", "on")]


def prepare(case, seed):
    ctx, held, new, q = _inputs(case, seed)
    n, b, io = case["n"], case["batch"], IO[case["io"]]
    lengths = [c + n for c in ctx]
    state = {"case": case, "ctx": ctx, "new": new, "q": q, "q_out": torch.empty_like(q)}
    if case["op"] == "attend":
        state["lse"] = torch.empty(q.shape[:2], device=DEV)
    if case["op"] == "append":
        state["back"] = tuple(torch.empty((b * n, case["hkv"], case["hd"]), dtype=io, device=DEV) for _ in range(2))
    if own:
        _prepare_own(case, state, held, lengths)
    else:
        _prepare_plain(case, state, held, lengths)
    return state


def _prepare_own(case, state, held, lengths):
    from paper_2606_31580_amd import laser as L

    n, ctx = case["n"], state["ctx"]
    if case["op"] != "attend":
        state["rope"] = _rope(case)
    if case["op"] == "rotate":
        state["runs"] = [L.rotate_run(n, pos, i * n, step) for i, (pos, step) in enumerate(_turn(case, c) for c in ctx)]
        return
    kv = state["kv"] = _cache(case, lengths)
    state["runs"] = [L.kv_run(i, c, n, i * n) for i, c in enumerate(ctx)]
    state["spans"] = [L.attend_span(i, n, c, i * n) for i, c in enumerate(ctx)]
    if held is not None:
        L.laser_kv_write(kv, 0, [L.kv_run(i, 0, x, sum(lengths[:i])) for i, x in enumerate(lengths)], *held)
    else:
        L.laser_kv_write(kv, 0, [])  # the block table goes up


def _prepare_plain(case, state, held, lengths):
    n, b, ctx = case["n"], case["batch"], state["ctx"]
    if case["op"] == "rotate":
        first = torch.tensor([_turn(case, c)[0] for c in ctx], device=DEV)
        state["pos"] = (first[:, None] + _turn(case, 0)[1] * torch.arange(n, device=DEV)[None, :]).flatten()
        return
    kv = state["kv"] = _PlainCache(case, lengths)
    state["seq"], state["pos"] = _places(ctx, [n] * b)
    if held is not None:
        kv.write(*_places([0] * b, lengths), *(x.double() for x in held))
        state["len"] = torch.tensor(lengths, device=DEV)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    from paper_2606_31580_amd import laser as L

    case = state["case"]
    if case["op"] == "rotate":
        L.laser_rotate(state["rope"], state["runs"], state["q"], state["q_out"])
        return state["q_out"]
    if case["op"] == "append":
        L.laser_kv_write_rotated(state["kv"], 0, state["rope"], state["runs"], *state["new"], q=state["q"], q_out=state["q_out"])
        L.laser_kv_read(state["kv"], 0, state["runs"], *state["back"])
        return state["back"] + (state["q_out"],)
    L.laser_attend(state["kv"], 0, state["spans"], state["q"], state["q_out"], lse=state["lse"], window=case["window"])
    return state["q_out"], state["lse"]


def _run_plain(state):
    case, q_out = state["case"], state["q_out"]
    if case["op"] == "attend":
        return _attend_plain(state)
    q_out.copy_(_turned(case, state["q"], state["pos"]))
    if case["op"] == "rotate":
        return q_out
    k, v = state["new"]
    state["kv"].write(state["seq"], state["pos"], _turned(case, k, state["pos"]), v.double())
    for out, x in zip(state["back"], state["kv"].read(state["seq"], state["pos"])):
        out.copy_(x)
    return state["back"] + (q_out,)


def _attend_plain(state):
    """All sequences at once, shorter ones padded with positions that no row sees."""
    case, kv, length = state["case"], state["kv"], state["len"]
    b, n, hq, hkv, hd = (case[x] for x in ("batch", "n", "hq", "hkv", "hd"))
    group, longest = hq // hkv, max(state["ctx"]) + n
    t = torch.arange(longest, device=DEV)
    at = torch.minimum(t[None, :], length[:, None] - 1)
    k, v = kv.read(torch.arange(b, device=DEV)[:, None], at)  # [b, longest, hkv, hd]
    q = state["q"].float().view(b, n, hkv, group, hd).permute(0, 2, 3, 1, 4).reshape(b, hkv, group * n, hd)
    s = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(hd)
    row = (length - n)[:, None] + torch.arange(n, device=DEV)[None, :]
    seen = t[None, None, :] <= row[:, :, None]
    if case["window"]:
        seen = seen & (t[None, None, :] > row[:, :, None] - case["window"])
    s = s.view(b, hkv, group, n, longest).masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, hkv, group * n, longest), v.permute(0, 2, 1, 3).contiguous()).view(b, hkv, group, n, hd) / total
    state["q_out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(b * n, hq, hd))
    state["lse"].copy_((torch.log(total) + top)[..., 0].permute(0, 3, 1, 2).reshape(b * n, hq))
    return state["q_out"], state["lse"]


def work(case):
    hq, hkv, hd, n, b = (case[k] for k in ("hq", "hkv", "hd", "n", "batch"))
    io = 2 if case["io"] == "bf16" else 4
    if case["op"] == "rotate":
        return {"bytes": 2 * b * n * hq * hd * io, "flops": 3 * b * n * hq * case["rot"]}
    # K and V of one position as the cache holds them
    place = 2 * hkv * {"mxfp4": hd // 2 + hd // 32, "int8": hd + 4, "fp8": hd, "bf16": 2 * hd}[case["kv"]]
    if case["op"] == "append":  # rows in, pages out and in, rows out
        return {"bytes": b * n * (2 * place + 4 * hkv * hd * io + 2 * hq * hd * io), "flops": 3 * b * n * (hq + hkv) * case["rot"]}
    w = case["window"]
    pairs = places = 0
    for c in _contexts(case):
        places += min(c + n, w + n - 1) if w else c + n
        pairs += sum(min(c + i + 1, w) if w else c + i + 1 for i in range(n))
    return {"bytes": places * place + b * n * hq * (2 * hd * io + 4), "flops": 4 * hd * hq * pairs}


# ------------------------------------------------------------------------------ the definition in 64 bits

def _kept(kv, x):
    """What a cache stands for once it holds the rows x [..., hd], in float64."""
    if kv == "mxfp4":  # the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times 2^e; half way: the one with the even code
        d = x.double().unflatten(-1, (-1, 32))
        top = d.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 7.0)).clamp(-100.0, 125.0)
        y = d.abs() * 2.0 ** -e
        code = torch.zeros_like(y)
        for i, half in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
            code += (y > half) if i % 2 == 0 else (y >= half)
        value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)[code.long()]
        return (torch.copysign(value, d) * 2.0 ** e).flatten(-2)
    if kv == "int8":
        x = x.double()
        top = x.abs().amax(-1, keepdim=True)
        return torch.where(top > 0, torch.round(127.0 * x / torch.where(top > 0, top, 1.0)) * top / 127.0, 0.0)
    if kv == "fp8":  # three fraction bits above 2^-6, steps of 2^-9 below, at most 448
        step = torch.exp2(torch.floor(torch.log2(x.double().abs().clamp_min(2.0 ** -6))).clamp(-6, 8) - 3)
        return (torch.round(x.double() / step) * step).clamp(-448.0, 448.0)
    # bf16: the neighbour below from the magnitude's upper bits, then up or not by what is left, half way to the even one
    d = x.double().abs()
    unit = torch.exp2(torch.floor(torch.log2(torch.where(d > 0, d, 1.0))) - 7)
    below = torch.floor(d / unit)
    left = d / unit - below
    return torch.copysign((below + ((left > 0.5) | ((left == 0.5) & (below % 2 == 1))).double()) * unit, x.double())


def _speed(case, i):
    """Radians per position of pair i."""
    r, theta, p, kind = case["rot"], _theta(case), SCALED[case["scaling"]], case["scaling"]
    f = math.exp(-2.0 * i / r * math.log(theta))
    if kind == "plain":
        return f
    if kind == "linear":
        return f / p["factor"]
    if kind == "base":
        return f if i == 0 else f * math.exp(-2.0 * i / (r - 2) * math.log(p["factor"]))
    if kind == "bands":
        wave = 2.0 * math.pi / f
        if wave < p["old_positions"] / p["high"]:
            return f
        if wave > p["old_positions"] / p["low"]:
            return f / p["factor"]
        keep = (p["old_positions"] / wave - p["low"]) / (p["high"] - p["low"])
        return (1.0 - keep) * f / p["factor"] + keep * f
    lo, hi = (r / 2 * math.log(p["old_positions"] / (2.0 * math.pi * t), theta) for t in (p["high"], p["low"]))
    lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), r - 1)
    slow = min(max((i - lo) / max(hi - lo, 1.0e-3), 0.0), 1.0)
    return (1.0 - slow) * f + slow * f / p["factor"]


def _at(case, x, pos):
    """Rows at their positions: each pair as a complex number times amplitude exp(i angle)."""
    r = case["rot"]
    f = torch.tensor([_speed(case, i) for i in range(r // 2)], dtype=torch.float64, device=DEV)
    amplitude = 0.1 * math.log(SCALED["ramp"]["factor"]) + 1.0 if case["scaling"] == "ramp" else 1.0
    turn = torch.polar(torch.full((), amplitude, dtype=torch.float64, device=DEV).expand(pos.shape[0], r // 2).contiguous(),
                       torch.outer(pos.double(), f))[:, None, :]
    out = x.double().clone()
    first, second = (slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    z = torch.complex(out[..., first].contiguous(), out[..., second].contiguous()) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def exact(case, seed):
    ctx, held, new, q = _inputs(case, seed)
    n, hd, group = case["n"], case["hd"], case["hq"] // case["hkv"]
    if case["op"] != "attend":
        pos = []
        for c in ctx:
            p, step = _turn(case, c)
            pos += [p + step * i for i in range(n)]
        pos = torch.tensor(pos, device=DEV)
        if case["op"] == "rotate":
            return _at(case, q, pos)
        return _kept(case["kv"], _at(case, new[0], pos)), _kept(case["kv"], new[1]), _at(case, q, pos)
    o = torch.empty(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device=DEV)
    at = 0
    for i, c in enumerate(ctx):
        k, v = (_kept(case["kv"], x[at:at + c + n]) for x in held)
        at += c + n
        rows = q[i * n:(i + 1) * n].double()
        for h in range(case["hq"]):  # head by head, a few hundred rows at a time
            kh, vh = k[:, h // group], v[:, h // group]
            for r0 in range(0, n, 512):
                r1 = min(n, r0 + 512)
                s = rows[r0:r1, h] @ kh.t() * hd ** -0.5
                t = torch.arange(c + n, device=DEV)
                r = torch.arange(c + r0, c + r1, device=DEV)[:, None]
                hidden = (t > r) | (t + case["window"] <= r) if case["window"] else t > r
                s[hidden] = -math.inf
                z = torch.logsumexp(s, -1)
                o[i * n + r0:i * n + r1, h] = torch.exp(s - z[:, None]) @ vh
                lse[i * n + r0:i * n + r1, h] = z
    return o, lse
