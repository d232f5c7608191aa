"""The paged KV cache's own operators, as cases that can be timed and checked.

  roundtrip  rows of K and V quantised into the cache as they are written (laser_kv_write), and the
             written positions read back as the values the cache now stands for (laser_kv_read);
  read       a sequence's K and V read out of the cache (laser_kv_read);
  attend     attention of new tokens, one or a chunk of them per sequence, over the sequences'
             cached positions (laser_attend): output rows and their log-sum-exps.

A case names its heads (hq query heads, hkv key/value heads of hd dimensions), the cache's element
type (int8 with a scale per position and head, fp8, bf16, f32), the type `io` of the caller's rows,
and `batch` sequences that hold `lo` to `hi` positions before `n` new ones come.  Heads are those of
the model shapes in configs.py.

With `own` false the operators run in their plain form: the cache is a paged array of stored values
(and scales), pages are gathered and everything is computed in float32.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
PAGE = 16
HEADS = [(12, 2, 128), (28, 4, 128), (32, 8, 128), (4, 2, 64)]
IO = {"bf16": torch.bfloat16, "f32": torch.float32}
STORE = {"int8": torch.int8, "fp8": torch.float8_e4m3fn, "bf16": torch.bfloat16, "f32": torch.float32}
ITEM = {"int8": 1, "fp8": 1, "bf16": 2, "f32": 4}


def _case(name, op, heads, kv, io, batch, lo, hi, n, window=0):
    c = {"op": op, "hq": heads[0], "hkv": heads[1], "hd": heads[2], "kv": kv, "io": io, "batch": batch, "lo": lo,
         "hi": hi, "n": n, "window": window}
    return c if name is None else dict(c, name=name)


def listed():
    q15, q7, l8, tiny = HEADS
    return [
        # one decoded token of one request goes into the cache of a layer: latency counts
        _case("roundtrip-1", "roundtrip", q7, "int8", "bf16", 1, 14001, 14001, 1),
        # a busy server's step: one token of each of 33 requests
        _case("roundtrip-b33-fp8", "roundtrip", l8, "fp8", "bf16", 33, 100, 14000, 1),
        # an answer's prompt of a few hundred tokens for five requests, fp32 rows
        _case("roundtrip-b5-f32rows", "roundtrip", q15, "int8", "f32", 5, 50, 275, 203),
        # a whole chain of thought arrives from another engine
        _case("roundtrip-14336", "roundtrip", l8, "int8", "bf16", 1, 0, 0, 14336),
        # a short prompt is read back in fp32; a long chain of thought in bf16
        _case("read-275", "read", tiny, "int8", "f32", 1, 275, 275, 0),
        _case("read-14001", "read", q7, "int8", "bf16", 1, 14001, 14001, 0),
        # the decode step of a toy model, and of one request at the end of a long chain of thought
        _case("attend-tiny", "attend", tiny, "f32", "f32", 1, 130, 130, 1),
        _case("attend-1", "attend", q7, "int8", "bf16", 1, 14335, 14335, 1),
        # decode of a ragged batch from a bf16 cache; of a full server from the int8 one
        _case("attend-b4-bf16", "attend", q7, "bf16", "f32", 4, 3000, 14000, 1),
        _case("attend-b64", "attend", l8, "int8", "bf16", 64, 3000, 14000, 1),
        # the probe's answer-inducing suffix behind a long chain of thought
        _case("attend-suffix-8", "attend", q7, "int8", "bf16", 1, 14001, 14001, 8),
        # a chunk of a long prompt: the matrix cores' work
        _case("attend-chunk-4096", "attend", l8, "int8", "bf16", 1, 12288, 12288, 4096),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["roundtrip", "read", "attend", "attend", "attend"])
    heads = rng.choice(HEADS)
    kv = rng.choice(["int8", "int8", "int8", "fp8", "bf16"]) if heads != HEADS[3] else rng.choice(["int8", "f32"])
    io = "f32" if heads == HEADS[3] or rng.random() < 0.25 else "bf16"
    batch = 1 if rng.random() < 0.4 else _log_int(rng, 2, 64)
    if op == "read":
        hi = _log_int(rng, 1, min(65000, 400000 // batch))
        return _case(None, op, heads, kv, io, batch, rng.randint(1, hi), hi, 0)
    if op == "roundtrip":
        n = 1 if rng.random() < 0.3 else _log_int(rng, 1, min(16384, 100000 // batch))
        hi = _log_int(rng, 1, 14336)
        return _case(None, op, heads, kv, io, batch, rng.randint(0, hi), hi, n)
    kind = rng.choice(["decode", "decode", "suffix", "chunk"])
    window = _log_int(rng, 16, 4096) if rng.random() < 0.15 else 0
    if kind == "decode":
        hi = _log_int(rng, 1, min(65000, 600000 // batch))
        return _case(None, op, heads, kv, io, batch, rng.randint(0, hi), hi, 1, window)
    if kind == "suffix":
        batch = min(batch, 16)
        hi = _log_int(rng, 1, 14336)
        return _case(None, op, heads, kv, io, batch, rng.randint(0, hi), hi, rng.randint(2, 40), window)
    batch = rng.choice([1, 1, 2, 3])
    n = _log_int(rng, 41, 4096 // batch)
    hi = _log_int(rng, 1, 14336)
    return _case(None, op, heads, kv, io, batch, rng.randint(0, hi), hi, n, window)


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


def _inputs(case, seed):
    """The cached rows (ragged, sequence after sequence), and the new rows or queries."""
    ctx = _contexts(case)
    io = IO[case["io"]]
    src = torch.float32 if case["kv"] == "f32" else torch.bfloat16
    n, b = case["n"], case["batch"]
    total = sum(ctx) + (b * n if case["op"] == "attend" else 0)
    held = None
    if case["op"] != "roundtrip":
        held = (_rows(case, total, seed, 1, src), _rows(case, total, seed, 2, src))
    new = q = None
    if case["op"] == "roundtrip":
        new = (_rows(case, b * n, seed, 3, io), _rows(case, b * n, seed, 4, io))
    if case["op"] == "attend":
        q = torch.randn((b * n, case["hq"], case["hd"]), generator=_gen(seed, 5), device=DEV).to(io)
    return ctx, held, new, q


# ------------------------------------------------------------------------------ the plain form's cache

def _quantise(kv, x):
    """Rows [..., hd] as the cache holds them: (stored values, scales or None)."""
    x = x.float()
    if kv == "int8":  # (127 x is exact for bf16 rows, so that a value half way between two steps is seen as one)
        top = x.abs().amax(-1)
        q = torch.where(top[..., None] > 0, torch.round(127.0 * x / top[..., None]), torch.zeros((), device=x.device))
        return q.clamp(-127, 127).to(torch.int8), top / torch.full((), 127.0, device=x.device)
    if kv == "fp8":
        return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn), None
    return x.to(STORE[kv]), None


def _values(stored, scale):
    return stored.float() if scale is None else stored.float() * scale[..., None]


class _PlainCache:
    """Pages [page, kv head, position in the page, hd] of stored values, scales [page, kv head, position]."""

    def __init__(self, case, lengths):
        pages = [-(-n // PAGE) for n in lengths]
        dims = (sum(pages), case["hkv"], PAGE, case["hd"])
        self.kv = case["kv"]
        self.pools = [torch.zeros(dims, dtype=STORE[self.kv], device=DEV) for _ in range(2)]
        self.scales = [torch.zeros(dims[:3], device=DEV) if self.kv == "int8" else None for _ in range(2)]
        self.tables, at = [], 0
        for p in pages:
            self.tables.append(torch.arange(at, at + p, device=DEV))
            at += p

    def places(self, seq, pos, n):
        t = torch.arange(pos, pos + n, device=DEV)
        return self.tables[seq][t // PAGE], t % PAGE

    def write(self, seq, pos, k, v):
        page, slot = self.places(seq, pos, k.shape[0])
        for i, x in enumerate((k, v)):
            stored, scale = _quantise(self.kv, x)
            # (as bytes: not every torch has indexed stores of 8-bit floats)
            pool = self.pools[i].view(torch.uint8) if self.kv == "fp8" else self.pools[i]
            pool[page, :, slot] = stored.view(torch.uint8) if self.kv == "fp8" else stored
            if scale is not None:
                self.scales[i][page, :, slot] = scale

    def read(self, seq, pos, n):
        page, slot = self.places(seq, pos, n)
        out = []
        for i in range(2):
            pool = self.pools[i]
            stored = pool.view(torch.uint8)[page, :, slot].view(pool.dtype) if self.kv == "fp8" else pool[page, :, slot]
            out.append(_values(stored, None if self.scales[i] is None else self.scales[i][page, :, slot]))
        return out


# ------------------------------------------------------------------------------ the framework's cache

_models = {}


def _model(case):
    """A model handle with the case's heads (one layer, everything else as small as it goes)."""
    from paper_2606_31580_amd import laser as L, synth
    from paper_2606_31580_amd.configs import ModelShape

    key = (case["hq"], case["hkv"], case["hd"], case["kv"])
    if key not in _models:
        dtype = "f32" if case["kv"] == "f32" else "bf16"
        shape = ModelShape("heads-%d-%d-%d" % key[:3], 1, 64, key[0], key[1], key[2], 64, 64, True, False, dtype, 1.0e4,
                           1.0e-6, kv_dtype=case["kv"] if case["kv"] in ("int8", "fp8") else "")
        _models[key] = L.Model(shape, synth.make_weights(shape, device=DEV), max_rows=1, max_positions=65536, tiles=False)
    return _models[key]


def _cache(case, lengths):
    from paper_2606_31580_amd import laser as L

    pages = [-(-n // PAGE) for n in lengths]
    kv = L.KVCache(_model(case), max(1, sum(pages)), len(lengths), max(1, max(pages)))
    for i, n in enumerate(lengths):
        kv.add_seq(i, n)
    return kv


# ------------------------------------------------------------------------------ the interface

def prepare(case, seed):
    ctx, held, new, q = _inputs(case, seed)
    n, b = case["n"], case["batch"]
    lengths = [c + n for c in ctx]
    state = {"case": case, "ctx": ctx, "new": new, "q": q}
    filled = ctx if case["op"] == "roundtrip" else lengths
    starts = [sum(filled[:i]) for i in range(b)]
    if own:
        from paper_2606_31580_amd import laser as L

        kv = state["kv"] = _cache(case, lengths)
        state["runs"] = [L.kv_run(i, c, n, i * n) for i, c in enumerate(ctx)]
        if held is not None:
            L.laser_kv_write(kv, 0, [L.kv_run(i, 0, filled[i], starts[i]) for i in range(b)], held[0], held[1])
            state["whole"] = [L.kv_run(i, 0, filled[i], starts[i]) for i in range(b)]
        else:
            L.laser_kv_write(kv, 0, [], new[0], new[1])  # the block table goes up
        state["spans"] = [L.attend_span(i, n, c, i * n) for i, c in enumerate(ctx)]
    else:
        kv = state["kv"] = _PlainCache(case, lengths)
        if held is not None:
            for i in range(b):
                part = slice(starts[i], starts[i] + filled[i])
                kv.write(i, 0, held[0][part], held[1][part])
    io = IO[case["io"]]
    if case["op"] == "attend":
        state["out"] = (torch.empty_like(q), torch.empty(q.shape[:2], device=DEV))
    else:
        rows = b * n if case["op"] == "roundtrip" else sum(filled)
        state["out"] = tuple(torch.empty((rows, case["hkv"], case["hd"]), dtype=io, device=DEV) for _ in range(2))
    return state


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    from paper_2606_31580_amd import laser as L

    case, kv, out = state["case"], state["kv"], state["out"]
    if case["op"] == "roundtrip":
        L.laser_kv_write(kv, 0, state["runs"], *state["new"])
        L.laser_kv_read(kv, 0, state["runs"], *out)
    elif case["op"] == "read":
        L.laser_kv_read(kv, 0, state["whole"], *out)
    else:
        L.laser_attend(kv, 0, state["spans"], state["q"], out[0], lse=out[1], window=case["window"])
    return out


def _run_plain(state):
    case, kv, out = state["case"], state["kv"], state["out"]
    n, at = case["n"], 0
    for i, c in enumerate(state["ctx"]):
        if case["op"] == "roundtrip":
            part = slice(i * n, (i + 1) * n)
            kv.write(i, c, state["new"][0][part], state["new"][1][part])
            for o, x in zip(out, kv.read(i, c, n)):
                o[part] = x.to(o.dtype)
        elif case["op"] == "read":
            for o, x in zip(out, kv.read(i, 0, c)):
                o[at:at + c] = x.to(o.dtype)
            at += c
        else:
            k, v = kv.read(i, 0, c + n)
            _attend(case, c, state["q"][i * n:(i + 1) * n].float(), k, v, out[0][i * n:(i + 1) * n],
                    out[1][i * n:(i + 1) * n])
    return out


def _seen(case, c, n):
    """Which of the c + n positions each of the n new rows sees."""
    row = torch.arange(c, c + n, device=DEV)[:, None]
    t = torch.arange(c + n, device=DEV)[None, :]
    seen = t <= row
    return seen & (t > row - case["window"]) if case["window"] else seen


def _attend(case, c, q, k, v, o, lse):
    """softmax(q k / sqrt(hd)) v per query head, in q's type (float32 plain, float64 exact)."""
    n, group = q.shape[0], case["hq"] // case["hkv"]
    seen = _seen(case, c, n).repeat(group, 1)
    for h in range(case["hkv"]):
        qh = q[:, h * group:(h + 1) * group].transpose(0, 1).reshape(group * n, -1)
        s = (qh @ k[:, h].t()) / math.sqrt(case["hd"])
        s = s.masked_fill(~seen, -math.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        oh = (p @ v[:, h]) / total
        o[:, h * group:(h + 1) * group] = oh.reshape(group, n, -1).transpose(0, 1).to(o.dtype)
        lse[:, h * group:(h + 1) * group] = (torch.log(total) + top).reshape(group, n).t().to(lse.dtype)


def work(case):
    hq, hkv, hd, n, b = (case[k] for k in ("hq", "hkv", "hd", "n", "batch"))
    ctx = _contexts(case)
    io = 2 if case["io"] == "bf16" else 4
    place = 2 * hkv * (hd * ITEM[case["kv"]] + (4 if case["kv"] == "int8" else 0))  # K and V of one position
    dense = 2 * hkv * hd * io
    if case["op"] == "roundtrip":
        return {"bytes": b * n * (2 * place + 2 * dense), "flops": 0}
    if case["op"] == "read":
        return {"bytes": sum(ctx) * (place + dense), "flops": 0}
    w = case["window"]
    pairs = places = 0
    for c in ctx:
        places += min(c + n, w + n - 1) if w else c + n
        pairs += sum(min(c + i + 1, w) if w else c + i + 1 for i in range(n))
    return {"bytes": places * place + b * n * hq * (2 * hd * io + 4), "flops": 4 * hd * hq * pairs}


# ------------------------------------------------------------------------------ the definition in 64 bits

def _stood_for(kv, x):
    """The values that a cache of type `kv` keeps of x, in float64."""
    x = x.double()
    if kv == "int8":
        top = x.abs().amax(-1, keepdim=True)
        return torch.where(top > 0, torch.round(127.0 * x / torch.where(top > 0, top, 1.0)) * top / 127.0, 0.0)
    if kv == "fp8":  # three fraction bits above 2^-6, steps of 2^-9 below, at most 448
        e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))).clamp(-6, 8)
        step = torch.exp2(e - 3)
        return (torch.round(x / step) * step).clamp(-448.0, 448.0)
    return x  # (bf16 and fp32 caches are given rows of their own type, or round them once)


def exact(case, seed):
    ctx, held, new, q = _inputs(case, seed)
    n = case["n"]

    def kept(x):
        return _stood_for(case["kv"], x.to(STORE[case["kv"]]) if case["kv"] in ("bf16", "f32") else x)

    if case["op"] == "roundtrip":
        return tuple(kept(x) for x in new)
    if case["op"] == "read":
        return tuple(kept(x) for x in held)
    o = torch.empty(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device=DEV)
    at = 0
    group = case["hq"] // case["hkv"]
    for i, c in enumerate(ctx):
        k, v = (kept(x[at:at + c + n]) for x in held)
        at += c + n
        rows = q[i * n:(i + 1) * n].double()
        for h in range(case["hq"]):  # head by head, a few hundred rows at a time
            kh, vh = k[:, h // group], v[:, h // group]
            for r0 in range(0, n, 512):
                r1 = min(n, r0 + 512)
                s = rows[r0:r1, h] @ kh.t() * case["hd"] ** -0.5
                t = torch.arange(c + n, device=DEV)
                r = torch.arange(c + r0, c + r1, device=DEV)[:, None]
                hidden = (t > r) | (t + case["window"] <= r) if case["window"] else t > r
                s[hidden] = -math.inf
                z = torch.logsumexp(s, -1)
                o[i * n + r0:i * n + r1, h] = torch.exp(s - z[:, None]) @ vh
                lse[i * n + r0:i * n + r1, h] = z
    return o, lse
