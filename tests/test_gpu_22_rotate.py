"""laser_rotate and laser_kv_write_rotated against rotations in extended precision: both layouts, all and part of the head,
scaled frequencies, far and negative positions, every cache and row type, strided, unaligned and in-place rows, capture; and
a decode loop of rotated appends and attention over every cache type."""
import numpy as np
import pytest
import torch

from gpu_helpers import compare_logits, require_gpu
from mxfp4_ref import IO, cache, f64, kept, rows
from oracle import transformer as OT
from oracle.numerics import round_bf16
from paged_ref import attend
from paper_2606_31580_amd import laser as L
from paper_2606_31580_amd import synth
from paper_2606_31580_amd.configs import ModelShape
from test_gpu_16_kv_rows import stored_tol
from test_gpu_17_attend import queries, tolerance

pytestmark = pytest.mark.gpu
SCALED = [("plain", {}), ("linear", {"factor": 4.0}), ("base", {"factor": 3.0}),
          ("bands", {"factor": 8.0, "old_positions": 8192.0, "low": 1.0, "high": 4.0}),
          ("ramp", {"factor": 4.0, "old_positions": 4096.0, "low": 1.0, "high": 32.0})]


def turned(rope, x, pos):
    """Rows x [n, heads, hd] at positions pos [n], in float64 from extended precision; and the size of what is summed, and
    the largest angle of each element's pair."""
    r = rope.rot_dim
    f = np.array(list(rope.held), dtype=np.longdouble)
    angle = np.asarray(pos, dtype=np.longdouble)[:, None] * f
    c, s = (rope.amplitude * t(angle) for t in (np.cos, np.sin))
    first, second = (slice(0, r // 2), slice(r // 2, r)) if rope.layout == 0 else (slice(0, r, 2), slice(1, r, 2))
    x = np.asarray(x, dtype=np.longdouble)
    out, size, far = x.copy(), np.abs(x), np.zeros(x.shape)
    a, b, c, s = x[..., first], x[..., second], c[:, None], s[:, None]
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    for part in (first, second):
        size[..., part] = (np.abs(a) + np.abs(b)) * abs(rope.amplitude)
        far[..., part] = np.abs(angle[:, None]).astype(np.float64)
    return out.astype(np.float64), size.astype(np.float64), far


def rotated_tol(io, ref, size, far):
    """Half a step of the type (bf16: over fp32), and what the double angle is off by: three roundings of 2^-53 of it, and as
    much for sine, cosine and sums."""
    half = 2.0 ** -24 if io == "f32" else 2.0 ** -8 + 2.0 ** -24
    return half * np.abs(ref) + size * (far * 2.0 ** -51 + 2.0 ** -50)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads,hd,rot", [(28, 128, 128), (3, 64, 64), (2, 128, 96), (5, 64, 18), (1, 256, 256), (4, 80, 80), (3, 80, 32),
                                          (2, 2, 2), (7, 6, 4), (1, 250, 130)])
def test_rotate(heads, hd, rot, layout, io):
    require_gpu()
    rng = np.random.default_rng(hd + rot)
    for scaling, more in SCALED:
        rope = L.rope(hd, 1.0e4, rot, layout, scaling, **more)
        spec = [(1, 0, 1), (1, 14335, 1), (17, -7, 1), (33, 200000, 1), (40, -60000, -1), (5, 77, 0), (0, 3, 1), (16, 2 ** 31 - 9, 1), (3, -2 ** 31, -5)]
        runs, pos, at = [], [], 2
        for n, p, step in spec:
            runs.append(L.rotate_run(n, p, at, step))
            pos += [(at + i, p + step * i) for i in range(n)]
            at += n + 1
        x = rows(rng, at + 1, heads, hd, io)
        out = torch.full_like(x, 7.0)
        L.laser_rotate(rope, [runs[i] for i in rng.permutation(len(runs))], x, out)
        torch.cuda.synchronize()
        idx = np.array([i for i, _ in pos])
        ref, size, far = turned(rope, f64(x)[idx], [p for _, p in pos])
        got = f64(out)
        assert np.all(np.abs(got[idx] - ref) <= rotated_tol(io, ref, size, far)), scaling
        assert np.all(got[np.setdiff1d(np.arange(at + 1), idx)] == 7.0)
        inplace = x.clone()
        L.laser_rotate(rope, runs, inplace, inplace)
        torch.cuda.synchronize()
        assert torch.equal(inplace[idx], out[idx])


def test_as_the_model_rotates():
    """Half layout, whole heads, plain frequencies: the oracle's rotation, which the forward follows."""
    require_gpu()
    x = rows(np.random.default_rng(0), 300, 4, 128, "f32")
    out = torch.empty_like(x)
    L.laser_rotate(L.rope(128, 1.0e4), [L.rotate_run(300, 1000)], x, out)
    torch.cuda.synchronize()
    x64 = f64(x)
    ref = np.stack([OT.rope(x64[i], 1000 + i, 1.0e4) for i in range(300)])
    size = np.abs(x64) + np.abs(np.roll(x64, 64, -1))
    assert np.all(np.abs(f64(out) - ref) <= 2.0 ** -24 * np.abs(ref) + size * (1300 * 2.0 ** -50))


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_strides(io):
    """Queries inside a fused projection's output, heads before rows, one element off 16 bytes, a broadcast row; many runs."""
    require_gpu()
    rng = np.random.default_rng(3)
    n, heads, hd = 150, 3, 64
    rope = L.rope(hd, 1.0e4, layout="half")
    fused = rows(rng, n, 8, hd, io)
    sources = [fused[:, 4:7], rows(rng, heads, n, hd, io).transpose(0, 1), rows(rng, n, heads, hd + 1, io)[:, :, 1:],
               rows(rng, 1, heads, hd, io).expand(n, heads, hd)]
    pos = rng.integers(0, 100000, n)
    runs = [L.rotate_run(1, int(p), i) for i, p in enumerate(pos)]  # (more than one launch takes)
    for x in sources:
        outs = [torch.empty(n, heads, hd, dtype=IO[io], device="cuda"), torch.zeros(heads, n, hd, dtype=IO[io], device="cuda").transpose(0, 1),
                torch.zeros(n, heads, hd + 3, dtype=IO[io], device="cuda")[:, :, 3:]]
        ref, size, far = turned(rope, f64(x), pos)
        for out in outs:
            L.laser_rotate(rope, runs, x, out)
            torch.cuda.synchronize()
            assert np.all(np.abs(f64(out) - ref) <= rotated_tol(io, ref, size, far))
    other = fused.clone()
    L.laser_rotate(rope, runs, fused[:, 4:7], fused[:, 4:7])
    torch.cuda.synchronize()
    assert torch.equal(fused[:, :4], other[:, :4]) and torch.equal(fused[:, 7:], other[:, 7:])
    ref, size, far = turned(rope, f64(other[:, 4:7]), pos)
    assert np.all(np.abs(f64(fused[:, 4:7]) - ref) <= rotated_tol(io, ref, size, far))


def test_back_and_shifted():
    """Turned back, rows are what they were; turned by a constant, they are rows of the shifted positions."""
    require_gpu()
    rng = np.random.default_rng(4)
    rope = L.rope(128, 5.0e5, scaling="bands", factor=8.0, old_positions=8192.0, low=1.0, high=4.0)
    x = rows(rng, 500, 8, 128, "f32")
    y, z, s, direct = (torch.empty_like(x) for _ in range(4))
    L.laser_rotate(rope, [L.rotate_run(500, 9000)], x, y)
    L.laser_rotate(rope, [L.rotate_run(500, -9000, 0, -1)], y, z)
    L.laser_rotate(rope, [L.rotate_run(500, -2500, 0, 0)], y, s)
    L.laser_rotate(rope, [L.rotate_run(500, 6500)], x, direct)
    torch.cuda.synchronize()
    size = torch.roll(x.abs(), 64, -1) + x.abs()
    # two roundings of 2^-24 of values that pairs' sizes bound, the first one turned
    assert float(((z - x).abs() / size).max()) <= 3 * 2.0 ** -24
    assert float(((s - direct).abs() / size).max()) <= 4 * 2.0 ** -24


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("heads,hd,rot", [(8192, 256, 256), (8191, 250, 130)])
def test_most_heads(heads, hd, rot, io):
    """The most heads of a call; against 64 bits in 3 of its 19 rows."""
    require_gpu()
    rng = np.random.default_rng(1)
    rope = L.rope(hd, 1.0e4, rot)
    x = rows(rng, 1, heads, hd, io).expand(19, heads, hd).contiguous()
    out = torch.full_like(x, 7.0)
    L.laser_rotate(rope, [L.rotate_run(18, 5000, 1)], x, out)
    torch.cuda.synchronize()
    assert bool((out[0] == 7.0).all())
    for i in (1, 16, 18):
        ref, size, far = turned(rope, f64(x[i:i + 1]), [5000 + i - 1])
        assert np.all(np.abs(f64(out[i:i + 1]) - ref) <= rotated_tol(io, ref, size, far))


def test_most_rows():
    """More rows than a launch takes of a run: each is turned by its own position."""
    require_gpu()
    n = 2 ** 21 + 37
    rope = L.rope(2, inv_freq=[2.0 ** -12])
    x = rows(np.random.default_rng(2), 1, 1, 2, "f32").expand(n, 1, 2).contiguous()
    L.laser_rotate(rope, [L.rotate_run(n, -3, 0, 2)], x, x)
    torch.cuda.synchronize()
    idx = np.concatenate([np.arange(0, n, 9973), np.arange(2 ** 21 - 20, n)])
    ref, size, far = turned(rope, np.broadcast_to(f64(rows(np.random.default_rng(2), 1, 1, 2, "f32")), (len(idx), 1, 2)), [int(2 * i - 3) for i in idx])
    assert np.all(np.abs(f64(x[torch.from_numpy(idx).cuda()]) - ref) <= rotated_tol("f32", ref, size, far))


def test_odd_values():
    """Infinities and NaN stay within their pair; other dims, heads and rows are as without them."""
    require_gpu()
    for layout in ("half", "interleaved"):
        rope = L.rope(64, 1.0e4, 32, layout)
        x = rows(np.random.default_rng(5), 20, 2, 64, "f32")
        clean, out = torch.empty_like(x), torch.empty_like(x)
        L.laser_rotate(rope, [L.rotate_run(20, 50)], x, clean)
        x[3, 1, 4], x[7, 0, 50], x[9, 0, 20] = float("nan"), float("inf"), -float("inf")
        L.laser_rotate(rope, [L.rotate_run(20, 50)], x, out)
        torch.cuda.synchronize()
        same = torch.isfinite(out)
        assert torch.equal(out[same], clean[same])
        pair = {"half": (lambda d: d + 16 if d < 16 else d - 16), "interleaved": (lambda d: d ^ 1)}[layout]
        bad = {(3, 1, 4), (3, 1, pair(4)), (7, 0, 50), (9, 0, 20), (9, 0, pair(20))}
        assert {tuple(int(i) for i in t) for t in (~same).nonzero()} == bad
        assert out[7, 0, 50] == float("inf")


RUNS = [(0, 0, 1), (0, 1, 2), (0, 3, 1), (1, 5, 27), (2, 0, 16), (3, 30, 33), (4, 0, 250), (5, 15, 2)]
LENS = [4, 40, 16, 63, 250, 17]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("layout,scaling,part", [("half", 0, 1.0), ("interleaved", 3, 1.0), ("half", 4, 0.75), ("interleaved", 1, 0.3)])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kind", ["mxfp4", "int8", "fp8", "bf16", "f32"])
def test_write_rotated(kind, hd, layout, scaling, part, io):
    """Keys turned and kept in the cache's type, rounded once from the turned value: exactly what the definition gives (a
    double sum lies on the wrong side of a border once in some 2^28 elements); INT8 from fp32, so next to a half either way.
    Values are what laser_kv_write keeps, queries turned into their rows, other positions and rows are left alone."""
    rng = np.random.default_rng(11)
    hkv, hq = (2, 4) if hd == 64 else (3, 6)
    kv, plain = (cache(hq, hkv, hd, kind=kind) for _ in range(2))
    name, more = SCALED[scaling]
    rope = L.rope(hd, 1.0e4, 2 * round(part * hd / 2), layout, name, **more)
    row0, at = [], 3
    for _, _, n in RUNS:
        row0.append(at)
        at += n + 1
    k, v, q = (rows(rng, at + 2, h, hd, io, 0.5) for h in (hkv, hkv, hq))
    old = [torch.full((n, hkv, hd), 0.5, dtype=IO[io], device="cuda") for n in LENS]
    for c in (kv, plain):
        for s, n in enumerate(LENS):
            c.add_seq(s, n)
            L.laser_kv_write(c, 1, [L.kv_run(s, 0, n)], old[s], old[s])
    runs = [L.kv_run(s, p, n, r) for (s, p, n), r in zip(RUNS, row0)]
    q_out = torch.full_like(q, 7.0)
    L.laser_kv_write_rotated(kv, 1, rope, runs, k, v, q, q_out)
    L.laser_kv_write(plain, 1, runs, k, v)
    back = [[torch.empty(n, hkv, hd, device="cuda") for _ in range(2)] for n in LENS]
    want_v = [[torch.empty(n, hkv, hd, device="cuda") for _ in range(2)] for n in LENS]
    for s, n in enumerate(LENS):
        L.laser_kv_read(kv, 1, [L.kv_run(s, 0, n)], *back[s])
        L.laser_kv_read(plain, 1, [L.kv_run(s, 0, n)], *want_v[s])
    torch.cuda.synchronize()
    inside = np.zeros(at + 2, dtype=bool)
    seen = [np.zeros(n, dtype=bool) for n in LENS]
    for (s, p, n), r in zip(RUNS, row0):
        pos = np.arange(p, p + n)
        inside[r:r + n] = True
        seen[s][p:p + n] = True
        ref, size, far = turned(rope, f64(q)[r:r + n], pos)
        assert np.all(np.abs(f64(q_out)[r:r + n] - ref) <= rotated_tol(io, ref, size, far))
        ref, _, _ = turned(rope, f64(k)[r:r + n], pos)
        got = f64(back[s][0])[p:p + n]
        if kind == "int8":
            y = ref.astype(np.float32).astype(np.float64)
            assert np.all(np.abs(got - kept(kind, y)) <= stored_tol(kind, "f32", kept(kind, y), y))
        else:
            assert np.array_equal(got, kept(kind, ref) if kind != "f32" else ref.astype(np.float32).astype(np.float64))
        assert torch.equal(back[s][1][p:p + n], want_v[s][1][p:p + n])
    assert np.all(f64(q_out)[~inside] == 7.0)
    for s in range(len(LENS)):
        for x in back[s]:
            assert np.allclose(f64(x)[~seen[s]], 0.5, rtol=2.0 ** -22, atol=0)
    assert torch.equal(kv.v_pool, plain.v_pool)
    # without queries, and one position at a time: the same bytes; queries in place
    one = cache(hq, hkv, hd, kind=kind)
    for s, n in enumerate(LENS):
        one.add_seq(s, n)
        L.laser_kv_write(one, 1, [L.kv_run(s, 0, n)], old[s], old[s])
    L.laser_kv_write_rotated(one, 1, rope, [L.kv_run(s, p + i, 1, r + i) for (s, p, n), r in zip(RUNS, row0) for i in range(n)], k, v)
    inplace = q.clone()
    L.laser_kv_write_rotated(kv, 1, rope, runs, k, v, inplace, inplace)
    torch.cuda.synchronize()
    assert torch.equal(one.k_pool, kv.k_pool) and torch.equal(one.v_pool, kv.v_pool)
    idx = torch.from_numpy(np.nonzero(inside)[0]).cuda()
    assert torch.equal(inplace[idx], q_out[idx])


@pytest.mark.parametrize("kind", ["mxfp4", "int8", "bf16"])
def test_write_rotated_strides(kind):
    """K, V and Q as parts of one projection's output, rows of different alignments, a row written to two sequences."""
    rng = np.random.default_rng(6)
    hq, hkv, hd, n = 4, 2, 64, 37
    rope = L.rope(hd, 1.0e4, layout="interleaved")
    fused = rows(rng, n, hq + 2 * hkv, hd, "bf16", 0.5)
    q, k, v = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    odd = rows(rng, n, hkv, hd + 1, "bf16", 0.5)[:, :, 1:]
    for ks, vs in ((k, v), (odd, v), (k, odd), (k[:1].expand(n, hkv, hd), v)):
        kv = cache(hq, hkv, hd, kind=kind)
        kv.add_seq(0, n)
        kv.add_seq(1, n + 3)
        L.laser_kv_write_rotated(kv, 0, rope, [L.kv_run(0, 0, n), L.kv_run(1, 3, n)], ks, vs)
        for s, p in ((0, 0), (1, 3)):
            out = [torch.zeros(n, hkv, hd, device="cuda") for _ in range(2)]
            L.laser_kv_read(kv, 0, [L.kv_run(s, p, n)], *out)
            torch.cuda.synchronize()
            y, _, _ = turned(rope, f64(ks), np.arange(p, p + n))
            y = y.astype(np.float32).astype(np.float64) if kind == "int8" else y
            assert np.all(np.abs(f64(out[0]) - kept(kind, y)) <= (stored_tol(kind, "f32", kept(kind, y), y) if kind == "int8" else 0))
            assert np.all(np.abs(f64(out[1]) - kept(kind, f64(vs))) <= (stored_tol(kind, "f32", kept(kind, f64(vs)), f64(vs)) if kind == "int8" else 0))
    whole = fused.clone()  # the queries in place, K and V of the same array untouched
    kv = cache(hq, hkv, hd, kind=kind)
    kv.add_seq(0, n)
    L.laser_kv_write_rotated(kv, 0, rope, [L.kv_run(0, 0, n)], whole[:, hq:hq + hkv], whole[:, hq + hkv:], whole[:, :hq], whole[:, :hq])
    torch.cuda.synchronize()
    assert torch.equal(whole[:, hq:], fused[:, hq:])
    ref, size, far = turned(rope, f64(q), np.arange(n))
    assert np.all(np.abs(f64(whole[:, :hq]) - ref) <= rotated_tol("bf16", ref, size, far))


@pytest.mark.parametrize("kind", ["mxfp4", "int8", "fp8", "bf16", "f32"])
def test_layers_of_a_callers_own(kind):
    """A prompt and some decoded tokens of two sequences, layer by layer: rotated appends and attention, against attention over
    what the cache holds, which is what the definition keeps of the turned keys."""
    rng = np.random.default_rng(9)
    hq, hkv, hd, io = 8, 2, 64, "f32" if kind == "f32" else "bf16"
    kv = cache(hq, hkv, hd, kind=kind)
    rope = L.rope(hd, 1.0e4, scaling="linear", factor=2.0)
    held = {}
    for s in (0, 1):
        kv.add_seq(s, 0)
    for step, grow in enumerate([(70, 33), (1, 1), (1, 1), (3, 1), (1, 0), (40, 1)]):
        start = [kv.seq_len(s) for s in (0, 1)]
        runs = [L.kv_run(s, start[s], g, s * grow[0]) for s, g in enumerate(grow)]
        spans = [L.attend_span(s, g, start[s], row0=s * grow[0]) for s, g in enumerate(grow)]
        for s, g in enumerate(grow):
            kv.append(s, g)
        for layer in (0, 1):
            n = sum(grow)
            k, v = (rows(rng, n, hkv, hd, io, 0.3) for _ in range(2))
            q = queries(rng, n, hq, hd, io)
            qr, o = torch.empty_like(q), torch.empty_like(q)
            L.laser_kv_write_rotated(kv, layer, rope, runs, k, v, q, qr)
            L.laser_attend(kv, layer, spans, qr, o)
            torch.cuda.synchronize()
            for s, g in enumerate(grow):
                r = slice(s * grow[0], s * grow[0] + g)
                if g == 0:
                    continue
                pos = np.arange(start[s], start[s] + g)
                y, _, _ = turned(rope, f64(k)[r], pos)
                qy, qsize, qfar = turned(rope, f64(q)[r], pos)
                assert np.all(np.abs(f64(qr)[r] - qy) <= rotated_tol(io, qy, qsize, qfar))
                new = (kept(kind, y.astype(np.float32).astype(np.float64) if kind in ("int8", "f32") else y), kept(kind, f64(v)[r]))
                had = held.get((s, layer))
                K, V = held[(s, layer)] = new if had is None else tuple(np.concatenate(p) for p in zip(had, new))
                back = [torch.empty(K.shape[0], hkv, hd, device="cuda") for _ in range(2)]
                L.laser_kv_read(kv, layer, [L.kv_run(s, 0, K.shape[0])], *back)
                torch.cuda.synchronize()
                for got, ref in zip(back, (K, V)):
                    assert np.all(np.abs(f64(got) - ref) <= (1.01 * np.abs(ref).max(-1, keepdims=True) / 127 if kind == "int8" else 0))
                K, V = (f64(x) for x in back)
                ref, _ = attend(f64(qr)[r], K, V, start[s], hd ** -0.5)
                assert np.all(np.abs(f64(o)[r] - ref) <= tolerance(io, ref, V, f64(qr)[r], K, hd ** -0.5)), (step, s, layer)


def test_captured():
    """Rotated append, attention and rotation in one graph, replayed on other rows between eager calls."""
    rng = np.random.default_rng(21)
    hq, hkv, hd, n = 8, 2, 128, 19
    kv = cache(hq, hkv, hd, pages=60, per_seq=40)
    rope = L.rope(hd, 1.0e4)
    kv.add_seq(0, 500)
    old = [rows(rng, 500, hkv, hd, "bf16") for _ in range(2)]
    L.laser_kv_write(kv, 1, [L.kv_run(0, 0, 500)], *old)
    runs, spans = [L.kv_run(0, 500 - n, n)], [L.attend_span(0, n, 500 - n)]
    new = [tuple(rows(rng, n, h, hd, "bf16") for h in (hkv, hkv, hq)) for _ in range(3)]
    k, v, q = (x.clone() for x in new[0])
    qr, o, turn = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    ws = torch.empty(max(16, L.laser_attend_workspace(kv, spans)), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.laser_kv_write_rotated(kv, 1, rope, runs, k, v, q, qr)
        L.laser_attend(kv, 1, spans, qr, o, workspace=ws)
        L.laser_rotate(rope, [L.rotate_run(n, 500 - n)], q, turn)
    for i in (0, 1, 2, 1):
        for dst, src in zip((k, v, q), new[i]):
            dst.copy_(src)
        g.replay()
        torch.cuda.synchronize()
        pools = kv.k_pool.clone(), kv.v_pool.clone()
        e = [torch.zeros_like(q) for _ in range(3)]
        L.laser_kv_write_rotated(kv, 1, rope, runs, *new[i], e[0])
        L.laser_attend(kv, 1, spans, e[0], e[1])
        L.laser_rotate(rope, [L.rotate_run(n, 500 - n)], new[i][2], e[2])
        torch.cuda.synchronize()
        assert torch.equal(e[0], qr) and torch.equal(e[1], o) and torch.equal(e[2], turn) and torch.equal(turn, qr)
        assert torch.equal(pools[0], kv.k_pool) and torch.equal(pools[1], kv.v_pool)


def test_on_another_stream():
    require_gpu()
    x = rows(np.random.default_rng(2), 3000, 8, 128, "bf16")
    rope = L.rope(128)
    here, there = torch.empty_like(x), torch.empty_like(x)
    L.laser_rotate(rope, [L.rotate_run(3000, 0)], x, here)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    L.laser_rotate(rope, [L.rotate_run(3000, 0)], x, there, stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(here, there)
    with pytest.raises(ValueError):
        L.laser_rotate(rope, [L.rotate_run(1, 0)], x.cpu(), here)
    with pytest.raises(ValueError):
        L.laser_rotate(rope, [L.rotate_run(1, 0)], x[:, :4], here)
    with pytest.raises(TypeError):
        L.laser_rotate(rope, [L.kv_run(0, 0, 1)][:1] + [1], x, here)


@pytest.mark.parametrize("kind", ["mxfp4", "int8", "fp8"])
@pytest.mark.parametrize("hd", [64, 128])
def test_two_calls_at_once(kind, hd):
    """Every other position of the same pages from two streams at once, bytes of whose blocks lie side by side: as one call."""
    rng = np.random.default_rng(8)
    hkv, n = 2, 120
    rope = L.rope(hd, 1.0e4)
    k, v = (rows(rng, n, hkv, hd, "bf16") for _ in range(2))
    one, two = (cache(4, hkv, hd, kind=kind) for _ in range(2))
    for c in (one, two):
        c.add_seq(0, n)
        L.laser_kv_write(c, 1, [])
    L.laser_kv_write_rotated(one, 1, rope, [L.kv_run(0, 0, n)], k, v)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for at in range(0, n, 40):
        for i, s in enumerate(streams):
            L.laser_kv_write_rotated(two, 1, rope, [L.kv_run(0, p, 1, p) for p in range(at + i, at + 40, 2)], k, v, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(one.k_pool, two.k_pool) and torch.equal(one.v_pool, two.v_pool)


@pytest.mark.parametrize("name,more", SCALED[1:], ids=[s[0] for s in SCALED[1:]])
def test_model_with_scaled_positions(monkeypatch, name, more):
    """A prompt and decode steps of a model with scaled frequencies against the oracle that turns by the same angles, then a
    position of the caller's own among the forward's keys: laser_kv_write_rotated keeps the bytes that a forward would."""
    require_gpu()
    shape = ModelShape("rope-scaled", 2, 256, 4, 2, 64, 688, 2048, False, False, "f32", 1.0e4, 1.0e-5)
    rope = L.rope(64, 1.0e4, scaling=name, **more)
    f = np.array(list(rope.held))
    w = synth.make_weights(shape)
    model = L.Model(shape, {k: v.cuda() for k, v in w.items()}, max_rows=8, max_positions=512, rope=rope)
    plain_rope = OT.rope

    def scaled(x, pos, theta):
        a = pos * f
        lo, hi = x[..., :32], x[..., 32:]
        return rope.amplitude * np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], axis=-1)

    assert np.allclose(scaled(np.ones(64), 0, 0), rope.amplitude * plain_rope(np.ones(64), 0, 1.0e4))
    monkeypatch.setattr(OT, "rope", scaled)
    orc = OT.DecoderOracle(shape, {k: synth.to_numpy(v) for k, v in w.items()})
    kv = L.KVCache(model, 20, 1, 20, poison=True)
    kv.add_seq(0, 0)
    st = OT.SeqState(shape, 512)
    toks = synth.make_tokens(41, shape.vocab, 5)
    logits = torch.zeros(1, shape.vocab, device="cuda")
    L.laser_prefill(model, kv, 0, toks[:40].cuda(), logits[0])
    torch.cuda.synchronize()
    for t in toks[:40]:
        ref = orc.decode_token(st, int(t))
    compare_logits(logits[0].cpu().numpy(), ref, "prompt")
    nxt, p = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda")
    L.laser_decode_step(model, kv, [0], toks[40:].cuda(), nxt, p, logits)
    torch.cuda.synchronize()
    compare_logits(logits[0].cpu().numpy(), orc.decode_token(st, int(toks[40])), "decode")
    # the forward's keys turned back, and written again by laser_kv_write_rotated
    for layer in range(2):
        k, v = (torch.empty(41, 2, 64, device="cuda") for _ in range(2))
        L.laser_kv_read(kv, layer, [L.kv_run(0, 0, 41)], k, v)
        raw, again = torch.empty_like(k), [torch.empty_like(k) for _ in range(2)]
        back = L.rope(64, inv_freq=list(f), amplitude=1.0 / rope.amplitude)
        L.laser_rotate(back, [L.rotate_run(41, 0, 0, -1)], k, raw)
        L.laser_kv_write_rotated(kv, layer, rope, [L.kv_run(0, 0, 41)], raw, v)
        L.laser_kv_read(kv, layer, [L.kv_run(0, 0, 41)], *again)
        torch.cuda.synchronize()
        # (three fp32 roundings of values that the pair's size bounds)
        size = k.abs() + torch.roll(k.abs(), 32, -1)
        assert bool(((again[0] - k).abs() <= 4 * 2.0 ** -24 * size).all()) and torch.equal(again[1], v)
