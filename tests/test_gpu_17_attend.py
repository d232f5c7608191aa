"""laser_attend (attention of a caller's rows over the paged cache) against float64, for every cache and
row type, one row to hundreds per sequence, ragged lengths, windows and key ranges, rows that see
nothing, infinities and NaN in unseen places, strided arrays, capture, and parts joined by their lse."""
import math

import numpy as np
import pytest
import torch

import test_gpu_16_kv_rows
from paged_ref import attend, kept
from paper_2606_31580_amd import laser as L
from test_gpu_16_kv_rows import IO, cache, f64, rows

pytestmark = pytest.mark.gpu
ROWS, TILES = 1, 2  # laser_model_set_attend_kernel: row kernels only; the tile kernel above 64 columns


@pytest.fixture(autouse=True)
def kernels(request):
    """Runs a test with the kernels that its `kernels` parameter names (by work: 0); models are shared, so it is set back."""
    from test_gpu_16_kv_rows import _models
    mode = request.param if hasattr(request, "param") else 0
    test_gpu_16_kv_rows.MODE = mode
    for m in _models.values():
        m.set_attend_kernel(mode)
    yield mode
    test_gpu_16_kv_rows.MODE = 0
    for m in _models.values():
        m.set_attend_kernel(0)


both = pytest.mark.parametrize("kernels", [ROWS, TILES], indirect=True, ids=["rows", "tiles"])


def fill(kv, kind, lens, hkv, hd, seed, layer=1, spread=1.0):
    """Sequences of these lengths in `layer`; their K and V as the cache keeps them (float64)."""
    rng = np.random.default_rng(seed)
    held = []
    for s, n in enumerate(lens):
        kv.add_seq(s, n)
        k, v = (torch.from_numpy((rng.standard_normal((n, hkv, hd)) * spread).astype(np.float32))
                .to(torch.float32 if kind == "f32" else torch.bfloat16).cuda() for _ in range(2))
        if n:
            L.laser_kv_write(kv, layer, [L.kv_run(s, 0, n)], k, v)
        held.append((kept(kind, f64(k)), kept(kind, f64(v))))
    return held


def queries(rng, n, hq, hd, io):
    return torch.from_numpy(rng.standard_normal((n, hq, hd)).astype(np.float32)).to(IO[io]).cuda()


def tolerance(io, ref, v, q, k, scale):
    """bf16 rows: the softmax weights are rounded to bf16 and so is the output.  A bf16 number in [1, 2) is a multiple
    of 2^-7, so rounding to nearest is off by at most 2^-8 = finfo(bfloat16).eps / 2 of the number: with sum w = 1,
    |sum (w' - w) v| <= 2^-8 sum w |v| <= 2^-8 max |v|, and the output by 2^-8 of itself.  Both: fp32 scores are off by at most hd roundings of
    their terms, 2^-24 hd scale max|q| max|k| sqrt(hd)-ish; four times the root-sum is taken, which moves every
    weight by that factor.  Sums over up to some thousand keys add 2^-24 sqrt(keys), inside the constant."""
    top = np.nanmax(np.abs(v)) if v.size else 1.0
    terms = abs(scale) * np.abs(q).max() * np.abs(k).max() * math.sqrt(q.shape[-1]) if k.size else 0.0
    tol = (4 * 2.0 ** -24 * terms + 64 * 2.0 ** -24) * top
    if io == "bf16":
        tol += 2.0 ** -8 * top + 2.0 ** -8 * np.abs(ref)
    return tol


def check(kv, kind, io, held, spans, q, scale=None, causal=True, window=0, layer=1, o=None):
    """Runs laser_attend and compares every row of every span; rows outside keep what they hold."""
    hd = q.shape[-1]
    o = torch.full_like(q, 5.0) if o is None else o
    lse = torch.full(q.shape[:2], 5.0, device="cuda")
    L.laser_attend(kv, layer, spans, q, o, lse=lse, scale=scale, causal=causal, window=window)
    torch.cuda.synchronize()
    scale = hd ** -0.5 if scale is None else scale
    go, gl, q64 = f64(o), lse.cpu().numpy().astype(np.float64), f64(q)
    seen = np.zeros(q.shape[0], dtype=bool)
    for s in spans:
        k, v = held[s.seq]
        end = k.shape[0] if s.kv_end == -1 else s.kv_end
        r = slice(s.row0, s.row0 + s.n)
        seen[r] = True
        ro, rl = attend(q64[r], k, v, s.pos, scale, causal, window, s.kv_begin, end)
        assert np.array_equal(np.isnan(go[r]), np.isnan(ro)), (s.seq, s.n, s.pos)
        assert np.array_equal(np.isinf(gl[r]), np.isinf(rl)) and np.array_equal(np.isnan(gl[r]), np.isnan(rl))
        if s.n == 0 or k.size == 0:
            assert np.all(go[r] == 0)
            continue
        fin = np.isfinite(ro)
        kf = np.where(np.isfinite(k), k, 0)
        tol = tolerance(io, ro, np.where(np.isfinite(v), v, 0), q64[r], kf, scale)
        err = np.abs(go[r] - ro)
        assert np.all(err[fin] <= np.broadcast_to(tol, err.shape)[fin]), (s.seq, s.n, s.pos, err[fin].max())
        lf = np.isfinite(rl)
        terms = abs(scale) * np.abs(q64[r]).max() * np.abs(kf).max() * math.sqrt(hd)
        # lse: the same score error, and 2^-23 of itself for the two roundings and the logarithm
        assert np.all(np.abs(gl[r][lf] - rl[lf]) <= (4 * 2.0 ** -24 * terms + 64 * 2.0 ** -24) + 2.0 ** -22 * np.abs(rl[lf]))
    assert np.all(go[~seen] == 5.0) and np.all(gl[~seen] == 5.0)
    return o, lse


@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 64), (7, 1, 128), (3, 3, 128), (32, 2, 64)])
@pytest.mark.parametrize("kind,io", [("int8", "bf16"), ("int8", "f32"), ("fp8", "bf16"), ("fp8", "f32"), ("bf16", "bf16"),
                                     ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_decode_rows(kind, io, hq, hkv, hd):
    """One row per sequence: lengths around page and pair edges, up to some that split."""
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 64, 129, 500, 1333, 0]
    kv = cache(kind, hq, hkv, hd, pages=200, seqs=len(lens), per_seq=100)
    held = fill(kv, kind, lens, hkv, hd, 5)
    q = queries(np.random.default_rng(6), len(lens) + 2, hq, hd, io)
    check(kv, kind, io, held, [L.attend_span(s, 1, max(n - 1, 0), row0=s + 1) for s, n in enumerate(lens)], q)


@both
@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 64), (7, 1, 128), (3, 3, 128)])
@pytest.mark.parametrize("kind,io", [("int8", "bf16"), ("int8", "f32"), ("fp8", "bf16"), ("bf16", "bf16"), ("bf16", "f32"),
                                     ("f32", "f32")])
def test_chunks(kind, io, hq, hkv, hd):
    """Chunks of 2 to some hundred rows behind contexts of every kind, in one call; the whole sequence as one chunk too."""
    lens = [2, 20, 37, 64, 100, 257, 600, 300]
    rowsn = [2, 5, 37, 9, 70, 200, 3, 300]
    kv = cache(kind, hq, hkv, hd, pages=200, seqs=len(lens), per_seq=100)
    held = fill(kv, kind, lens, hkv, hd, 7)
    q = queries(np.random.default_rng(8), sum(rowsn), hq, hd, io)
    spans, at = [], 0
    for s, (n, r) in enumerate(zip(lens, rowsn)):
        spans.append(L.attend_span(s, r, n - r, row0=at))
        at += r
    check(kv, kind, io, held, spans, q)


@both
@pytest.mark.parametrize("kind,io", [("int8", "bf16"), ("bf16", "f32"), ("fp8", "bf16")])
@pytest.mark.parametrize("causal,window", [(True, 1), (True, 16), (True, 77), (False, 0), (False, 40)])
def test_masks_and_ranges(kind, io, causal, window):
    """Windows, key ranges that start and end inside pages, rows in front of and behind all their keys."""
    hq, hkv, hd = 6, 2, 64
    lens = [300, 300, 90, 300, 40]
    kv = cache(kind, hq, hkv, hd, pages=100, seqs=5, per_seq=40)
    held = fill(kv, kind, lens, hkv, hd, 9)
    spans = [L.attend_span(0, 40, 260, row0=0), L.attend_span(1, 33, 100, row0=40, kv_begin=37, kv_end=211),
             L.attend_span(2, 20, 5, row0=73, kv_begin=13, kv_end=13), L.attend_span(3, 25, 0, row0=93, kv_begin=11),
             L.attend_span(4, 30, 1000, row0=118), L.attend_span(0, 1, 150, row0=148, kv_begin=149, kv_end=151),
             L.attend_span(0, 100, 120, row0=149, kv_begin=160)]
    q = queries(np.random.default_rng(10), 250, hq, hd, io)
    check(kv, kind, io, held, spans, q, causal=causal, window=window)


@both
@pytest.mark.parametrize("kind,io", [("bf16", "bf16"), ("bf16", "f32"), ("fp8", "bf16"), ("int8", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("n", [3, 40, 150])
def test_odd_values_in_unseen_places(kind, io, n):
    """Infinities and NaN in K and V: rows that do not see the position are as if it were not there."""
    hq, hkv, hd, length = 4, 2, 64, 330
    kv = cache(kind, hq, hkv, hd, pages=60, seqs=2, per_seq=30)
    held = fill(kv, kind, [length], hkv, hd, 12)
    k, v = held[0]
    # V odd at some positions of the chunk, K odd at others, one head each
    bad_v, bad_k = length - n + n // 2, length - 1
    for pos, is_v, val, head in ((bad_v, True, np.nan, 0), (bad_k, False, np.inf, 1), (length - 1, True, np.inf, 0)):
        src = torch.zeros(1, hkv, hd)
        src[0] = torch.from_numpy((v if is_v else k)[pos].astype(np.float32))
        src[0, head, 5] = val
        other = torch.from_numpy((k if is_v else v)[pos:pos + 1].astype(np.float32))
        t = torch.float32 if kind == "f32" else torch.bfloat16
        a, b = (other, src) if is_v else (src, other)
        L.laser_kv_write(kv, 1, [L.kv_run(0, pos, 1)], a.to(t).cuda(), b.to(t).cuda())
        k[pos], v[pos] = kept(kind, f64(a.to(t)))[0], kept(kind, f64(b.to(t)))[0]
    q = queries(np.random.default_rng(13), n, hq, hd, io).abs()
    o = torch.full_like(q, 5.0)
    L.laser_attend(kv, 1, [L.attend_span(0, n, length - n)], q, o)
    torch.cuda.synchronize()
    g = f64(o)
    last = 1 if n > 1 else 0
    ref, _ = attend(f64(q), k, v, length - n, hd ** -0.5)
    clean = [i for i in range(n) if length - n + i < bad_v]
    assert clean or n // 2 == 0
    # rows in front of every odd position: untouched
    assert np.isfinite(g[clean]).all()
    tol = tolerance(io, ref[clean], np.where(np.isfinite(v), v, 0), f64(q), np.where(np.isfinite(k), k, 0), hd ** -0.5)
    assert np.all(np.abs(g[clean] - ref[clean]) <= tol)
    # rows that see the NaN in V: heads of kv head 0 are NaN there and only there (an INT8 vector: all of it)
    for i in range(n // 2, n - last):
        bad = np.isnan(g[i, 0:2])
        assert bad.all() if kind == "int8" else (bad[:, 5].all() and bad.sum() == 2), i
        assert np.isfinite(g[i, 2:4]).all()
    # window rows behind it do not see it either
    o2 = torch.full_like(q, 5.0)
    L.laser_attend(kv, 1, [L.attend_span(0, n, length - n)], q, o2, window=n // 2)
    torch.cuda.synchronize()
    g2, (ref2, _) = f64(o2), attend(f64(q), k, v, length - n, hd ** -0.5, window=n // 2)
    assert np.array_equal(np.isnan(g2[:n - last]), np.isnan(ref2[:n - last]))


def test_poisoned_neighbours():
    """Slots past the length, pages of other sequences and other layers hold NaN bytes."""
    for kind in ("bf16", "int8", "fp8"):
        kv = cache(kind, 4, 2, 64, pages=40, seqs=3, per_seq=20)
        held = fill(kv, kind, [17, 33, 50], 2, 64, 14)
        q = queries(np.random.default_rng(15), 12, 4, 64, "bf16")
        check(kv, kind, "bf16", held, [L.attend_span(0, 5, 12), L.attend_span(1, 1, 32, row0=5), L.attend_span(2, 6, 44, row0=6)], q)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_large_scores(io):
    """Scores of some hundreds of either sign, growing along the keys (the running maximum moves at every page)."""
    hq, hkv, hd, n = 4, 2, 64, 700
    kv = cache("bf16", hq, hkv, hd, pages=60, seqs=1, per_seq=60)
    kv.add_seq(0, n)
    rng = np.random.default_rng(16)
    k = rng.standard_normal((n, hkv, hd)) * 0.1 + np.linspace(-4, 4, n)[:, None, None]
    k, v = (torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda() for x in (k, rng.standard_normal((n, hkv, hd))))
    L.laser_kv_write(kv, 1, [L.kv_run(0, 0, n)], k, v)
    q = torch.ones(3, hq, hd, dtype=IO[io], device="cuda") * torch.tensor([1.0, -1.0, 0.5]).to(IO[io]).cuda()[:, None, None]
    check(kv, "bf16", io, [(f64(k), f64(v))], [L.attend_span(0, 3, n - 3)], q, scale=2.0)


def test_strides_alias_and_unaligned():
    """Queries inside a fused projection's output, o as q itself, heads before rows, rows off 16 bytes."""
    hq, hkv, hd, n = 4, 2, 64, 21
    rng = np.random.default_rng(17)
    kv = cache("int8", hq, hkv, hd, pages=40, seqs=1, per_seq=40)
    held = fill(kv, "int8", [500], hkv, hd, 18)
    spans = [L.attend_span(0, n, 500 - n)]
    for io in ("bf16", "f32"):
        ref, _ = check(kv, "int8", io, held, spans, queries(rng, n, hq, hd, io))
        base = queries(rng, n, hq, hd, io)
        want, _ = check(kv, "int8", io, held, spans, base)
        fused = torch.zeros(n, hq + 2 * hkv, hd, dtype=IO[io], device="cuda")
        fused[:, :hq] = base
        firsts = torch.full((hq, n, hd + 1), 5.0, dtype=IO[io], device="cuda").transpose(0, 1)[:, :, 1:]
        got, _ = check(kv, "int8", io, held, spans, fused[:, :hq], o=firsts)
        assert torch.equal(got, want)
        odd = torch.zeros(n, hq, hd + 1, dtype=IO[io], device="cuda")[:, :, :hd]
        odd.copy_(base)
        L.laser_attend(kv, 1, spans, odd, odd)  # in place
        assert torch.equal(odd, want)


def test_parts_joined_by_lse():
    """Outputs over two ranges of keys, weighted by their lse, are the output over all."""
    hq, hkv, hd = 6, 2, 64
    kv = cache("int8", hq, hkv, hd, pages=40, seqs=1, per_seq=40)
    fill(kv, "int8", [411], hkv, hd, 19)
    q = queries(np.random.default_rng(20), 30, hq, hd, "f32")
    outs = []
    for b, e in ((0, 411), (0, 203), (203, 411)):
        o, lse = torch.empty_like(q), torch.empty(30, hq, device="cuda")
        L.laser_attend(kv, 1, [L.attend_span(0, 30, 381, kv_begin=b, kv_end=e)], q, o, lse=lse)
        outs.append((o.double(), lse.double()))
    (o, lse), (o1, l1), (o2, l2) = outs
    joined = torch.logaddexp(l1, l2)
    both = o1 * torch.exp(l1 - joined)[..., None] + o2 * torch.exp(l2 - joined)[..., None]
    assert float((both - o).abs().max()) <= 1e-5 and float((joined - lse).abs().max()) <= 1e-5


def test_write_attend_loop_with_fork():
    """As it is used: a prompt written and attended as one chunk, tokens appended and attended one by one, a
    fork that goes its own way beside the request, and a position taken back."""
    hq, hkv, hd = 7, 1, 128
    rng = np.random.default_rng(22)
    kv = cache("int8", hq, hkv, hd, pages=40, seqs=3, per_seq=20)
    held = fill(kv, "int8", [77], hkv, hd, 23)
    seqs = {0: held[0]}
    check(kv, "int8", "bf16", seqs, [L.attend_span(0, 77, 0)], queries(rng, 77, hq, hd, "bf16"))
    for step in range(6):
        if step == 2:
            kv.fork(0, 2)
            seqs[2] = tuple(x.copy() for x in seqs[0])
        new = rows(rng, len(seqs), hkv, hd, "bf16"), rows(rng, len(seqs), hkv, hd, "bf16")
        runs = []
        for i, s in enumerate(seqs):
            n = seqs[s][0].shape[0]
            kv.append(s, 1)
            runs.append(L.kv_run(s, n, 1, i))
            seqs[s] = tuple(np.concatenate([x, kept("int8", f64(y[i:i + 1]))]) for x, y in zip(seqs[s], new))
        L.laser_kv_write(kv, 1, runs, *new)
        spans = [L.attend_span(s, 1, seqs[s][0].shape[0] - 1, row0=i) for i, s in enumerate(seqs)]
        check(kv, "int8", "bf16", seqs, spans, queries(rng, len(seqs), hq, hd, "bf16"))
    kv.truncate(2, 80)
    seqs[2] = tuple(x[:80] for x in seqs[2])
    check(kv, "int8", "bf16", seqs, [L.attend_span(2, 3, 77)], queries(rng, 3, hq, hd, "bf16"))


def test_many_spans_streams_and_capture():
    """More spans than a launch takes, on a stream of their own; captured and replayed with other queries beside
    an eager call with its own workspace; equal bits each time."""
    hq, hkv, hd = 4, 2, 64
    rng = np.random.default_rng(24)
    lens = [int(x) for x in rng.integers(1, 900, 70)]
    kv = cache("int8", hq, hkv, hd, pages=2400, seqs=70, per_seq=60)
    held = fill(kv, "int8", lens, hkv, hd, 25)
    spans = [L.attend_span(s, 1 + s % 3 if n > 3 else 1, n - (1 + s % 3 if n > 3 else 1), row0=3 * s) for s, n in enumerate(lens)]
    q = queries(rng, 210, hq, hd, "bf16")
    o, lse = torch.full_like(q, 5.0), torch.full((210, hq), 5.0, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    L.laser_attend(kv, 1, spans, q, o, lse=lse, stream=side)
    side.synchronize()
    want, wl = check(kv, "int8", "bf16", held, spans, q)
    assert torch.equal(o, want) and torch.equal(lse, wl)
    g = torch.cuda.CUDAGraph()
    qc, oc = q.clone(), torch.full_like(q, 5.0)
    with torch.cuda.graph(g):
        L.laser_attend(kv, 1, spans, qc, oc)
    for i in range(3):
        qc.copy_(q * (1.0 + i))
        g.replay()
        eager = torch.full_like(q, 5.0)
        L.laser_attend(kv, 1, spans, qc, eager)
        torch.cuda.synchronize()
        assert torch.equal(eager, oc), i
    assert torch.equal(torch.full_like(q, 5.0)[-1:], oc[-1:]) or spans[-1].n == 3


def test_long_context():
    """60,000 positions, split over many workgroups, one row and a few."""
    hq, hkv, hd, n = 7, 1, 128, 60001
    kv = cache("int8", hq, hkv, hd, pages=3800, seqs=1, per_seq=3800)
    held = fill(kv, "int8", [n], hkv, hd, 26)
    q = queries(np.random.default_rng(27), 9, hq, hd, "f32")
    check(kv, "int8", "f32", held, [L.attend_span(0, 1, n - 1), L.attend_span(0, 8, n - 8, row0=1)], q)


@both
@pytest.mark.parametrize("kind,io", [("int8", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 0.9])
def test_scales(kind, io, scale):
    """A negative scale turns the order of the scores, a zero one weighs every seen key alike."""
    hq, hkv, hd = 4, 2, 64
    kv = cache(kind, hq, hkv, hd, pages=40, seqs=1, per_seq=40)
    held = fill(kv, kind, [333], hkv, hd, 28)
    q = queries(np.random.default_rng(29), 60, hq, hd, io)
    check(kv, kind, io, held, [L.attend_span(0, 2, 331), L.attend_span(0, 50, 283, row0=5)], q, scale=scale)


@both
@pytest.mark.parametrize("n", [2, 70])
def test_int8_scales_far_apart(n):
    """Value rows of 2^-60 to 2^60, rows of zeros, beside ordinary ones: each weight counts once in the sum and once,
    times its row's scale, in the output."""
    hq, hkv, hd, length = 4, 2, 64, 300
    kv = cache("int8", hq, hkv, hd, pages=40, seqs=1, per_seq=40)
    rng = np.random.default_rng(30)
    kv.add_seq(0, length)
    k, v = (rng.standard_normal((length, hkv, hd)).astype(np.float32) for _ in range(2))
    v[10] *= 2.0 ** 60
    v[50:70] = 0.0
    v[100:120] *= 2.0 ** -60
    v[200] *= 2.0 ** -30
    v[230] *= 2.0 ** 38
    k, v = (torch.from_numpy(x).to(torch.bfloat16).cuda() for x in (k, v))
    L.laser_kv_write(kv, 1, [L.kv_run(0, 0, length)], k, v)
    held = [(kept("int8", f64(k)), kept("int8", f64(v)))]
    q = queries(rng, n, hq, hd, "bf16")
    # over all keys the largest row decides; over the keys behind it and in front of the next large one, the others do
    check(kv, "int8", "bf16", held, [L.attend_span(0, n, length - n)], q)
    check(kv, "int8", "bf16", [(held[0][0], np.where(np.arange(length)[:, None, None] < 230, held[0][1], 0))],
          [L.attend_span(0, n, length - n, kv_begin=11, kv_end=229)], q)
    o, _ = check(kv, "int8", "bf16", held, [L.attend_span(0, n, length - n, kv_begin=100, kv_end=120)], q)
    assert float(o.float().abs().max()) > 2.0 ** -64  # (the small rows by themselves are not lost)


def device_reference(kv, layer, spans, q, scale, causal, window, hkv):
    """The definition in float64 on the device, over the values that laser_kv_read gives: (o, lse) with 5.0 in other rows."""
    rows_, hq, hd = q.shape
    o = torch.full(q.shape, 5.0, dtype=torch.float64, device="cuda")
    lse = torch.full((rows_, hq), 5.0, dtype=torch.float64, device="cuda")
    top = 0.0
    for s in spans:
        n = kv.seq_len(s.seq)
        end = n if s.kv_end == -1 else s.kv_end
        k, v = (torch.zeros(n, hkv, hd, device="cuda") for _ in range(2))
        if n:
            L.laser_kv_read(kv, layer, [L.kv_run(s.seq, 0, n)], k, v)
            top = max(top, float(v.abs().max()))
        row = torch.arange(s.pos, s.pos + s.n, device="cuda")[:, None]
        t = torch.arange(n, device="cuda")[None, :]
        seen = (t >= s.kv_begin) & (t < end)
        seen = seen & (t <= row) if causal else seen.expand(s.n, n)
        if window:
            seen = seen & (t > row - window)
        r = slice(s.row0, s.row0 + s.n)
        for h in range(hq):
            x = (q[r, h].double() @ k[:, h // (hq // hkv)].double().t()) * scale
            x = x.masked_fill(~seen, -math.inf)
            z = torch.logsumexp(x, -1)
            w = torch.where(torch.isinf(z)[:, None], 0.0, torch.exp(x - z[:, None]))
            o[r, h], lse[r, h] = w @ v[:, h // (hq // hkv)].double(), z
    return o, lse, top


def check_device(kv, io, spans, q, causal=True, window=0, layer=1, o=None, hkv=2):
    o = torch.full_like(q, 5.0) if o is None else o
    lse = torch.full(q.shape[:2], 5.0, device="cuda")
    scale = q.shape[-1] ** -0.5
    ref, rl, top = device_reference(kv, layer, spans, q.clone(), scale, causal, window, hkv)
    L.laser_attend(kv, layer, spans, q, o, lse=lse, causal=causal, window=window)
    torch.cuda.synchronize()
    # (as `tolerance` has it; scores of standard-normal rows stay below 40, their errors below 40 x 2^-22)
    tol = 40 * 2.0 ** -22 * top + (2.0 ** -8 * top + 2.0 ** -8 * ref.abs() if io == "bf16" else 2.0 ** -20 * top)
    assert bool(((o.double() - ref).abs() <= tol).all()), float(((o.double() - ref).abs() - tol).max())
    assert torch.equal(torch.isinf(lse), torch.isinf(rl))
    fin = ~torch.isinf(rl)
    assert bool(((lse.double() - rl).abs()[fin] <= 40 * 2.0 ** -22 + 2.0 ** -22 * rl.abs()[fin]).all())
    return o


@both
@pytest.mark.parametrize("kind,io", [("int8", "bf16"), ("fp8", "f32"), ("bf16", "bf16")])
def test_many_rows_few_splits(kind, io):
    """Some hundred rows behind a long context: tiles whose keys are split a few times, joined row by row; a long prompt
    beside it that is not split; the same in place."""
    hq, hkv, hd = 28, 4, 128
    kv = cache(kind, hq, hkv, hd, pages=700, seqs=3, per_seq=400)
    fill(kv, kind, [4200, 1500, 37], hkv, hd, 31)
    rng = np.random.default_rng(32)
    q = queries(rng, 400 + 700 + 30, hq, hd, io)
    spans = [L.attend_span(0, 400, 3800), L.attend_span(1, 700, 800, row0=400), L.attend_span(2, 3, 34, row0=1101)]
    want = check_device(kv, io, spans, q, hkv=hkv)
    got = check_device(kv, io, spans[:1], q, hkv=hkv)
    assert bool((got[:400].float() - want[:400].float()).abs().max() <= 2.0 ** -7 * float(want[:400].abs().max()))
    again = q.clone()
    L.laser_attend(kv, 1, spans, again, again)
    for s in spans:
        assert torch.equal(again[s.row0:s.row0 + s.n], want[s.row0:s.row0 + s.n])


@both
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_tile_strides(io):
    """Chunks wide enough for tiles: heads before rows, rows off 16 bytes, in and out."""
    hq, hkv, hd, n = 6, 2, 64, 190
    kv = cache("int8", hq, hkv, hd, pages=60, seqs=1, per_seq=60)
    fill(kv, "int8", [800], hkv, hd, 33)
    rng = np.random.default_rng(34)
    base = queries(rng, n, hq, hd, io)
    spans = [L.attend_span(0, n, 800 - n)]
    want = check_device(kv, io, spans, base)
    odd = torch.zeros(n, hq, hd + 1, dtype=IO[io], device="cuda")[:, :, 1:]
    odd.copy_(base)
    out = torch.full((hq, n, hd + 3), 5.0, dtype=IO[io], device="cuda").transpose(0, 1)[:, :, 3:]
    assert torch.equal(check_device(kv, io, spans, odd, o=out), want)


@both
@pytest.mark.parametrize("seed", range(12))
def test_random_calls(seed):
    """Calls of random shape: heads, types, spans of all sizes in one call, key ranges, windows, causal or not."""
    rng = np.random.default_rng(1000 + seed)
    hq, hkv, hd = [(4, 2, 64), (7, 1, 128), (16, 1, 64), (3, 3, 128), (12, 2, 128)][int(rng.integers(5))]
    kind = ["int8", "int8", "fp8", "bf16", "f32"][int(rng.integers(5))]
    io = ["bf16", "f32"][int(rng.integers(2))]
    b = int(rng.integers(1, 9))
    lens = [int(2 ** rng.uniform(0, 11.5)) for _ in range(b)]
    kv = cache(kind, hq, hkv, hd, pages=sum(-(-n // 16) for n in lens) + 1, seqs=b, per_seq=200)
    fill(kv, kind, lens, hkv, hd, 2000 + seed)
    causal, window = bool(rng.random() < 0.8), int(rng.choice([0, 0, 1, 33, 500]))
    spans, at = [], 1
    for _ in range(int(rng.integers(1, 7))):
        s = int(rng.integers(b))
        n = int(2 ** rng.uniform(0, 8.5))
        lo = int(rng.integers(0, lens[s] + 1)) if rng.random() < 0.3 else 0
        hi = int(rng.integers(lo, lens[s] + 1)) if rng.random() < 0.3 else -1
        pos = max(0, lens[s] - n) if rng.random() < 0.6 else int(rng.integers(0, lens[s] + 50))
        spans.append(L.attend_span(s, n, pos, row0=at, kv_begin=lo, kv_end=hi))
        at += n + int(rng.integers(0, 3))
    check_device(kv, io, spans, queries(rng, at + 1, hq, hd, io), causal=causal, window=window, hkv=hkv)


@pytest.mark.parametrize("kernels", [ROWS], indirect=True, ids=["rows"])
@pytest.mark.parametrize("hq,hkv,hd", [(15, 3, 128), (10, 5, 128), (28, 4, 128), (16, 8, 64), (11, 11, 64)])
@pytest.mark.parametrize("kind,io", [("int8", "bf16"), ("bf16", "f32"), ("fp8", "bf16"), ("f32", "f32")])
def test_tiles_that_read_the_same_pages(hq, hkv, hd, kind, io):
    """Row kernels, spans of several tiles beside spans of one: workgroups are dealt out so that a page's tiles share an
    XCD, over numbers of splits and kv heads that no 8 divides."""
    lens = [2900, 1300, 700, 40]
    kv = cache(kind, hq, hkv, hd, pages=320, seqs=4, per_seq=190)
    fill(kv, kind, lens, hkv, hd, 35)
    rng = np.random.default_rng(36)
    spans = [L.attend_span(0, 37, 2863), L.attend_span(1, 1, 1299, row0=40), L.attend_span(2, 90, 610, row0=41),
             L.attend_span(3, 2, 38, row0=131), L.attend_span(0, 9, 2500, row0=133, kv_begin=17, kv_end=2450)]
    check_device(kv, io, spans, queries(rng, 143, hq, hd, io), hkv=hkv)
    check_device(kv, io, spans[2:3], queries(rng, 143, hq, hd, io), window=100, hkv=hkv)
