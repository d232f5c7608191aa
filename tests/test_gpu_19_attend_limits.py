"""laser_attend at the edges of its number types, against the definition in float64: infinities that a row sees in
K, V or its own query, for every type of rows and cache that can hold them and both kernels."""
import numpy as np
import pytest
import torch

from paged_ref import attend, kept
from paper_2606_31580_amd import laser as L
from test_gpu_16_kv_rows import IO, cache, f64
from test_gpu_17_attend import both, check, fill, kernels, queries  # noqa: F401  (kernels: an automatic fixture)

pytestmark = pytest.mark.gpu
POOLS = pytest.mark.parametrize("kind,io", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])


def put(kv, kind, held, seq, pos, is_v, head, dim, value):
    """One element of a cached position replaced, in the cache and in the reference's copy."""
    held[seq][is_v][pos, head, dim] = value
    rows = [torch.from_numpy(x[pos:pos + 1].astype(np.float32)).to(torch.float32 if kind == "f32" else torch.bfloat16).cuda()
            for x in held[seq]]
    L.laser_kv_write(kv, 1, [L.kv_run(seq, pos, 1)], *rows)


def check_all(kv, kind, io, held, spans, q, **kw):
    """`check`, and infinities of the same sign in the same places; returns the reference's rows of each span."""
    o, lse = check(kv, kind, io, held, spans, q, **kw)
    out = []
    for s in spans:
        k, v = held[s.seq]
        r = slice(s.row0, s.row0 + s.n)
        with np.errstate(over="ignore", invalid="ignore"):
            ro, rl = attend(f64(q)[r], k, v, s.pos, q.shape[-1] ** -0.5, True, kw.get("window", 0))
        for got, ref in ((f64(o)[r], ro), (f64(lse)[r], rl)):
            assert np.array_equal(np.isposinf(got), np.isposinf(ref)) and np.array_equal(np.isneginf(got), np.isneginf(ref))
        out.append((ro, rl))
    return out


@both
@POOLS
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n,length", [(2, 330), (90, 330), (1, 3001), (90, 2100)])
def test_seen_infinities(kind, io, hd, n, length):
    """Keys of -infinity weigh nothing, values of either infinity come out, next to queries that parts of bf16 hold
    exactly (1.0: the lower parts are zero) and others; keys of +infinity make the row NaN."""
    hq, hkv = 6, 2
    kv = cache(kind, hq, hkv, hd, pages=2 * (length // 16 + 1), seqs=2, per_seq=190)
    held = fill(kv, kind, [length, length], hkv, hd, 41)
    q = queries(np.random.default_rng(42), 2 * n, hq, hd, io).abs() + 0.25
    q[:, 1::2, :] = 1.0
    q = q.to(IO[io])
    for pos, head, dim in ((3, 0, 5), (length - n, 0, 9), (length // 2, 1, 0), (length // 2 + 1, 1, 63)):
        put(kv, kind, held, 0, pos, False, head, dim, -np.inf)
    for pos, dim, val in ((7, 3, np.inf), (length // 2, 4, -np.inf), (length - n, 8, np.inf)):
        put(kv, kind, held, 0, pos, True, 0, dim, val)
    put(kv, kind, held, 1, length // 3, False, 0, 7, np.inf)
    spans = [L.attend_span(0, n, length - n), L.attend_span(1, n, length - n, row0=n)]
    (o, lse), (o1, lse1) = check_all(kv, kind, io, held, spans, q)
    # (the case is what it says: finite rows beside infinite dims, NaN only where an infinity has weight zero)
    assert np.isfinite(lse).all() and np.isposinf(o[:, 0, 3]).all() and np.isfinite(o[:, 3:]).all()
    assert np.isnan(o1[:, :3]).all() and np.isfinite(o1[:, 3:]).all()


@both
@POOLS
@pytest.mark.parametrize("n", [1, 90])
def test_only_scores_of_minus_infinity(kind, io, n):
    """All keys that a row sees score -infinity: o = 0 and lse = -infinity."""
    hq, hkv, hd, length = 4, 2, 64, 300
    kv = cache(kind, hq, hkv, hd, pages=40, seqs=1, per_seq=40)
    held = fill(kv, kind, [length], hkv, hd, 43)
    held[0][0][:, 0, 11] = -np.inf
    t = torch.float32 if kind == "f32" else torch.bfloat16
    k, v = (torch.from_numpy(x.astype(np.float32)).to(t).cuda() for x in held[0])
    L.laser_kv_write(kv, 1, [L.kv_run(0, 0, length)], k, v)
    q = queries(np.random.default_rng(44), n, hq, hd, io)
    q[:, :2, 11] = 1.0
    ((o, lse),) = check_all(kv, kind, io, held, [L.attend_span(0, n, length - n)], q)
    assert np.isneginf(lse[:, :2]).all() and (o[:, :2] == 0).all()


@both
@POOLS
@pytest.mark.parametrize("n,length", [(1, 300), (90, 300), (1, 3000), (90, 3000)])
def test_only_scores_of_minus_infinity_and_odd_values(kind, io, n, length):
    """The same where V is infinite or NaN at seen positions; keys in one workgroup and in several."""
    hq, hkv, hd = 6, 2, 64
    kv = cache(kind, hq, hkv, hd, pages=length // 16 + 1, seqs=1, per_seq=190)
    held = fill(kv, kind, [length], hkv, hd, 48)
    held[0][0][:, 0, 11] = -np.inf
    held[0][1][5, 0, 1], held[0][1][length - n, 0, 2], held[0][1][length // 2, 0, 3] = np.inf, np.nan, -np.inf
    t = torch.float32 if kind == "f32" else torch.bfloat16
    k, v = (torch.from_numpy(x.astype(np.float32)).to(t).cuda() for x in held[0])
    L.laser_kv_write(kv, 1, [L.kv_run(0, 0, length)], k, v)
    q = queries(np.random.default_rng(49), n, hq, hd, io)
    q[:, :3, 11] = 1.0
    ((o, lse),) = check_all(kv, kind, io, held, [L.attend_span(0, n, length - n)], q)
    assert np.isneginf(lse[:, :3]).all() and (o[:, :3] == 0).all() and np.isfinite(lse[:, 3:]).all()


@both
@pytest.mark.parametrize("kind,io", [("bf16", "f32"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("int8", "f32"), ("fp8", "f32")])
def test_infinite_queries(kind, io):
    """A query of -infinity against keys of one sign scores -infinity everywhere (o = 0), of both signs NaN; a NaN
    whose upper half alone would be an infinity is a NaN."""
    hq, hkv, hd, length, n = 4, 2, 64, 300, 80
    kv = cache(kind, hq, hkv, hd, pages=40, seqs=1, per_seq=40)
    kv.add_seq(0, length)
    rng = np.random.default_rng(45)
    t = torch.float32 if kind == "f32" else torch.bfloat16
    k, v = (rng.standard_normal((length, hkv, hd)).astype(np.float32) for _ in range(2))
    k[:, :, 7] = np.abs(k[:, :, 7]) + 0.5
    k, v = (torch.from_numpy(x).to(t).cuda() for x in (k, v))
    L.laser_kv_write(kv, 1, [L.kv_run(0, 0, length)], k, v)
    back = [torch.empty(length, hkv, hd, device="cuda") for _ in range(2)]
    L.laser_kv_read(kv, 1, [L.kv_run(0, 0, length)], *back)
    held = [tuple(f64(x) for x in back)]
    q = queries(rng, n, hq, hd, io)
    q[3, 0, 7] = q[40, 3, 7] = -np.inf
    q[5, 1, 8] = np.inf
    spans = [L.attend_span(0, n, length - n)]
    if io == "f32":
        q[8, 2, 1] = torch.tensor([0x7f800001], dtype=torch.int32).view(torch.float32).cuda()[0]
    else:
        q[8, 2, 1] = np.nan
    assert torch.isnan(q[8, 2, 1])
    ref = attend(f64(q), *held[0], length - n, hd ** -0.5)
    assert np.isneginf(ref[1][3, 0]) and np.isnan(ref[1][5, 1]) and np.isnan(ref[1][8, 2])
    o, lse = torch.full_like(q, 5.0), torch.full((n, hq), 5.0, device="cuda")
    L.laser_attend(kv, 1, spans, q, o, lse=lse)
    torch.cuda.synchronize()
    o, lse = f64(o), f64(lse)
    for got, want in ((o, ref[0]), (lse, ref[1])):
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isneginf(got), np.isneginf(want))
    assert (o[3, 0] == 0).all() and (o[40, 3] == 0).all()
    fine = np.isfinite(ref[1])
    # (bf16 weights and output: 2^-8 of the largest V and of the output; fp32: the scores' roundings, below 2^-18 here)
    tol = (2.0 ** -8 * np.abs(held[0][1]).max() * 2 if io == "bf16" else 2.0 ** -18 * np.abs(held[0][1]).max())
    assert np.abs(o - ref[0])[fine].max() <= tol


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_low_nan_bits_in_the_cache(io):
    """An fp32 cache keeps a NaN's lowest bits, whose upper half alone is an infinity: it stays a NaN."""
    hq, hkv, hd, length = 2, 2, 64, 100
    kv = cache("f32", hq, hkv, hd, pages=10, seqs=1, per_seq=10)
    fill(kv, "f32", [length], hkv, hd, 46)
    low = torch.tensor([0x7f800001], dtype=torch.int32).view(torch.float32)
    k, v = torch.zeros(1, hkv, hd), torch.zeros(1, hkv, hd)
    k.view(torch.int32)[0, 0, 3] = low.view(torch.int32)[0]
    v.view(torch.int32)[0, 1, 5] = low.view(torch.int32)[0]
    L.laser_kv_write(kv, 1, [L.kv_run(0, 20, 1)], k.cuda(), v.cuda())
    q = queries(np.random.default_rng(47), 1, hq, hd, io)
    o = torch.empty_like(q)
    L.laser_attend(kv, 1, [L.attend_span(0, 1, length - 1)], q, o)
    torch.cuda.synchronize()
    bad = torch.isnan(o[0]).cpu()
    assert bad[0].all() and bad[1, 5] and int(bad[1].sum()) == 1 and torch.isfinite(o[0, 1, :5]).all()


@both
@pytest.mark.parametrize("kind,io", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16"), ("int8", "bf16"), ("int8", "f32")])
@pytest.mark.parametrize("n", [2, 90])
def test_values_near_the_largest(kind, io, n):
    """V of 2^122, at keys that score 5.4 above all before them (2^7.8 times their weight): no sum leaves fp32."""
    hq, hkv, hd, length = 4, 2, 64, 480
    kv = cache(kind, hq, hkv, hd, pages=40, seqs=1, per_seq=40)
    kv.add_seq(0, length)
    k, v = np.zeros((length, hkv, hd)), np.random.default_rng(50).standard_normal((length, hkv, hd)) * 2.0 ** 110
    for pos in (100, 310, length - n):
        k[pos, :, 0] = 43.0 if pos == 310 else 21.5  # (times q 2 and 1/8: 10.75 and 5.375)
        v[pos] = 2.0 ** 122 * (1 - 2 * (np.arange(hd) % 2))
    t = torch.float32 if kind == "f32" else torch.bfloat16
    dk, dv = (torch.from_numpy(x.astype(np.float32)).to(t).cuda() for x in (k, v))
    L.laser_kv_write(kv, 1, [L.kv_run(0, 0, length)], dk, dv)
    held = [(kept(kind, f64(dk)), kept(kind, f64(dv)))]
    q = torch.zeros(n, hq, hd, dtype=IO[io], device="cuda")
    q[:, :, 0] = 2.0
    o, _ = check(kv, kind, io, held, [L.attend_span(0, n, length - n)], q)
    assert bool(torch.isfinite(o).all()) and float(o.float().abs().max()) > 2.0 ** 120


@both
@pytest.mark.parametrize("kind,io", [("bf16", "bf16"), ("bf16", "f32"), ("int8", "bf16")])
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -126, -(2.0 ** -126), 2.0 ** -140])
def test_smallest_scales(kind, io, scale):
    """Products of 2^124 times a scale of next to nothing: scores of 1/4 or none."""
    hq, hkv, hd, length, n = 4, 2, 64, 300, 90
    kv = cache(kind, hq, hkv, hd, pages=40, seqs=1, per_seq=40)
    kv.add_seq(0, length)
    rng = np.random.default_rng(51)
    k, v = np.zeros((length, hkv, hd)), rng.standard_normal((length, hkv, hd))
    k[:, :, 3] = 2.0 ** 62 * np.where(np.arange(length) % 3 == 0, 1.0, -0.5)[:, None]
    k, v = (torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda() for x in (k, v))
    L.laser_kv_write(kv, 1, [L.kv_run(0, 0, length)], k, v)
    q = torch.zeros(n, hq, hd, dtype=IO[io], device="cuda")
    q[:, :, 3] = 2.0 ** 62
    # (the scores' own error: a scale of 2^-126 is exact, products with it below 1 are; `check` counts far more)
    check(kv, kind, io, [(kept(kind, f64(k)), kept(kind, f64(v)))], [L.attend_span(0, n, length - n)], q, scale=scale)


@both
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["bf16", "int8", "fp8"])
def test_large_scores_in_chunks(kind, io):
    """Scores of some hundreds of either sign that grow along the keys, in chunks that fill tiles: the running maximum
    moves at every page, and rows of the other sign never move it."""
    hq, hkv, hd, length, n = 4, 2, 64, 700, 96
    kv = cache(kind, hq, hkv, hd, pages=60, seqs=1, per_seq=60)
    kv.add_seq(0, length)
    rng = np.random.default_rng(52)
    k = rng.standard_normal((length, hkv, hd)) * 0.1 + np.linspace(-4, 4, length)[:, None, None]
    k, v = (torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda() for x in (k, rng.standard_normal((length, hkv, hd))))
    L.laser_kv_write(kv, 1, [L.kv_run(0, 0, length)], k, v)
    k, v = kept(kind, f64(k)), kept(kind, f64(v))
    q = (torch.tensor([1.0, -1.0, 0.5] * (n // 3))[:, None, None].expand(n, hq, hd)).to(IO[io]).cuda()
    o, lse = torch.empty(n, hq, hd, dtype=IO[io], device="cuda"), torch.empty(n, hq, device="cuda")
    L.laser_attend(kv, 1, [L.attend_span(0, n, length - n)], q, o, lse=lse, scale=2.0)
    torch.cuda.synchronize()
    ref, rl = attend(f64(q), k, v, length - n, 2.0)
    # Scores: 64 fp32 additions of terms of one size and two products, 2^-24 of a sum below 600 each at most, 66 x 600 x
    # 2^-24 = 2.4e-3 if all erred one way; errors of both signs leave the root of their number, 3e-4, and 1e-3 is
    # allowed: every weight is off by that factor, top and bottom.  bf16 rows: weights and output by 2^-8 each.
    top = np.abs(v).max()
    tol = 2.0e-3 * top + (2.0 ** -8 * (top + np.abs(ref)) if io == "bf16" else 0.0)
    assert np.abs(rl).max() > 300 and np.all(np.abs(f64(o) - ref) <= tol)
    assert np.all(np.abs(f64(lse) - rl) <= 1.0e-3)


@both
@pytest.mark.parametrize("kind,io", [("int8", "bf16"), ("bf16", "f32")])
def test_captured_chunks(kind, io):
    """Chunks in one piece and in several, captured, replayed with other queries beside eager calls: equal bits."""
    hq, hkv, hd = 8, 2, 128
    lens, rowsn = [2600, 300], [200, 120]
    kv = cache(kind, hq, hkv, hd, pages=190, seqs=2, per_seq=170)
    fill(kv, kind, lens, hkv, hd, 53)
    base = queries(np.random.default_rng(54), sum(rowsn), hq, hd, io)
    spans = [L.attend_span(0, rowsn[0], lens[0] - rowsn[0]), L.attend_span(1, rowsn[1], lens[1] - rowsn[1], row0=rowsn[0])]
    dtype = L.DTYPE_BF16 if io == "bf16" else L.DTYPE_F32
    assert L.laser_attend_workspace(kv, spans, dtype) > 0
    L.laser_kv_write(kv, 1, [])
    q, o, lse = base.clone(), torch.full_like(base, 5.0), torch.full(base.shape[:2], 5.0, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.laser_attend(kv, 1, spans, q, o, lse=lse)
    for i in range(4):
        q.copy_(base * (1.0 - 0.5 * i))
        g.replay()
        eager, el = torch.full_like(base, 7.0), torch.empty_like(lse)
        L.laser_attend(kv, 1, spans, q, eager, lse=el)
        torch.cuda.synchronize()
        assert torch.equal(eager, o) and torch.equal(el, lse), i


@pytest.mark.parametrize("kind", ["int8", "fp8", "bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd,n", [(4, 2, 64, 1), (7, 1, 128, 2), (16, 1, 64, 1)])
@pytest.mark.parametrize("length", [40, 500, 3000])
def test_weights_of_few_columns_keep_16_bits(kind, hq, hkv, hd, n, length):
    """bf16 rows, up to 16 columns: the output is off by its own rounding, and by 2^-16 of the values' largest."""
    kv = cache(kind, hq, hkv, hd, pages=length // 16 + 1, seqs=1, per_seq=190)
    held = fill(kv, kind, [length], hkv, hd, 55)
    q = queries(np.random.default_rng(56), n, hq, hd, "bf16") * 2
    o = torch.empty_like(q)
    L.laser_attend(kv, 1, [L.attend_span(0, n, length - n)], q, o)
    torch.cuda.synchronize()
    k, v = held[0]
    ref, _ = attend(f64(q), k, v, length - n, hd ** -0.5)
    # Two bf16 parts: the second is what the first is off by (2^-8 of the weight at most), off by 2^-8 of that.  Scores
    # as `tolerance` of test_gpu_17_attend has them; E4M3 and INT8 values are exact, and a scale and product of three
    # fp32 roundings.  The output's half step is 2^-8 of itself.
    top, terms = np.abs(v).max(), hd ** -0.5 * np.abs(f64(q)).max() * np.abs(k).max() * hd ** 0.5
    tol = 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -8) + (2.0 ** -16 + (4 * terms + 64) * 2.0 ** -24) * top
    assert np.all(np.abs(f64(o) - ref) <= tol), (np.abs(f64(o) - ref) - tol).max()
