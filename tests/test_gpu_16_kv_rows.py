"""laser_kv_write and laser_kv_read (a caller's rows of K and V on the paged cache) against float64
definitions: every cache type and row type, both head dimensions, runs that start and end anywhere in
a page, strided and unaligned rows, other positions and rows left alone; and import, export and fork of
INT8 caches."""
import numpy as np
import pytest
import torch

from gpu_helpers import require_gpu
from paged_ref import kept
from paper_2606_31580_amd import laser as L
from paper_2606_31580_amd import synth
from paper_2606_31580_amd.configs import ModelShape

pytestmark = pytest.mark.gpu
IO = {"bf16": torch.bfloat16, "f32": torch.float32}
_models = {}
MODE = 0  # kernels of laser_attend in new models (set by its tests)


def cache(kind, hq=4, hkv=2, hd=64, pages=96, seqs=6, per_seq=64, layers=2, poison=True):
    require_gpu()
    key = (kind, hq, hkv, hd, layers)
    if key not in _models:
        shape = ModelShape("rows-%s-%d-%d-%d-%d" % key, layers, 64, hq, hkv, hd, 64, 64, True, False,
                           "f32" if kind == "f32" else "bf16", 1.0e4, 1.0e-5, kind if kind in ("fp8", "int8") else "")
        w = {k: v.cuda() for k, v in synth.make_weights(shape).items()}
        _models[key] = L.Model(shape, w, max_rows=4, max_positions=65536, tiles=False)
        _models[key].set_attend_kernel(MODE)
    return L.KVCache(_models[key], pages, seqs, per_seq, poison=poison)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rows(rng, n, hkv, hd, io):
    """Rows with heads and channels of different size; row 0 (if any) all zero but one element."""
    x = rng.standard_normal((n, hkv, hd)) * np.exp(rng.standard_normal((n, hkv, 1)) * 2) * np.exp(rng.standard_normal((1, hkv, hd)))
    if n:
        x[0] = 0
        x[0, 0, 3] = -1.5
    return torch.from_numpy(x.astype(np.float32)).to(IO[io]).cuda()


def stored_tol(kind, io, ref, src):
    """How far a value read back may be from the float64 definition: the fp32 scale and product (2^-24 each,
    three roundings), the rows' own type, and for fp32 rows of an 8-bit integer cache the step itself where the
    fp32 quotient and the exact one fall on different sides of a half (within 127 x 2^-23 steps of it)."""
    tol = 3 * 2.0 ** -24 * np.abs(ref)
    if io == "bf16":
        tol = tol + 2.0 ** -8 * np.abs(ref)
    if kind == "int8":
        top = np.abs(src).max(-1, keepdims=True)
        with np.errstate(invalid="ignore", divide="ignore"):
            r = np.where(top > 0, 127.0 * src / np.where(top > 0, top, 1), 0.0)
        near = np.abs(np.abs(r - np.rint(r)) - 0.5) < 127 * 2.0 ** -23
        # (exact for bf16 rows: 127 x has 15 bits, and the quotient is a half or at least 1/255 from it)
        tol = tol + (near & (np.abs(r - np.rint(r)) != 0.5)) * top / 127.0
    return tol


RUNS = [(0, 0, 1), (0, 1, 2), (0, 3, 1), (1, 5, 27), (2, 0, 16), (3, 17, 0), (3, 30, 33), (4, 0, 250), (5, 15, 2)]
LENS = [4, 40, 16, 63, 250, 17]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["int8", "fp8", "bf16", "f32"])
def test_write_read(kind, io, hd):
    rng = np.random.default_rng(11)
    hkv = 2 if hd == 64 else 3
    kv = cache(kind, hq=2 * hkv, hkv=hkv, hd=hd)
    for s, n in enumerate(LENS):
        kv.add_seq(s, n)
    total = sum(r[2] for r in RUNS)
    order = rng.permutation(len(RUNS))  # rows of the runs are not in the runs' order
    row0, at = [0] * len(RUNS), 3
    for i in order:
        row0[i] = at
        at += RUNS[i][2] + 1
    k, v = rows(rng, at + 2, hkv, hd, io), rows(rng, at + 2, hkv, hd, io)
    runs = [L.kv_run(s, p, n, r) for (s, p, n), r in zip(RUNS, row0)]
    before = (kv.k_pool.clone(), kv.v_pool.clone())
    L.laser_kv_write(kv, 1, runs, k, v)
    out = [torch.full_like(k, 7.0) for _ in range(2)]
    L.laser_kv_read(kv, 1, runs, *out)
    torch.cuda.synchronize()
    inside = np.zeros(at + 2, dtype=bool)
    for (s, p, n), r in zip(RUNS, row0):
        inside[r:r + n] = True
    assert inside.sum() == total
    for src, got in zip((k, v), out):
        s64, g64 = f64(src), f64(got)
        ref = kept(kind, s64)
        assert np.all(g64[~inside] == 7.0)  # rows outside the runs
        assert np.all(np.abs(g64 - ref)[inside] <= stored_tol(kind, io, ref, s64)[inside])
    # layer 0 and unwritten slots keep their bytes: as many changed as were written, at most
    es = {"int8": 1, "fp8": 1, "bf16": 2, "f32": 4}[kind]
    for pool, old in zip((kv.k_pool, kv.v_pool), before):
        assert torch.equal(pool[:96 * hkv * 16 * hd * es], old[:96 * hkv * 16 * hd * es])
        changed = int((pool[:2 * 96 * hkv * 16 * hd * es] != old[:2 * 96 * hkv * 16 * hd * es]).sum())
        assert changed <= total * hkv * hd * es
    # written one position at a time, the cache holds the same bytes
    one = cache(kind, hq=2 * hkv, hkv=hkv, hd=hd)
    for s, n in enumerate(LENS):
        one.add_seq(s, n)
    singles = [L.kv_run(s, p + i, 1, r + i) for (s, p, n), r in zip(RUNS, row0) for i in range(n)]
    L.laser_kv_write(one, 1, singles, k, v)  # (more runs than one launch takes)
    torch.cuda.synchronize()
    assert torch.equal(one.k_pool, kv.k_pool) and torch.equal(one.v_pool, kv.v_pool)


@pytest.mark.parametrize("kind", ["int8", "fp8", "bf16"])
def test_strides_and_alignment(kind):
    """K and V as parts of a fused projection's output, heads before rows, a broadcast row, one element off 16 bytes."""
    rng = np.random.default_rng(3)
    hkv, hd, n = 2, 64, 37
    kv = cache(kind, hkv=hkv, hd=hd)
    kv.add_seq(0, n)
    kv.add_seq(1, n)
    fused = rows(rng, n, 8, hd, "bf16")
    heads_first = rows(rng, hkv, n, hd, "bf16").transpose(0, 1)
    odd = rows(rng, n, hkv, hd + 1, "bf16")[:, :, 1:]
    one = rows(rng, 1, hkv, hd, "bf16").expand(n, hkv, hd)
    for k, v in ((fused[:, 4:6], fused[:, 6:8]), (heads_first, odd), (one, fused[:, 1:3])):
        L.laser_kv_write(kv, 0, [L.kv_run(1, 0, n)], k, v)
        outs = (torch.zeros(n, 3 * hkv, hd, dtype=torch.float32, device="cuda")[:, hkv:2 * hkv],
                torch.zeros(hkv, n, hd + 3, dtype=torch.float32, device="cuda").transpose(0, 1)[:, :, 3:])
        L.laser_kv_read(kv, 0, [L.kv_run(1, 0, n)], *outs)
        torch.cuda.synchronize()
        for src, got in zip((k, v), outs):
            ref = kept(kind, f64(src))
            assert np.all(np.abs(f64(got) - ref) <= stored_tol(kind, "f32", ref, f64(src)))


def test_int8_odd_values():
    """Zeros, the type's smallest and largest values, ties, infinities and NaN."""
    hd = 64
    kv = cache("int8", hd=hd)
    x = torch.zeros(9, 2, hd)
    x[1, :, 0] = 2.0 ** -133            # amax is subnormal: 127 x and 1 / amax leave the normal range
    x[1, :, 1] = -(2.0 ** -133)
    x[2] = torch.linspace(-1, 1, hd) * 3.3e38
    x[3, :, 0], x[3, :, 1:9] = 3.0, torch.tensor([1.5, -1.5, 0.75, 3.0, -3.0, 2.25, 0.0, -0.0])  # 63.5 steps: to 64
    x[4, :, 0], x[4, :, 1:4] = 254.0, torch.tensor([1.0, 3.0, -5.0])  # half steps: 0.5, 1.5, -2.5 -> 0, 2, -2
    x[5, 0, 7] = float("inf")
    x[6, 0, 7] = float("nan")
    x[7, 1, 9] = float("-inf")
    x[8] = 1.0
    xb = x.to(torch.bfloat16).cuda()
    kv.add_seq(0, 9)
    L.laser_kv_write(kv, 0, [L.kv_run(0, 0, 9)], xb, xb)
    out = [torch.empty(9, 2, hd, device="cuda") for _ in range(2)]
    L.laser_kv_read(kv, 0, [L.kv_run(0, 0, 9)], *out)
    torch.cuda.synchronize()
    ref = kept("int8", f64(xb))
    for o in out:
        o = f64(o)
        assert np.array_equal(np.isnan(o), np.isnan(ref))
        assert np.isnan(o[5, 0]).all() and np.isnan(o[6, 0]).all() and np.isnan(o[7, 1]).all() and not np.isnan(o[5, 1]).any()
        # (subnormal amax: its scale amax / 127 keeps few bits, an absolute 2^-150)
        ok = np.abs(o - ref) <= 3 * 2.0 ** -24 * np.abs(ref) + 127 * 2.0 ** -150
        assert ok[~np.isnan(ref)].all()
        assert o[3, 0, 1] == o[3, 0, 0] * 64 / 127 or abs(o[3, 0, 1] - 3.0 * 64 / 127) < 1e-6
        assert list(o[4, 0, 1:4]) == [0.0, 4.0, -4.0]


def test_fp8_every_boundary():
    """E4M3 of every bf16 value up to 512 (all ties among them), and beyond the largest."""
    kv = cache("fp8", hkv=2, hd=64, pages=8192 // 16 // 2 + 8, per_seq=600)
    bits = np.arange(0, 0x4400, dtype=np.uint32)  # +0 .. 512
    vals = (bits << 16).view(np.float32)
    vals = np.concatenate([vals, -vals, np.float32([1e38, -1e38, np.nan])])
    n = -(-vals.size // 128)
    x = torch.from_numpy(np.resize(vals, n * 128).reshape(n, 2, 64)).to(torch.bfloat16).cuda()
    kv.add_seq(0, n)
    L.laser_kv_write(kv, 0, [L.kv_run(0, 0, n)], x, x)
    out = [torch.empty(n, 2, 64, device="cuda") for _ in range(2)]
    L.laser_kv_read(kv, 0, [L.kv_run(0, 0, n)], *out)
    torch.cuda.synchronize()
    for o in out:
        assert np.array_equal(f64(o), kept("fp8", f64(x)), equal_nan=True)


def test_int8_import_export_fork():
    """Dense bf16 K/V in and out of an INT8 cache, and a fork whose partial page (scales too) is its own."""
    rng = np.random.default_rng(8)
    n, hkv, hd = 37, 2, 64
    kv = cache("int8")
    kv.add_seq(3, 5)
    kv.add_seq(0, n)
    k, v = (torch.stack([rows(rng, n, hkv, hd, "bf16") for _ in range(2)]) for _ in range(2))
    kv.import_kv(0, k, v)
    kv.fork(0, 1)
    kv.append(1, 3)
    kv.append(0, 2)
    new = rows(rng, 5, hkv, hd, "bf16")
    for layer in range(2):
        L.laser_kv_write(kv, layer, [L.kv_run(1, n, 3, 0), L.kv_run(0, n, 2, 3)], new, new)
    got = {}
    for seq, m in ((0, n + 2), (1, n + 3)):
        o = [torch.empty(2, m, hkv, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        kv.export_kv(seq, *o)
        got[seq] = o
    torch.cuda.synchronize()
    for seq, tail in ((0, new[3:5]), (1, new[0:3])):
        for src, o in zip((k, v), got[seq]):
            full = torch.cat([src, tail.expand(2, *tail.shape)], 1)
            ref = kept("int8", f64(full))
            assert np.all(np.abs(f64(o) - ref) <= stored_tol("int8", "bf16", ref, f64(full)))
    with pytest.raises(L.LaserError, match="fork shares"):
        L.laser_kv_write(kv, 0, [L.kv_run(0, 20, 4, 0)], new, new)
    L.laser_kv_write(kv, 0, [L.kv_run(0, 32, 5, 0)], new, new)  # (its own partial page)


def test_captured_write_and_read():
    """A write and a read captured into a graph, replayed with other rows between eager calls."""
    rng = np.random.default_rng(21)
    hkv, hd, n = 2, 64, 19
    kv = cache("int8")
    kv.add_seq(0, 50)
    x = [rows(rng, n, hkv, hd, "bf16") for _ in range(4)]
    k, v = x[0].clone(), x[1].clone()
    out = [torch.zeros_like(k) for _ in range(2)]
    runs = [L.kv_run(0, 13, n)]
    g = torch.cuda.CUDAGraph()
    with pytest.raises(L.LaserError, match="before the capture"):
        with torch.cuda.graph(g):
            L.laser_kv_write(kv, 1, runs, k, v)
    L.laser_kv_write(kv, 0, [])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.laser_kv_write(kv, 1, runs, k, v)
        L.laser_kv_read(kv, 1, runs, *out)
    for a, b in ((0, 1), (2, 3), (1, 2)):
        k.copy_(x[a])
        v.copy_(x[b])
        g.replay()
        torch.cuda.synchronize()
        for src, o in ((x[a], out[0]), (x[b], out[1])):
            ref = kept("int8", f64(src))
            assert np.all(np.abs(f64(o) - ref) <= stored_tol("int8", "bf16", ref, f64(src)))
        other = [torch.zeros_like(k) for _ in range(2)]
        L.laser_kv_read(kv, 1, runs, *other)
        assert torch.equal(other[0], out[0]) and torch.equal(other[1], out[1])
