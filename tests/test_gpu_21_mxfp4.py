"""The 4-bit KV cache (E2M1 codes, a power of two per 32 dims of a position and head): writes and reads against the
format's definition, import, export and fork, attention of a caller's rows over it, and the model's own forward against
the oracle that rounds K and V the same way."""
import numpy as np
import pytest
import torch

from gpu_helpers import check_prob, check_token, compare_logits, make_pair, require_gpu
from mxfp4_ref import cache, f64, fill, kept, rows
from oracle.numerics import mxfp4_blocks, round_mxfp4_rows
from oracle.transformer import SeqState, lm_stats
from paged_ref import attend
from paper_2606_31580_amd import laser as L
from paper_2606_31580_amd import synth
from paper_2606_31580_amd.configs import QWEN_1P5B_FP4KV, QWEN_7B_FP4KV, ModelShape
from test_gpu_17_attend import check, queries, tolerance
from test_gpu_2_full_shapes import Setup

pytestmark = pytest.mark.gpu

RUNS = [(0, 0, 1), (0, 1, 2), (0, 3, 1), (1, 5, 27), (2, 0, 16), (3, 17, 0), (3, 30, 33), (4, 0, 250), (5, 15, 2)]
LENS = [4, 40, 16, 63, 250, 17]


def _bytes(pool, layers, pages, hkv, hd):
    """Blocks [layer, page, head, bytes] and scales [layer, page, head, 16, hd / 32] of a pool."""
    raw = pool.cpu().numpy()
    n = layers * pages * hkv * 8 * hd
    return raw[:n].reshape(layers, pages, hkv, 8 * hd), raw[n:].reshape(layers, pages, hkv, 16, hd // 32)


def _stored(blocks, scales, is_v, hd, layer, page, head, t):
    """Codes and scale bytes of a position, from the layout that laser.h documents."""
    ns, b = hd // 32, blocks[layer, page, head]
    codes = np.zeros(hd, dtype=np.int64)
    for d in range(hd):
        if is_v:
            byte = b[4 * ((t // 4 * 16 + d % 16) * ns + d // 32) + t % 4]
            codes[d] = byte >> 4 if d % 32 >= 16 else byte & 15
        else:
            byte = b[4 * ((d % 32 // 8 * 16 + t) * ns + d // 32) + d % 8 // 2]
            codes[d] = byte >> 4 if d % 2 else byte & 15
    return codes, scales[layer, page, head, t]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_write_read(io, hd):
    """Runs that start and end anywhere in a page: exact values back (a code times a power of two is exact in both row
    types), the documented bytes, everything else left alone; one position at a time gives the same bytes."""
    rng = np.random.default_rng(11)
    hkv = 2 if hd == 64 else 3
    kv = cache(2 * hkv, hkv, hd)
    for s, n in enumerate(LENS):
        kv.add_seq(s, n)
    order = rng.permutation(len(RUNS))  # rows of the runs are not in the runs' order
    row0, at = [0] * len(RUNS), 3
    for i in order:
        row0[i] = at
        at += RUNS[i][2] + 1
    k, v = rows(rng, at + 2, hkv, hd, io, 2.0), rows(rng, at + 2, hkv, hd, io, 2.0)
    k[row0[3]] = 0
    k[row0[3] + 1, 0] = 0
    k[row0[3] + 1, 0, 3] = -1.5
    runs = [L.kv_run(s, p, n, r) for (s, p, n), r in zip(RUNS, row0)]
    before = [p.clone() for p in (kv.k_pool, kv.v_pool)]
    L.laser_kv_write(kv, 1, runs, k, v)
    out = [torch.full_like(k, 7.0) for _ in range(2)]
    L.laser_kv_read(kv, 1, runs, *out)
    torch.cuda.synchronize()
    inside = np.zeros(at + 2, dtype=bool)
    for (s, p, n), r in zip(RUNS, row0):
        inside[r:r + n] = True
    for src, got in zip((k, v), out):
        g64, ref = f64(got), kept("mxfp4", f64(src))
        assert np.all(g64[~inside] == 7.0)
        assert np.array_equal(g64[inside], ref[inside])
    for is_v, pool, old, src in ((False, kv.k_pool, before[0], k), (True, kv.v_pool, before[1], v)):
        blocks, scales = _bytes(pool, 2, 96, hkv, hd)
        was_b, was_s = _bytes(old, 2, 96, hkv, hd)
        codes, exps = mxfp4_blocks(f64(src))
        want_b, want_s = was_b.copy(), was_s.copy()
        for (s, p, n), r in zip(RUNS, row0):
            table = kv.page_table(s)
            for i in range(n):
                page, t = table[(p + i) // 16], (p + i) % 16
                for h in range(hkv):
                    c, sc = _stored(blocks, scales, is_v, hd, 1, page, h, t)
                    assert np.array_equal(c, codes[r + i, h]), (is_v, s, p + i, h)
                    assert np.array_equal(sc.astype(int) - 127, exps[r + i, h])
                    ns = hd // 32  # the bytes of this position may change, no others
                    for d in range(hd):
                        at_b = 4 * ((t // 4 * 16 + d % 16) * ns + d // 32) + t % 4 if is_v else 4 * ((d % 32 // 8 * 16 + t) * ns + d // 32) + d % 8 // 2
                        want_b[1, page, h, at_b] = blocks[1, page, h, at_b]
                    want_s[1, page, h, t] = scales[1, page, h, t]
        assert np.array_equal(want_b, blocks) and np.array_equal(want_s, scales)
    one = cache(2 * hkv, hkv, hd)
    for s, n in enumerate(LENS):
        one.add_seq(s, n)
    L.laser_kv_write(one, 1, [L.kv_run(s, p + i, 1, r + i) for (s, p, n), r in zip(RUNS, row0) for i in range(n)], k, v)
    torch.cuda.synchronize()
    assert torch.equal(one.k_pool, kv.k_pool) and torch.equal(one.v_pool, kv.v_pool)


def test_strides_and_alignment():
    """K and V as parts of a fused projection's output, heads before rows, a broadcast row, one element off 16 bytes."""
    rng = np.random.default_rng(3)
    hkv, hd, n = 2, 64, 37
    kv = cache(hkv=hkv, hd=hd)
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
            assert np.array_equal(f64(got), kept("mxfp4", f64(src)))


def test_every_border():
    """All borders between codes at several exponents, the ends of the exponents' range, zeros, infinities and NaN."""
    hd = 64
    near = [0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0]
    x = []
    for e in (-130, -104, -101, -100, -99, -30, 0, 7, 120, 124, 125, 126):
        for top in (4.0, 6.0, 7.0, 7.03125):
            if top * 2.0 ** e >= 2.0 ** 128:
                continue
            x.append([np.float32(s * v * 2.0 ** e) for s in (1, -1) for v in near] + [0.0, np.float32(top * 2.0 ** e)] + [1.0] * 32)
    x.append([np.nan] + [1.0] * 63)
    x.append([1.0] * 40 + [-np.inf] + [2.0] * 23)
    x.append([0.0, -0.0] * 32)
    x.append([3.38e38, -3.38e38] * 32)
    x = np.array(x, dtype=np.float32)
    n = x.shape[0]
    kv = cache(hd=hd)
    kv.add_seq(0, n)
    for io in ("f32", "bf16"):
        src = torch.from_numpy(x).to(torch.float32 if io == "f32" else torch.bfloat16)[:, None, :].expand(n, 2, hd).contiguous().cuda()
        L.laser_kv_write(kv, 0, [L.kv_run(0, 0, n)], src, src)
        out = [torch.empty(n, 2, hd, device="cuda") for _ in range(2)]
        L.laser_kv_read(kv, 0, [L.kv_run(0, 0, n)], *out)
        torch.cuda.synchronize()
        for o in out:
            assert np.array_equal(f64(o), kept("mxfp4", f64(src)), equal_nan=True)


def test_import_export_fork():
    """Dense bf16 K/V in and out, and a fork whose partial page (scales too) is its own."""
    for hd in (64, 128):
        rng = np.random.default_rng(8)
        n, hkv = 37, 2
        kv = cache(hd=hd)
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
                assert np.array_equal(f64(o), kept("mxfp4", f64(full)))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 64), (7, 1, 128), (3, 3, 128), (32, 2, 64)])
def test_decode_rows(io, hq, hkv, hd):
    """One row per sequence: lengths around page and pair edges, up to some that split."""
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 64, 129, 500, 1333, 0]
    kv = cache(hq, hkv, hd, pages=200, seqs=len(lens), per_seq=100)
    held = fill(kv, lens, hkv, hd, 5)
    q = queries(np.random.default_rng(6), len(lens) + 2, hq, hd, io)
    check(kv, "mxfp4", io, held, [L.attend_span(s, 1, max(n - 1, 0), row0=s + 1) for s, n in enumerate(lens)], q)


@pytest.mark.parametrize("mode", [1, 2], ids=["rows", "tiles"])
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 64), (7, 1, 128), (3, 3, 128)])
def test_chunks(mode, io, hq, hkv, hd):
    """Chunks of 2 to some hundred rows behind contexts of every kind, in one call; the whole sequence as one chunk too."""
    lens = [2, 20, 37, 64, 100, 257, 600, 300]
    rowsn = [2, 5, 37, 9, 70, 200, 3, 300]
    kv = cache(hq, hkv, hd, pages=200, seqs=len(lens), per_seq=100, mode=mode)
    held = fill(kv, lens, hkv, hd, 7)
    q = queries(np.random.default_rng(8), sum(rowsn), hq, hd, io)
    spans, at = [], 0
    for s, (n, r) in enumerate(zip(lens, rowsn)):
        spans.append(L.attend_span(s, r, n - r, row0=at))
        at += r
    check(kv, "mxfp4", io, held, spans, q)


@pytest.mark.parametrize("mode", [1, 2], ids=["rows", "tiles"])
@pytest.mark.parametrize("io,hd", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("causal,window", [(True, 1), (True, 16), (True, 77), (False, 0), (False, 40)])
def test_masks_and_ranges(mode, io, hd, causal, window):
    """Windows, key ranges that start and end inside pages, rows in front of and behind all their keys."""
    hq, hkv = 6, 2
    lens = [300, 300, 90, 300, 40]
    kv = cache(hq, hkv, hd, pages=100, seqs=5, per_seq=40, mode=mode)
    held = fill(kv, lens, hkv, hd, 9)
    spans = [L.attend_span(0, 40, 260, row0=0), L.attend_span(1, 33, 100, row0=40, kv_begin=37, kv_end=211),
             L.attend_span(2, 20, 5, row0=73, kv_begin=13, kv_end=13), L.attend_span(3, 25, 0, row0=93, kv_begin=11),
             L.attend_span(4, 30, 1000, row0=118), L.attend_span(0, 1, 150, row0=148, kv_begin=149, kv_end=151),
             L.attend_span(0, 100, 120, row0=149, kv_begin=160)]
    q = queries(np.random.default_rng(10), 250, hq, hd, io)
    check(kv, "mxfp4", io, held, spans, q, causal=causal, window=window)


@pytest.mark.parametrize("mode", [1, 2], ids=["rows", "tiles"])
@pytest.mark.parametrize("io,hd", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("n", [1, 3, 40, 150])
def test_nan_in_unseen_places(mode, io, hd, n):
    """A block that is NaN in K or V: rows that do not see its position are as if it were not there; of rows that see it in V,
    the 32 dims are NaN and no others; in K, all of the head."""
    hq, hkv, length = 4, 2, 330
    kv = cache(hq, hkv, hd, pages=60, seqs=2, per_seq=30, mode=mode)
    k, v = fill(kv, [length], hkv, hd, 12)[0]
    bad_v, bad_k = length - n + n // 2, length - 1
    for pos, x, head, dim in ((bad_v, v, 0, 37), (bad_k, k, 1, 5)):
        x[pos, head, dim] = np.nan
        a, b = (torch.from_numpy(y[pos:pos + 1].astype(np.float32)).to(torch.bfloat16).cuda() for y in (k, v))
        L.laser_kv_write(kv, 1, [L.kv_run(0, pos, 1)], a, b)
        x[pos, head] = kept("mxfp4", x[pos, head])
    q = queries(np.random.default_rng(13), n, hq, hd, io)
    for window in (0, max(1, n // 2)):
        o, lse = torch.full_like(q, 5.0), torch.full((n, hq), 5.0, device="cuda")
        L.laser_attend(kv, 1, [L.attend_span(0, n, length - n)], q, o, lse=lse, window=window)
        torch.cuda.synchronize()
        ref, ref_lse = attend(f64(q), k, v, length - n, hd ** -0.5, window=window)
        assert np.isnan(ref).any() and np.array_equal(np.isnan(f64(o)), np.isnan(ref))
        assert np.array_equal(np.isnan(f64(lse)), np.isnan(ref_lse))
        fine = ~np.isnan(ref)
        tol = np.broadcast_to(tolerance(io, ref, np.nan_to_num(v), f64(q), np.nan_to_num(k), hd ** -0.5), ref.shape)
        assert np.all(np.abs(f64(o) - ref)[fine] <= tol[fine])


@pytest.mark.parametrize("mode", [1, 2], ids=["rows", "tiles"])
@pytest.mark.parametrize("byte", [0xFF, 0xFE, 0xFD, 0xFC, 0x77, 0x00])
def test_poisoned_neighbours(byte, mode):
    """Slots past the length, pages of other sequences and other layers hold scales that are NaN, that make codes infinite,
    or are the largest that do not."""
    for hd in (64, 128):
        kv = cache(4, 2, hd, pages=40, seqs=4, per_seq=20, mode=mode)
        kv.k_pool.fill_(byte)
        kv.v_pool.fill_(byte)
        held = fill(kv, [17, 33, 50, 101], 2, hd, 14)
        q = queries(np.random.default_rng(15), 62, 4, hd, "bf16")
        check(kv, "mxfp4", "bf16", held, [L.attend_span(0, 1, 16, 0), L.attend_span(1, 5, 28, 1), L.attend_span(2, 6, 44, 6), L.attend_span(3, 50, 51, 12)], q)


@pytest.mark.parametrize("kind", ["mxfp4", "int8"])
def test_far_into_a_pool(kind):
    """Pages that lie past 2^32 bytes of their pool: what a small cache gives, from rotated write to attention, and of a fork."""
    rng = np.random.default_rng(14)
    hq, hkv, hd, n = 8, 8, 128, 90
    pages, layer = {"mxfp4": 140000, "int8": 75000}[kind], 4
    small, far = (cache(hq, hkv, hd, pages=p, layers=5, kind=kind) for p in (30, pages))
    k, v, q = (rows(rng, n, h, hd, "bf16") for h in (hkv, hkv, hq))
    rope = L.rope(hd, 1.0e4)
    got = []
    for kv in (small, far):
        assert kv is small or layer * pages * hkv * hd * 16 // (2 if kind == "mxfp4" else 1) > 2 ** 32
        kv.add_seq(0, n)
        out = [torch.zeros_like(x) for x in (q, k, v, q, q, k, v)]
        L.laser_kv_write_rotated(kv, layer, rope, [L.kv_run(0, 0, n)], k, v, q, out[0])
        L.laser_kv_read(kv, layer, [L.kv_run(0, 0, n)], *out[1:3])
        for mode, o in zip((1, 2), out[3:5]):
            kv.model.set_attend_kernel(mode)
            L.laser_attend(kv, layer, [L.attend_span(0, n, 0)], out[0], o)
        kv.model.set_attend_kernel(0)
        kv.fork(0, 1)
        L.laser_kv_read(kv, layer, [L.kv_run(1, 0, n)], *out[5:])
        torch.cuda.synchronize()
        got.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert torch.equal(got[0][1], got[0][5]) and torch.equal(got[0][2], got[0][6])
    assert np.array_equal(f64(got[0][2]), kept(kind, f64(v))) if kind == "mxfp4" else True


def test_captured():
    """Write, attention and read in one graph, replayed with other rows between eager calls on the same cache."""
    rng = np.random.default_rng(21)
    hq, hkv, hd, n = 8, 2, 128, 19
    kv = cache(hq, hkv, hd, pages=200, per_seq=180)
    held = fill(kv, [2500], hkv, hd, 22)[0]
    spans, runs = [L.attend_span(0, n, 2500 - n)], [L.kv_run(0, 2500 - n, n)]
    new = [(rows(rng, n, hkv, hd, "bf16"), rows(rng, n, hkv, hd, "bf16"), queries(rng, n, hq, hd, "bf16")) for _ in range(3)]
    k, v, q = (x.clone() for x in new[0])
    o, out = torch.zeros_like(q), [torch.zeros_like(k) for _ in range(2)]
    ws = torch.empty(max(16, L.laser_attend_workspace(kv, spans)), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.laser_kv_write(kv, 1, runs, k, v)
        L.laser_attend(kv, 1, spans, q, o, workspace=ws)
        L.laser_kv_read(kv, 1, runs, *out)
    for i in (0, 1, 2, 1):
        for dst, src in zip((k, v, q), new[i]):
            dst.copy_(src)
        g.replay()
        torch.cuda.synchronize()
        for src, got in zip(new[i], out):
            assert np.array_equal(f64(got), kept("mxfp4", f64(src)))
        K, V = (np.concatenate([h[:-n], f64(x)]) for h, x in zip(held, out))
        ref, _ = attend(f64(q), K, V, 2500 - n, hd ** -0.5)
        assert np.all(np.abs(f64(o) - ref) <= tolerance("bf16", ref, V, f64(q), K, hd ** -0.5))
        eager = torch.zeros_like(o)
        L.laser_attend(kv, 1, spans, q, eager)
        torch.cuda.synchronize()
        assert torch.equal(eager, o)


# ------------------------------------------------------------------------------ the model's own forward

SMALL = ModelShape("small-mxfp4kv", 2, 256, 4, 2, 64, 672, 2048, False, True, "bf16", 1.0e4, 1.0e-5, "mxfp4")
WIDE = ModelShape("small-mxfp4kv-128", 2, 256, 7, 1, 128, 680, 2048, True, False, "bf16", 1.0e4, 1.0e-5, "mxfp4")


def _export(kv, shape, seq):
    n = kv.seq_len(seq)
    o = [torch.empty((shape.n_layers, n, shape.n_kv_heads, shape.head_dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kv.export_kv(seq, *o)
    torch.cuda.synchronize()
    return [f64(t) for t in o]


def _adopt(kv, shape, seq, state, at):
    """Checks positions `at` .. of the cache against the oracle's and gives the oracle the cache's values there.

    The forward's K and V (fp32 projections) differ from the oracle's by some 2^-20 of the vector's size: an element
    that close to a border takes the neighbouring code, and a largest one that close to 7 2^e the next scale, with all
    its block.  Either way a value is off by at most the larger scale's step at its size: 2 2^e, e the block's.  With
    few codes per vector that is rare; the oracle goes on from what the cache holds, so that later logits compare."""
    moved = total = 0
    for got, ref in zip(_export(kv, shape, seq), (state.K, state.V)):
        mine = ref[:, at:got.shape[1]]
        new = got[:, at:]
        block = np.abs(mine).reshape(mine.shape[:-1] + (-1, 32)).max(-1, keepdims=True)
        step = np.broadcast_to(block, block.shape[:-1] + (32,)).reshape(mine.shape)  # (at least 2 steps of 2^e: 4 2^e <= block)
        assert np.all(np.abs(new - mine) <= 0.51 * step)
        moved += int((new != mine).sum())
        total += new.size
        ref[:, at:got.shape[1]] = new
    assert moved <= max(4, total // 500), (moved, total)


def _states(kv, shape, lens, capacity):
    out = []
    for s, n in enumerate(lens):
        k0, v0 = synth.make_prefill_kv(shape, n, s)
        kv.add_seq(s, n)
        if n:
            kv.import_kv(s, k0.cuda(), v0.cuda())
        k, v = (round_mxfp4_rows(t.float().numpy()) for t in (k0, v0))
        out.append(SeqState.from_prefill(shape, k, v, capacity))
        for got, ref in zip(_export(kv, shape, s), (k, v)):
            assert np.array_equal(got, ref)
    return out


@pytest.mark.parametrize("shape", [SMALL, WIDE], ids=lambda s: s.name)
@pytest.mark.parametrize("batch", [1, 2, 3, 16, 40])
@pytest.mark.parametrize("static", [False, True])
def test_forward_decode(shape, batch, static):
    require_gpu()
    model, orc, _ = make_pair(shape, max_rows=64, max_positions=1024)
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(1, 260 if batch > 3 else 900, batch)]
    lens[0] = 47
    kv = L.KVCache(model, sum(n // 16 + 2 for n in lens) + 4, batch, 64, poison=True)
    states = _states(kv, shape, lens, 1024)
    step = L.laser_decode_step_static if static else L.laser_decode_step
    toks = [int(t) for t in synth.make_tokens(batch, shape.vocab, 77)]
    for turn in range(2):
        d_tok = torch.tensor(toks, dtype=torch.int32, device="cuda")
        d_next, d_p = torch.zeros_like(d_tok), torch.zeros(batch, device="cuda")
        d_logits = torch.zeros(batch, shape.vocab, device="cuda")
        step(model, kv, list(range(batch)), d_tok, d_next, d_p, d_logits)
        torch.cuda.synchronize()
        for b in range(batch):
            ref = orc.decode_token(states[b], toks[b])
            if turn == 0 or batch <= 3:
                _adopt(kv, shape, b, states[b], lens[b] + turn)
            compare_logits(d_logits[b].cpu().numpy(), ref, f"seq {b}")
            check_token(d_next[b].item(), ref, f"seq {b}")
            check_prob(d_p[b].item(), lm_stats(ref)[1])
            toks[b] = lm_stats(ref)[0]


@pytest.mark.parametrize("shape", [SMALL, WIDE], ids=lambda s: s.name)
@pytest.mark.parametrize("n", [1, 5, 33, 200])
def test_prefill_then_own_rows(shape, n):
    """A prompt through laser_prefill, its first layer's keys as the oracle's; what the cache holds, attended by laser_attend."""
    require_gpu()
    model, orc, _ = make_pair(shape, max_rows=64, max_positions=512)
    kv = L.KVCache(model, 40, 1, 20, poison=True)
    kv.add_seq(0, 0)
    st = SeqState(shape, 512)
    toks = synth.make_tokens(n, shape.vocab, 5)
    L.laser_prefill(model, kv, 0, toks.cuda(), torch.zeros(shape.vocab, device="cuda"))
    torch.cuda.synchronize()
    for t in toks:
        orc.decode_token(st, int(t))
    K, V = _export(kv, shape, 0)
    for got, ref in ((K, st.K), (V, st.V)):  # (layer 0 depends on no attention: a few codes next to borders at most)
        assert (got[0] != ref[0, :n]).mean() <= 0.002 + 4 / got[0].size
    for layer in range(shape.n_layers):
        q = torch.randn(n, shape.n_q_heads, shape.head_dim, device="cuda")
        o = torch.empty_like(q)
        L.laser_attend(kv, layer, [L.attend_span(0, n, 0)], q, o)
        torch.cuda.synchronize()
        ref, _ = attend(f64(q), K[layer], V[layer], 0, shape.head_dim ** -0.5)
        assert np.all(np.abs(f64(o) - ref) <= tolerance("f32", ref, V[layer], f64(q), K[layer], shape.head_dim ** -0.5))


def test_fork_and_probe():
    """The probe call, and a probe on a fork beside a decode step (its partial page, scales included, is a copy)."""
    require_gpu()
    shape = SMALL
    model, orc, _ = make_pair(shape, max_rows=64, max_positions=512)
    kv = L.KVCache(model, 60, 4, 30, poison=True)
    states = _states(kv, shape, [37, 100], 512)
    suffix = [int(t) for t in synth.make_suffix(8, shape.vocab)]
    d_suffix = torch.tensor(suffix, dtype=torch.int32, device="cuda")
    before = [_export(kv, shape, s) for s in (0, 1)]
    conf, arg = torch.zeros(2, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    L.laser_probe_confidence(model, kv, [0, 1], d_suffix, 4, conf, arg)
    kv.fork(0, 2)
    tok = torch.tensor([11], dtype=torch.int32, device="cuda")
    t0, p0, t1, p1 = (torch.zeros(1, dtype=d, device="cuda") for d in (torch.int32, torch.float32) * 2)
    logits, flog = torch.zeros(1, shape.vocab, device="cuda"), torch.zeros(1, shape.vocab, device="cuda")
    L.laser_forward(model, kv, [L.span(0, 1, 0, 0, out=(0, 0)), L.span(2, 8, 1, 0, out=(1, 0))], tok, d_suffix, t0, p0, t1, p1,
                    logits, flog)
    torch.cuda.synchronize()
    assert torch.isfinite(conf).all() and (conf > 0).all() and (conf <= 1).all()
    for s in (0, 1):  # what was there is as it was
        for got, ref in zip(_export(kv, shape, s), before[s]):
            assert np.array_equal(got[:, :ref.shape[1]], ref)
    fork = SeqState.from_prefill(shape, states[0].K[:, :37], states[0].V[:, :37], 512)
    compare_logits(logits[0].cpu().numpy(), orc.decode_token(states[0], 11), "decode beside the probe")
    # the fork's suffix, token by token from what the cache holds
    K, V = _export(kv, shape, 2)
    for i, t in enumerate(suffix):
        ref = orc.decode_token(fork, t)
        fork.K[:, 37 + i], fork.V[:, 37 + i] = K[:, 37 + i], V[:, 37 + i]
    compare_logits(flog[0].cpu().numpy(), ref, "fork")


class Setup4(Setup):
    """Setup, with the oracle's pre-filled K/V as the 4-bit cache keeps them."""

    def __init__(self, shape, lens):
        super().__init__(shape, lens)
        for st, n in zip(self.states, lens):
            for x in (st.K, st.V):
                x[:, :n] = round_mxfp4_rows(x[:, :n])


@pytest.mark.parametrize("shape,lens", [(QWEN_1P5B_FP4KV, [4096]), (QWEN_7B_FP4KV, [14336])], ids=["1.5B", "7B"])
def test_full_shapes(shape, lens):
    st = Setup4(shape, lens)
    st.decode(1)
    st.release()
