"""What a forward leaves in an INT8 cache, exactly: a model whose first layer makes K and V rows that are known to the
last bit, against the definition in float64 and against the same rows through laser_kv_write, on every projection path;
and prompts at the edge of a forward's 512 rows against the oracle.

With embeddings of 8 at one of 64 dims the norm's 1 / rms is 1, so that a token's normalised input is 8 at its dim
and its V (and K at position 0, where the rotation is none) is 8 times a column of the weights (plus the bias)."""
import numpy as np
import pytest
import torch

from gpu_helpers import compare_logits, make_pair, require_gpu
from oracle.transformer import SeqState
from paged_ref import kept
from paper_2606_31580_amd import laser as L
from paper_2606_31580_amd import synth
from paper_2606_31580_amd.configs import ModelShape
from test_gpu_16_kv_rows import f64, stored_tol
from test_gpu_18_int8_kv import SMALL, WIDE, _check_kv

pytestmark = pytest.mark.gpu
_made = {}


def known(hq, hkv, hd, bias):
    """(model, float32 K and V rows of each token) of a shape."""
    require_gpu()
    key = (hq, hkv, hd, bias)
    if key not in _made:
        shape = ModelShape("known-%d-%d-%d-%d" % key, 1, 64, hq, hkv, hd, 64, 64, False, bias, "bf16", 1.0e4, 1.0e-30, "int8")
        w = synth.make_weights(shape, seed_base=7000)
        w["embed"] = (8 * torch.eye(64)).to(torch.bfloat16)
        g = torch.Generator().manual_seed(60)
        rows = []
        for name in ("k", "v"):
            m = torch.randn(hkv * hd, 64, generator=g) * torch.exp(torch.randn(hkv * hd, 64, generator=g))
            m[:, 5] = 0.0                                                  # a token whose row is zero but for the bias
            m[:, 6] = 0.5 ** torch.randint(0, 9, (hkv * hd,), generator=g)   # amax / 2: 63.5 steps, and so on
            m[:, 7] = torch.randint(-254, 255, (hkv * hd,), generator=g) / 254.0  # (in bf16 most are no half steps)
            m[0, 7] = 1.0
            w["layers.0.w" + name] = m.to(torch.bfloat16)
            x = 8.0 * w["layers.0.w" + name].float().t()
            if bias:
                w["layers.0.b" + name] = torch.randn(hkv * hd, generator=g).to(torch.bfloat16)
                x = x + w["layers.0.b" + name].float()
            rows.append(x.reshape(64, hkv, hd).contiguous())
        model = L.Model(shape, {k: t.cuda() for k, t in w.items()}, max_rows=64, max_positions=1024, poison=True)
        _made[key] = (model, rows)
    return _made[key]


SHAPES = pytest.mark.parametrize("hq,hkv,hd,bias", [(4, 2, 64, False), (7, 1, 128, True), (6, 3, 128, False)])


def check_rows(got, src, bias):
    """Values read back in fp32 against the definition: rows of bf16 numbers exactly (their quotients are a half or far
    from it), sums with a bias as test_gpu_16_kv_rows has it for fp32 rows."""
    ref = kept("int8", src)
    assert np.all(np.abs(got - ref) <= stored_tol("int8", "f32", ref, src)), np.abs(got - ref).max()
    if not bias:
        assert np.all(np.abs(got - ref) <= 3 * 2.0 ** -24 * np.abs(ref))


@SHAPES
@pytest.mark.parametrize("batch", [1, 2, 4, 5, 16, 17, 40, 64])
@pytest.mark.parametrize("static", [False, True])
def test_first_positions_of_a_batch(hq, hkv, hd, bias, batch, static):
    model, rows = known(hq, hkv, hd, bias)
    toks = torch.arange(batch, dtype=torch.int32) * 11 % 64
    caches = [L.KVCache(model, batch + 3, batch, 4, poison=True) for _ in range(2)]
    for s in range(batch):
        for kv in caches:
            kv.add_seq(s, 0)
    nxt, p = torch.zeros(batch, dtype=torch.int32, device="cuda"), torch.zeros(batch, device="cuda")
    step = L.laser_decode_step_static if static else L.laser_decode_step
    step(model, caches[0], list(range(batch)), toks.cuda(), nxt, p)
    src = [x[toks.long()] for x in rows]
    runs = [L.kv_run(s, 0, 1, s) for s in range(batch)]
    for s in range(batch):
        caches[1].append(s, 1)
    L.laser_kv_write(caches[1], 0, runs, *(x.cuda() for x in src))
    out = [torch.empty_like(x, device="cuda") for x in src]
    L.laser_kv_read(caches[0], 0, runs, *out)
    torch.cuda.synchronize()
    # the same bytes, scales and untouched places among them
    assert torch.equal(caches[0].k_pool, caches[1].k_pool) and torch.equal(caches[0].v_pool, caches[1].v_pool)
    for got, x in zip(out, src):
        check_rows(f64(got), f64(x), bias)


@SHAPES
@pytest.mark.parametrize("n", [3, 16, 33, 200, 512, 513, 700])
def test_values_of_a_prompt(hq, hkv, hd, bias, n):
    """V of every position of a prompt, also over the 512 rows of a forward; K within half a step of the rotated rows."""
    model, (rk, rv) = known(hq, hkv, hd, bias)
    caches = [L.KVCache(model, 50, 1, 50, poison=True) for _ in range(2)]
    caches[0].add_seq(0, 0)
    caches[1].add_seq(0, n)
    toks = synth.make_tokens(n, 64, 9)
    L.laser_prefill(model, caches[0], 0, toks.cuda(), torch.zeros(64, device="cuda"))
    k, v = rk[toks.long()], rv[toks.long()]
    run = [L.kv_run(0, 0, n)]
    L.laser_kv_write(caches[1], 0, run, k.cuda(), v.cuda())
    out = [torch.empty_like(k, device="cuda") for _ in range(2)]
    L.laser_kv_read(caches[0], 0, run, *out)
    torch.cuda.synchronize()
    assert torch.equal(caches[0].v_pool, caches[1].v_pool)
    check_rows(f64(out[1]), f64(v), bias)
    angle = np.arange(n)[:, None] * 1.0e4 ** (-np.arange(hd // 2) / (hd // 2))[None, :]
    c, s = np.cos(angle)[:, None, :], np.sin(angle)[:, None, :]
    lo, hi = f64(k)[..., :hd // 2], f64(k)[..., hd // 2:]
    turned = np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)
    top = np.abs(turned).max(-1, keepdims=True)
    # Half a step (amax / 127).  The fp32 rotation is off by less than 1e-4 amax before it: angles up to 700 are fp32
    # numbers, 700 x 2^-24 = 4.2e-5 off each in sine and cosine, of a lo and a hi of up to amax each.
    assert np.all(np.abs(f64(out[0]) - turned) <= (0.5 / 127 + 1.0e-4) * top + 1e-30)


@pytest.mark.parametrize("shape", [SMALL, WIDE], ids=lambda s: s.name)
@pytest.mark.parametrize("n", [512, 513])
def test_prompts_at_the_edge_of_a_forward(shape, n):
    model, orc, _ = make_pair(shape, max_rows=64, max_positions=1024)
    kv = L.KVCache(model, 40, 1, 40, poison=True)
    kv.add_seq(0, 0)
    st = SeqState(shape, 1024)
    toks = synth.make_tokens(n, shape.vocab, 5)
    logits = torch.zeros(shape.vocab, device="cuda")
    L.laser_prefill(model, kv, 0, toks.cuda(), logits)
    torch.cuda.synchronize()
    for t in toks:
        ref = orc.decode_token(st, int(t))
    compare_logits(logits.cpu().numpy(), ref, f"prefill {n}")
    _check_kv(kv, shape, 0, st)
