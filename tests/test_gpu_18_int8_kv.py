"""The INT8 KV cache (8-bit integers, a scale per position and kv head) under the model's own forward,
against the oracle that rounds K/V the same way: tiny models on every projection path (1 to 64 rows,
prompts in wide forwards), forks and riding probes, the static decode step, and state injection at
full size as in test_gpu_2_full_shapes."""
import numpy as np
import pytest
import torch

from gpu_helpers import check_prob, check_token, compare_logits, make_pair, require_gpu
from oracle.numerics import round_int8_rows
from oracle.transformer import SeqState, lm_stats
from paper_2606_31580_amd import laser as L
from paper_2606_31580_amd import synth
from paper_2606_31580_amd.configs import ModelShape, QWEN_1P5B_INT8KV, QWEN_7B_INT8KV
from test_gpu_2_full_shapes import Setup, log

pytestmark = pytest.mark.gpu

SMALL = ModelShape("small-int8kv", 2, 256, 4, 2, 64, 672, 2048, False, True, "bf16", 1.0e4, 1.0e-5, "int8")
WIDE = ModelShape("small-int8kv-128", 2, 256, 7, 1, 128, 680, 2048, True, False, "bf16", 1.0e4, 1.0e-5, "int8")


def _states(kv, shape, lens, capacity):
    """Sequences with pre-filled bf16 K/V on the device, and what the INT8 cache makes of them in the oracle."""
    out = []
    for s, n in enumerate(lens):
        k0, v0 = synth.make_prefill_kv(shape, n, s)
        kv.add_seq(s, n)
        if n:
            kv.import_kv(s, k0.cuda(), v0.cuda())
        k, v = (round_int8_rows(t.float().numpy()) for t in (k0, v0))
        out.append(SeqState.from_prefill(shape, k, v, capacity))
    return out


def _export(kv, shape, seq):
    n = kv.seq_len(seq)
    o = [torch.empty((shape.n_layers, n, shape.n_kv_heads, shape.head_dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kv.export_kv(seq, *o)
    torch.cuda.synchronize()
    return [t.float().cpu().numpy().astype(np.float64) for t in o]


def _check_kv(kv, shape, seq, state):
    """Cached K/V within one step (amax / 127) of the oracle's, and the bf16 of the export."""
    for got, ref in zip(_export(kv, shape, seq), (state.K, state.V)):
        ref = ref[:, :got.shape[1]]
        step = np.abs(ref).max(-1, keepdims=True) / 127.0
        assert np.all(np.abs(got - ref) <= 1.02 * step + 2.0 ** -8 * np.abs(ref))


@pytest.mark.parametrize("shape", [SMALL, WIDE], ids=lambda s: s.name)
@pytest.mark.parametrize("batch", [1, 2, 3, 16, 20, 40, 64])
@pytest.mark.parametrize("static", [False, True])
def test_decode(shape, batch, static):
    require_gpu()
    model, orc, _ = make_pair(shape, max_rows=64, max_positions=1024)
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(1, 260 if batch > 3 else 900, batch)]
    lens[0] = 47
    kv = L.KVCache(model, sum(n // 16 + 2 for n in lens) + 4, batch, 64, poison=True)
    states = _states(kv, shape, lens, 1024)
    step = L.laser_decode_step_static if static else L.laser_decode_step
    toks = [int(t) for t in synth.make_tokens(batch, shape.vocab, 77)]
    for _ in range(2):
        d_tok = torch.tensor(toks, dtype=torch.int32, device="cuda")
        d_next, d_p = torch.zeros_like(d_tok), torch.zeros(batch, device="cuda")
        d_logits = torch.zeros(batch, shape.vocab, device="cuda")
        step(model, kv, list(range(batch)), d_tok, d_next, d_p, d_logits)
        torch.cuda.synchronize()
        for b in range(batch):
            ref = orc.decode_token(states[b], toks[b])
            compare_logits(d_logits[b].cpu().numpy(), ref, f"seq {b}")
            check_token(d_next[b].item(), ref, f"seq {b}")
            check_prob(d_p[b].item(), lm_stats(ref)[1])
            toks[b] = lm_stats(ref)[0]
    for b in range(0, batch, 7):
        _check_kv(kv, shape, b, states[b])


@pytest.mark.parametrize("shape", [SMALL, WIDE], ids=lambda s: s.name)
@pytest.mark.parametrize("n", [1, 5, 33, 200])
def test_prefill_then_own_rows(shape, n):
    """A prompt through laser_prefill; its cached positions attended by laser_attend give what the cache holds."""
    require_gpu()
    model, orc, _ = make_pair(shape, max_rows=64, max_positions=512)
    kv = L.KVCache(model, 40, 1, 20, poison=True)
    kv.add_seq(0, 0)
    st = SeqState(shape, 512)
    toks = synth.make_tokens(n, shape.vocab, 5)
    logits = torch.zeros(shape.vocab, device="cuda")
    L.laser_prefill(model, kv, 0, toks.cuda(), logits)
    torch.cuda.synchronize()
    for t in toks:
        ref = orc.decode_token(st, int(t))
    compare_logits(logits.cpu().numpy(), ref, f"prefill {n}")
    _check_kv(kv, shape, 0, st)
    # the forward's write and laser_kv_write agree on the bytes: read back, written again, the pools are the same
    for layer in range(shape.n_layers):
        k, v = (torch.empty(n, shape.n_kv_heads, shape.head_dim, device="cuda") for _ in range(2))
        L.laser_kv_read(kv, layer, [L.kv_run(0, 0, n)], k, v)
        q = torch.randn(n, shape.n_q_heads, shape.head_dim, device="cuda")
        o = torch.empty_like(q)
        L.laser_attend(kv, layer, [L.attend_span(0, n, 0)], q, o)
        torch.cuda.synchronize()
        g = shape.n_q_heads // shape.n_kv_heads
        K, V = (x.double().repeat_interleave(g, 1).transpose(0, 1) for x in (k, v))
        s = (q.double().transpose(0, 1) @ K.transpose(1, 2).contiguous()) * shape.head_dim ** -0.5
        s = s.masked_fill(~torch.ones(n, n, dtype=torch.bool, device="cuda").tril(), float("-inf"))
        ref = (torch.softmax(s, -1) @ V).transpose(0, 1)
        assert float((o.double() - ref).abs().max()) <= 1e-5 * float(V.abs().max())


def test_fork_and_riding_probe():
    """A probe on a fork beside decode steps (its partial page, scales included, is a copy), and the probe call."""
    require_gpu()
    shape = SMALL
    model, orc, _ = make_pair(shape, max_rows=64, max_positions=512)
    kv = L.KVCache(model, 60, 4, 30, poison=True)
    states = _states(kv, shape, [37, 100], 512)
    suffix = [int(t) for t in synth.make_suffix(8, shape.vocab)]
    d_suffix = torch.tensor(suffix, dtype=torch.int32, device="cuda")
    conf, arg = torch.zeros(2, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    L.laser_probe_confidence(model, kv, [0, 1], d_suffix, 4, conf, arg)
    torch.cuda.synchronize()
    for b in range(2):
        res = orc.probe(states[b], suffix, 4)
        if [int(x) for x in arg[4 * b:4 * b + 4].cpu()] == res.tokens:
            check_prob(conf[b].item(), res.confidence)
        else:
            assert min(res.margins) <= 1e-2
    # fork 0 -> 2, decode 0 and run the suffix on the fork in one forward
    kv.fork(0, 2)
    tok = torch.tensor([11], dtype=torch.int32, device="cuda")
    t0, p0, t1, p1 = (torch.zeros(1, dtype=d, device="cuda") for d in (torch.int32, torch.float32) * 2)
    logits = torch.zeros(1, shape.vocab, device="cuda")
    flog = torch.zeros(1, shape.vocab, device="cuda")
    L.laser_forward(model, kv, [L.span(0, 1, 0, 0, out=(0, 0)), L.span(2, 8, 1, 0, out=(1, 0))], tok, d_suffix, t0, p0, t1, p1,
                    logits, flog)
    torch.cuda.synchronize()
    fork = SeqState.from_prefill(shape, states[0].K[:, :37], states[0].V[:, :37], 512)
    compare_logits(logits[0].cpu().numpy(), orc.decode_token(states[0], 11), "decode beside the probe")
    for t in suffix:
        ref = orc.decode_token(fork, t)
    compare_logits(flog[0].cpu().numpy(), ref, "fork")
    _check_kv(kv, shape, 2, fork)
    _check_kv(kv, shape, 0, states[0])


class SetupInt8(Setup):
    """Setup, with the oracle's pre-filled K/V as the INT8 cache keeps them."""

    def __init__(self, shape, lens):
        super().__init__(shape, lens)
        for st, n in zip(self.states, lens):
            for x in (st.K, st.V):
                x[:, :n] = round_int8_rows(x[:, :n])


@pytest.mark.parametrize("shape,lens", [(QWEN_1P5B_INT8KV, [4096]), (QWEN_7B_INT8KV, [14336])], ids=["1.5B", "7B"])
def test_full_shapes(shape, lens):
    st = SetupInt8(shape, lens)
    st.decode(2 if shape is QWEN_1P5B_INT8KV else 1)
    st.probe([0])
    st.release()
