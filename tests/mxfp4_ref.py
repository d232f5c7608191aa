"""What the tests of 4-bit caches share: caches of small models, rows, and sequences filled with them."""
import numpy as np
import torch

from gpu_helpers import require_gpu
from oracle.numerics import round_mxfp4_rows
from paged_ref import kept as kept_others
from paper_2606_31580_amd import laser as L
from paper_2606_31580_amd import synth
from paper_2606_31580_amd.configs import ModelShape

IO = {"bf16": torch.bfloat16, "f32": torch.float32}
_models = {}


def kept(kind, x):
    """The values that a cache of type `kind` stands for once it holds the rows x [..., hd]."""
    return round_mxfp4_rows(x) if kind == "mxfp4" else kept_others(kind, x)


def cache(hq=4, hkv=2, hd=64, pages=96, seqs=6, per_seq=64, layers=2, kind="mxfp4", poison=True, mode=0):
    require_gpu()
    key = (kind, hq, hkv, hd, layers)
    if key not in _models:
        shape = ModelShape("rows-%s-%d-%d-%d-%d" % key, layers, 64, hq, hkv, hd, 64, 64, True, False,
                           "f32" if kind == "f32" else "bf16", 1.0e4, 1.0e-5, kind if kind in ("fp8", "int8", "mxfp4") else "")
        w = {k: v.cuda() for k, v in synth.make_weights(shape).items()}
        _models[key] = L.Model(shape, w, max_rows=4, max_positions=65536, tiles=False)
    _models[key].set_attend_kernel(mode)
    return L.KVCache(_models[key], pages, seqs, per_seq, poison=poison)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rows(rng, n, heads, hd, io, spread=1.0):
    """Rows whose heads, rows and channels differ in size."""
    x = rng.standard_normal((n, heads, hd)) * np.exp(spread * rng.standard_normal((n, heads, 1))) * np.exp(spread * rng.standard_normal((1, heads, hd)))
    return torch.from_numpy(x.astype(np.float32)).to(IO[io]).cuda()


def fill(kv, lens, hkv, hd, seed, layer=1, kind="mxfp4"):
    """Sequences of these lengths in `layer`; their K and V as the cache keeps them (float64)."""
    rng = np.random.default_rng(seed)
    held = []
    for s, n in enumerate(lens):
        kv.add_seq(s, n)
        k, v = (rows(rng, n, hkv, hd, "bf16", 0.3) for _ in range(2))
        if n:
            L.laser_kv_write(kv, layer, [L.kv_run(s, 0, n)], k, v)
        held.append((kept(kind, f64(k)), kept(kind, f64(v))))
    return held
