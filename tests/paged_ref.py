"""Float64 definitions of the paged cache's operators, for the tests: what a cache of each element type
keeps of a row, and attention over it.  numpy only; nothing here comes from the library."""
import numpy as np

from oracle.numerics import round_bf16, round_fp8_e4m3


def kept(kind, x):
    """The values that a cache of type `kind` stands for once it holds the rows x [..., hd]."""
    x = np.asarray(x, dtype=np.float64)
    if kind == "int8":
        top = np.abs(x).max(-1, keepdims=True)
        with np.errstate(invalid="ignore", divide="ignore"):
            q = np.where(top > 0, np.rint(127.0 * x / np.where(top > 0, top, 1.0)), 0.0)
            out = q * (top / 127.0)
        return np.where(np.isfinite(x).all(-1, keepdims=True), out, np.nan)
    if kind == "fp8":
        return round_fp8_e4m3(x)
    return round_bf16(x) if kind == "bf16" else x


def attend(q, k, v, pos, scale, causal=True, window=0, kv_begin=0, kv_end=None):
    """q [n, hq, hd] at positions pos .. over k, v [len, hkv, hd]: (o [n, hq, hd], lse [n, hq]) in float64."""
    n, hq, hd = q.shape
    kv_end = k.shape[0] if kv_end is None else kv_end
    group = hq // k.shape[1]
    o, lse = np.zeros((n, hq, hd)), np.full((n, hq), -np.inf)
    for i in range(n):
        lo = kv_begin if window == 0 else max(kv_begin, pos + i - window + 1)
        hi = min(kv_end, pos + i + 1) if causal else kv_end
        if hi <= lo:
            continue
        for h in range(hq):
            s = scale * (k[lo:hi, h // group] @ q[i, h])
            if np.isnan(s).any() or np.isposinf(s).any():
                o[i, h], lse[i, h] = np.nan, np.nan
                continue
            m = s.max()
            if np.isneginf(m):
                continue
            p = np.exp(s - m)
            with np.errstate(invalid="ignore"):
                o[i, h] = (p / p.sum()) @ v[lo:hi, h // group]
            lse[i, h] = m + np.log(p.sum())
    return o, lse
