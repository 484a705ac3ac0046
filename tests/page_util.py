"""Plain 64-bit definitions of the paged-cache operators for the tests (numpy; nothing of the library in here)."""
import math

import numpy as np
import torch

STORES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}
ROWS = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TOP = {"i8": 127.0, "e4m3": 448.0}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}   # finfo.eps / 2
E4M3 = np.array([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1])


def f64(t):
    """Any tensor as a float64 array (8-bit floats through float32, which holds them)."""
    return (t.float() if t.dtype != torch.float64 else t).double().cpu().numpy()


def nearest_e4m3(y):
    a = np.abs(y)
    hi = np.clip(np.searchsorted(E4M3, a), 1, len(E4M3) - 1)
    lo = hi - 1
    below, above = a - E4M3[lo], E4M3[hi] - a
    return np.copysign(E4M3[np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)], y)


def quantise(x, store):
    """float64 rows [..., dim] -> (stored values, fp32 scales); rows that are not finite: (0, NaN)."""
    top = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1)
    with np.errstate(invalid="ignore"):
        scale = np.maximum((top / TOP[store]).astype(np.float32), np.float32(2.0 ** -80))
        y = x / scale.astype(np.float64)[..., None]
    scale[bad], y[bad] = np.nan, 0.0
    return (np.rint(y) if store == "i8" else nearest_e4m3(y)), scale


def pool_values(pages, layer=0):
    """k, v of a layer as float64 [page, head, row, dim], scales applied."""
    out = []
    for x, s in ((pages.k, pages.k_scale), (pages.v, pages.v_scale)):
        w = f64(x.view(torch.uint8)[layer].view(x.dtype) if x.dtype == torch.float8_e4m3fn else x[layer])
        out.append(w if s is None else w * f64(s[layer])[..., None])
    return out


def attention(q, k, v, scale):
    """q [heads, dim], k, v [positions, dim] -> [heads, dim] and the largest sum of |q||k| scale."""
    if len(k) == 0:
        return np.zeros_like(q), 0.0
    s = q @ k.T * scale
    w = np.exp(s - s.max(-1, keepdims=True))
    return (w @ v) / w.sum(-1, keepdims=True), float((np.abs(q) @ np.abs(k).T).max() * abs(scale))


def select(logits, scores, finished, eos):
    """[groups, width, vocab] float64 -> tokens, parents, scores, finished; ties: lower beam, then lower token."""
    g, w, v = logits.shape
    tokens, parents = np.zeros((g, w), np.int32), np.zeros((g, w), np.int32)
    out, done = np.zeros((g, w)), np.zeros((g, w), bool)
    for b in range(g):
        found = []
        for i in range(w):
            if finished is not None and finished[b, i]:
                found.append((scores[b, i], i, eos))
                continue
            if scores[b, i] == -math.inf:
                found += [(-math.inf, i, j) for j in range(min(w, v))]
                continue
            x = logits[b, i]
            m = x.max()
            with np.errstate(invalid="ignore", divide="ignore"):
                lse = m + np.log(np.exp(x - m).sum())
            for j in np.argsort(-x, kind="stable")[:w]:
                found.append((scores[b, i] + (x[j] - lse) if x[j] != -math.inf else -math.inf, i, int(j)))
        found.sort(key=lambda f: (-f[0], f[1], f[2]))
        for r, (s, i, j) in enumerate(found[:w]):
            tokens[b, r], parents[b, r], out[b, r] = j, i, s
            done[b, r] = (finished is not None and finished[b, i]) or j == eos
    return tokens, parents, out, done
