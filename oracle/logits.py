"""Oracle: guidance, penalties along a row's path, biases and masks on the target's logits, row by row in float64.

TEST INFRASTRUCTURE ONLY -- never imported by the product path.
"""
import numpy as np


def adjust_logits(parent, cond, uncond=None, cfg_scale=0.0, tokens=None, counts=None, repetition=None, frequency=None,
                  presence=None, bias=None, mask=None):
    """cond [B,M,V] -> (adjusted [B,M,V], size [B,M,V]: the sum of the magnitudes that went into every value).

    bias [V] or [B,V];  mask bool, broadcastable to [B,M,V], True = allowed."""
    cond = np.asarray(cond, dtype=np.float64)
    B, M, V = cond.shape
    out, size = np.empty_like(cond), np.empty_like(cond)
    for b in range(B):
        rep = 1.0 if repetition is None else float(repetition[b])
        freq = 0.0 if frequency is None else float(frequency[b])
        pres = 0.0 if presence is None else float(presence[b])
        for i in range(M):
            n = np.zeros(V) if counts is None else np.array(counts[b], dtype=np.float64)
            t = i
            while tokens is not None and t > 0:
                n[min(max(int(tokens[b, t]), 0), V - 1)] += 1
                t = int(parent[t])
            with np.errstate(invalid="ignore"):
                l, s = cond[b, i].copy(), np.abs(cond[b, i])
                if uncond is not None:
                    u = np.asarray(uncond[b, i], dtype=np.float64)
                    l, s = u + cfg_scale * (l - u), np.abs(u) + abs(cfg_scale) * (s + np.abs(u))
                l = np.where(n > 0, np.where(l > 0, l / rep, l * rep) - freq * n - pres, l)
                s = np.where(n > 0, s * max(abs(rep), 1 / abs(rep)) + abs(freq) * n + abs(pres), s)
                if bias is not None:
                    add = np.asarray(bias if np.ndim(bias) == 1 else bias[b], dtype=np.float64)
                    l, s = l + add, s + np.abs(add)
            out[b, i], size[b, i] = l, s
    if mask is not None:
        out[~np.broadcast_to(mask, out.shape)] = -np.inf
    return out, size
