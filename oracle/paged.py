"""Oracle: attention of new tokens over a cache in pages, and what commit and append write into it (App. A.2 for the tree;
a chunk is plain causal attention).

TEST INFRASTRUCTURE ONLY -- never imported by the product path.

Position p of item b lies in slot p % size of page table[b, p // size]; pages are [n_pages, Hkv, size, Dh].
"""
from typing import Optional, Tuple

import numpy as np

from .attention import ancestor_mask


def gather_pages(pages: np.ndarray, table: np.ndarray, b: int, n: int) -> np.ndarray:
    """Positions [0, n) of item b: [Hkv, n, Dh] float64 (table entries clamped to the pool)."""
    size = pages.shape[2]
    at = np.arange(n)
    page = np.clip(table[b, at // size], 0, pages.shape[0] - 1)
    return np.asarray(pages[page, :, at % size], dtype=np.float64).transpose(1, 0, 2)


def paged_attention(q: np.ndarray, k_pages: np.ndarray, v_pages: np.ndarray, table: np.ndarray, k_new: np.ndarray,
                    v_new: np.ndarray, seq_len: np.ndarray, parent: Optional[np.ndarray] = None,
                    row_len: Optional[np.ndarray] = None, scale: Optional[float] = None) -> np.ndarray:
    """q [B,H,M,Dh], k_new and v_new [B,Hkv,M,Dh] -> out [B,H,M,Dh] float64; rows behind row_len are NaN.

    Every row sees its item's cached positions; of the new rows it sees its ancestors and itself (``parent`` given) or those up to
    and with itself.  What a row does not see plays no part, whatever it holds."""
    B, H, M, Dh = q.shape
    Hkv = k_new.shape[1]
    scale = 1.0 / np.sqrt(Dh) if not scale else float(scale)
    sees = ancestor_mask(parent) if parent is not None else np.tril(np.ones((M, M), dtype=bool))
    out = np.full((B, H, M, Dh), np.nan)
    for b in range(B):
        n = int(seq_len[b])
        K, V = gather_pages(k_pages, table, b, n), gather_pages(v_pages, table, b, n)
        for h in range(H):
            g = h // (H // Hkv)
            for i in range(M if row_len is None else int(row_len[b])):
                new = np.nonzero(sees[i])[0]
                Ki = np.concatenate([K[g], np.asarray(k_new[b, g, new], dtype=np.float64)])
                Vi = np.concatenate([V[g], np.asarray(v_new[b, g, new], dtype=np.float64)])
                with np.errstate(invalid="ignore"):      # (infinities that a row sees)
                    s = Ki @ np.asarray(q[b, h, i], dtype=np.float64) * scale
                    w = np.exp(s - s.max())
                    out[b, h, i] = (w / w.sum()) @ Vi
    return out


def paged_write(k_pages: np.ndarray, v_pages: np.ndarray, k_new: np.ndarray, v_new: np.ndarray, rows, table: np.ndarray,
                seq_len: np.ndarray) -> Tuple[np.ndarray, np.ndarray, np.ndarray]:
    """Rows ``rows[b]`` (a list) of item b go to positions seq_len[b], ...; copies (k_pages', v_pages', new_len)."""
    k, v = np.array(k_pages, copy=True), np.array(v_pages, copy=True)
    size, capacity = k.shape[2], table.shape[1] * k.shape[2]
    new_len = np.zeros(len(rows), dtype=np.int32)
    for b, kept in enumerate(rows):
        pos = min(max(int(seq_len[b]), 0), capacity)
        for r in kept:
            if pos < capacity and 0 <= table[b, pos // size] < k.shape[0]:
                k[table[b, pos // size], :, pos % size] = k_new[b, :, r]
                v[table[b, pos // size], :, pos % size] = v_new[b, :, r]
            pos += 1
        new_len[b] = min(pos, capacity)
    return k, v, new_len
