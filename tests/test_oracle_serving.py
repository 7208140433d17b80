"""Pins of the oracles for pages, rotary positions and adjusted logits (CPU)."""
import math

import numpy as np
import pytest

from oracle import (adjust_logits, commit_kv, gather_pages, paged_attention, paged_write, rotary_angles, rotate, tree_attention)
from workloads import static_tree


def _pages(rng, B, Hkv, Dh, size, per_item):
    n = B * per_item + 2
    table = rng.permutation(n)[:B * per_item].reshape(B, per_item).astype(np.int32)
    return rng.standard_normal((n, Hkv, size, Dh)), rng.standard_normal((n, Hkv, size, Dh)), table


def test_paged_attention_is_tree_attention_on_the_gathered_cache():
    rng = np.random.default_rng(1)
    parent = static_tree((3, 2, 1), 9)
    B, H, Hkv, M, Dh, size = 2, 4, 2, 10, 8, 16
    kp, vp, table = _pages(rng, B, Hkv, Dh, size, 3)
    q, kn, vn = (rng.standard_normal((B, h, M, Dh)) for h in (H, Hkv, Hkv))
    lens = np.array([41, 7])
    got = paged_attention(q, kp, vp, table, kn, vn, lens, parent)
    for b in range(B):
        k, v = (gather_pages(x, table, b, lens[b])[None] for x in (kp, vp))
        want = tree_attention(q[b:b + 1], k, v, kn[b:b + 1], vn[b:b + 1], parent)
        assert np.allclose(got[b], want[0], rtol=0, atol=1e-13)


def test_a_chunk_is_a_chain_of_rows_and_ends_at_its_length():
    rng = np.random.default_rng(2)
    B, H, M, Dh, size = 2, 2, 6, 8, 16
    kp, vp, table = _pages(rng, B, H, Dh, size, 2)
    q, kn, vn = (rng.standard_normal((B, H, M, Dh)) for _ in range(3))
    lens = np.array([20, 0])
    chain = np.arange(-1, M - 1)
    whole = paged_attention(q, kp, vp, table, kn, vn, lens, chain)
    kn[1, :, 4:] = np.nan
    got = paged_attention(q, kp, vp, table, kn, vn, lens, row_len=np.array([6, 4]))
    assert np.allclose(got[0], whole[0], rtol=0, atol=1e-13) and np.allclose(got[1, :, :4], whole[1, :, :4], rtol=0, atol=1e-13)
    assert np.isnan(got[1, :, 4:]).all()


def test_paged_write_is_commit_on_the_gathered_cache():
    rng = np.random.default_rng(3)
    B, H, M, Dh, size, per = 3, 2, 7, 4, 16, 2
    kp, vp, table = _pages(rng, B, H, Dh, size, per)
    kn, vn = (rng.standard_normal((B, H, M, Dh)) for _ in range(2))
    path = np.array([[2, 5, -1], [1, -1, -1], [3, 4, 6]])
    accept, lens = np.array([2, 0, 3]), np.array([9, 31, 29])
    rows = [[0] + path[b, :accept[b]].tolist() for b in range(B)]
    k2, v2, new_len = paged_write(kp, vp, kn, vn, rows, table, lens)
    full = [np.stack([gather_pages(x, table, b, per * size) for b in range(B)]) for x in (kp, vp)]
    kc, vc, want = commit_kv(full[0], full[1], kn, vn, path, accept, lens)
    assert np.array_equal(new_len, want)
    for b in range(B):
        assert np.array_equal(gather_pages(k2, table, b, per * size), kc[b])
        assert np.array_equal(gather_pages(v2, table, b, per * size), vc[b])
    table[1, 1] = -1                                       # a position without a page is left out
    k3, _, new_len = paged_write(kp, vp, kn, vn, rows, table, lens)
    assert new_len[1] == want[1] and np.array_equal(k3[k3 != k2], kp[k3 != k2])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
def test_products_depend_on_distance_alone(layout, scaling):
    rng = np.random.default_rng(4)
    theta, m = rotary_angles(16, scaling=scaling, factor=4.0, original_len=64)
    x, y = rng.standard_normal((2, 24))

    def product(p, r):
        return float(rotate(x, p, theta, m, layout) @ rotate(y, r, theta, m, layout))

    assert math.isclose(product(3, 11), product(103, 111), rel_tol=1e-9)
    assert np.allclose(rotate(x, 0, theta, 1.0, layout), x)
    assert np.array_equal(rotate(x, 9, theta, m, layout)[16:], x[16:])


def test_rotary_hand_values():
    theta, m = rotary_angles(4)
    assert np.allclose(theta, [1.0, 0.01]) and m == 1.0
    y = rotate(np.array([1.0, 0.0, 0.0, 0.0]), math.pi / 2, theta, 1.0, "half")
    assert np.allclose(y, [0, 0, 1, 0], atol=1e-15)
    y = rotate(np.array([1.0, 0.0, 0.0, 0.0]), math.pi / 2, theta, 1.0, "interleaved")
    assert np.allclose(y, [0, 1, 0, 0], atol=1e-15)
    assert np.allclose(rotary_angles(4, scaling="linear", factor=2.0)[0], [0.5, 0.005])
    assert np.allclose(rotary_angles(4, scaling="ntk", factor=2.0)[0], [1.0, (10000.0 * 4) ** -0.5])
    # turns in 4096 positions: 652 (keeps its angle) and 6.5 (between slow and fast)
    t, m = rotary_angles(4, scaling="yarn", factor=8.0, original_len=4096)
    g = (40.96 / (2 * math.pi) - 1) / 31
    assert np.allclose(t, [1.0, 0.01 * (g + (1 - g) / 8)]) and math.isclose(m, 1 + 0.1 * math.log(8))


def test_adjusted_logits_special_cases():
    rng = np.random.default_rng(5)
    parent = np.array([-1, 0, 0, 1])
    c, u = rng.standard_normal((2, 1, 4, 5))
    assert np.array_equal(adjust_logits(parent, c)[0], c)
    assert np.allclose(adjust_logits(parent, c, u, 1.0)[0], c) and np.array_equal(adjust_logits(parent, c, u, 0.0)[0], u)
    tokens = np.array([[4, 2, 2, 2]])
    got = adjust_logits(parent, c, tokens=tokens, frequency=[10.0], presence=[100.0])[0]
    want = c.copy()
    want[0, 1, 2] -= 110
    want[0, 2, 2] -= 110
    want[0, 3, 2] -= 120                                   # twice on its path; the root's token is history
    assert np.allclose(got, want)
    counts = np.array([[0, 3, 0, 0, 0]])
    got = adjust_logits(parent, c, counts=counts, repetition=[2.0])[0]
    want = c.copy()
    want[..., 1] = np.where(c[..., 1] > 0, c[..., 1] / 2, c[..., 1] * 2)
    assert np.allclose(got, want)
    c[0, 0, 0] = np.nan
    got = adjust_logits(parent, c, mask=np.zeros(5, dtype=bool))[0]
    assert (got == -np.inf).all()
