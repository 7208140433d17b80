"""GPU: commit and append into pages against the oracle, bit for bit (pure data movement)."""
import numpy as np
import pytest
import torch

import paper_2502_06352_amd as lpp
from oracle import paged_write
from workloads import static_tree
from gpu_common import DEV, dev

pytestmark = pytest.mark.gpu


def _case(rng, B, Hkv, M, Dh, size, per_item, dtype):
    n = B * per_item + 2
    table = rng.permutation(n)[:B * per_item].reshape(B, per_item).astype(np.int32)

    def t(*shape):
        return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(dtype)

    return dict(kp=t(n, Hkv, size, Dh), vp=t(n, Hkv, size, Dh), kn=t(B, Hkv, M, Dh), vn=t(B, Hkv, M, Dh)), table


def _compare(x, table, rows, seq, got, new_len):
    host = {n: v.float().numpy() for n, v in x.items()}
    k, v, want = paged_write(host["kp"], host["vp"], host["kn"], host["vn"], rows, table, seq)
    assert np.array_equal(new_len.cpu().numpy(), want)
    assert np.array_equal(got[0].float().cpu().numpy(), k) and np.array_equal(got[1].float().cpu().numpy(), v)


@pytest.mark.parametrize("dtype,Dh,Hkv,size,B", [("bf16", 64, 24, 64, 4), ("bf16", 128, 8, 16, 3), ("f32", 64, 1, 32, 1),
                                                 ("f32", 128, 5, 256, 5)])
def test_commit(dtype, Dh, Hkv, size, B):
    rng = np.random.default_rng(B)
    parent = static_tree((6, 3, 2, 2, 1, 1), 60)
    tree = lpp.Tree(parent)
    code, tt = (lpp.LPP_BF16, torch.bfloat16) if dtype == "bf16" else (lpp.LPP_F32, torch.float32)
    x, table = _case(rng, B, Hkv, tree.M, Dh, size, 3, tt)
    cap = 3 * size
    # empty, over a page's end, room for part of the path, none, a length out of range
    seq = np.array([0, size - 2, cap - 2, cap, -5][:B], dtype=np.int32)
    path = np.full((B, tree.depth), -1, dtype=np.int32)
    accept = np.zeros(B, dtype=np.int32)
    for b in range(B):
        node, kept = int(rng.integers(1, tree.M)), []
        while node > 0:
            kept.append(node)
            node = int(parent[node])
        kept = kept[::-1] if b != 1 else kept[::-1] + [-1]
        accept[b] = len([r for r in kept if r >= 0])
        path[b, :accept[b]] = kept[:accept[b]]
    if B == 5:
        accept[4], table[0, 0] = -1, -7              # a walk that gave up keeps the root; a position without a page
    cache = lpp.PagedCache(code, Hkv, Dh, size, x["kp"].shape[0])
    d = {n: v.to(DEV) for n, v in x.items()}
    new_len = torch.full((B,), -7, dtype=torch.int32, device=DEV)
    lpp.lpp_paged_commit_kv(cache, tree, d["kn"], d["vn"], dev(path), dev(accept), dev(table), dev(seq), B, d["kp"], d["vp"], new_len)
    rows = [[0] + path[b, :max(accept[b], 0)].tolist() for b in range(B)]
    _compare(x, table, rows, seq, (d["kp"], d["vp"]), new_len)


@pytest.mark.parametrize("dtype,Dh,Hkv,size,M,per", [("bf16", 64, 3, 16, 1, 4), ("bf16", 64, 2, 16, 130, 10), ("bf16", 128, 8, 64, 200, 4),
                                                     ("f32", 64, 2, 32, 67, 5), ("f32", 128, 1, 128, 33, 2)])
def test_append(dtype, Dh, Hkv, size, M, per):
    rng = np.random.default_rng(M)
    B = 5
    code, tt = (lpp.LPP_BF16, torch.bfloat16) if dtype == "bf16" else (lpp.LPP_F32, torch.float32)
    x, table = _case(rng, B, Hkv, M, Dh, size, per, tt)
    cap = per * size
    seq = np.array([0, size - 1, cap - M // 2 - 1, cap, cap + 9], dtype=np.int32)
    row_len = np.array([M, M // 2 + 1, M, M, M], dtype=np.int32)
    table[1, per - 1] = x["kp"].shape[0]
    cache = lpp.PagedCache(code, Hkv, Dh, size, x["kp"].shape[0])
    for given in (row_len, np.array([0, M + 3, -2, 1, M], dtype=np.int32), None):
        d = {n: v.to(DEV) for n, v in x.items()}
        new_len = torch.full((B,), -7, dtype=torch.int32, device=DEV)
        lpp.lpp_paged_append_kv(cache, d["kn"], d["vn"], None if given is None else dev(given), dev(table), dev(seq), B, M, d["kp"],
                                d["vp"], new_len)
        n = [M] * B if given is None else np.clip(given, 0, M).tolist()
        _compare(x, table, [range(r) for r in n], seq, (d["kp"], d["vp"]), new_len)


def test_a_root_alone_and_a_pool_of_other_rows():
    """A tree without drafted nodes; the pages of the items are parts of a pool whose other pages stay as they were."""
    rng = np.random.default_rng(9)
    tree = lpp.Tree([-1])
    x, table = _case(rng, 3, 4, 1, 64, 16, 2, torch.bfloat16)
    seq = np.array([0, 15, 31], dtype=np.int32)
    cache = lpp.PagedCache(lpp.LPP_BF16, 4, 64, 16, x["kp"].shape[0])
    d = {n: v.to(DEV) for n, v in x.items()}
    new_len = torch.full((3,), -7, dtype=torch.int32, device=DEV)
    junk = torch.full((3,), 1 << 30, dtype=torch.int32, device=DEV)
    lpp.lpp_paged_commit_kv(cache, tree, d["kn"], d["vn"], junk[:0].view(3, 0), dev(np.zeros(3, dtype=np.int32)), dev(table), dev(seq),
                            3, d["kp"], d["vp"], new_len)
    _compare(x, table, [[0]] * 3, seq, (d["kp"], d["vp"]), new_len)
