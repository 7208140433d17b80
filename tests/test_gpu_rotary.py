"""GPU: rotary positions against the oracle.

Tolerance, float32: an angle's fraction of a turn (at most 1/2) is rounded to float32 (2^-26 of a turn: 2 pi 2^-26 of an angle), cosine
and sine are within 4 units in the last place (4 * 2^-23), then the magnitude, a product and a fused product and sum are rounded
(3 * 2^-24): 13 * 2^-24 of m (|x1| + |x2|) in all.  bf16 adds half a step, 2^-8 of the value."""
import numpy as np
import pytest
import torch

import paper_2502_06352_amd as lpp
from oracle import rotary_angles, rotate
from workloads import static_tree, tree_depths
from gpu_common import DEV, dev

pytestmark = pytest.mark.gpu

SCALINGS = {"none": (lpp.LPP_ROTARY_NONE, {}), "linear": (lpp.LPP_ROTARY_LINEAR, dict(factor=4.0)),
            "ntk": (lpp.LPP_ROTARY_NTK, dict(factor=2.5)), "yarn": (lpp.LPP_ROTARY_YARN, dict(factor=8.0, original_len=4096))}


def _check(x, y, pos, theta, m, layout, half_step):
    """x [..., Dh] as handed in, y what came back, pos one position for each."""
    want = rotate(x, pos, theta, m, layout)
    n, size = len(theta), np.abs(x).astype(np.float64)
    first = np.arange(n) if layout == "half" else 2 * np.arange(n)
    second = first + n if layout == "half" else first + 1
    tol = np.zeros_like(size)
    tol[..., first] = tol[..., second] = 13 * 2.0 ** -24 * m * (size[..., first] + size[..., second])
    tol += half_step * (np.abs(want) + tol)
    tol[..., 2 * n:] = 0.0                              # copied
    assert np.all(np.abs(y - want) <= tol), np.max(np.abs(y - want) - tol)


def _run(B, M, H, Hkv, Dh, dim, layout, scaling, dtype, first, row_len=None, tree=None, base=0.0, parts="qkv", seed=0):
    rng = np.random.default_rng(seed)
    code, tt = (lpp.LPP_BF16, torch.bfloat16) if dtype == "bf16" else (lpp.LPP_F32, torch.float32)
    kind, extra = SCALINGS[scaling]
    rotary = lpp.Rotary(dim, layout=lpp.LPP_ROTARY_HALF if layout == "half" else lpp.LPP_ROTARY_INTERLEAVED, scaling=kind, base=base, **extra)
    qkv = torch.from_numpy(rng.standard_normal((B, M, H + 2 * Hkv, Dh), dtype=np.float32)).to(tt)
    ins = dict(zip("qkv", qkv.to(DEV).split([H, Hkv, Hkv], 2)))
    outs = {n: torch.full((B, h, M, Dh), 7.0, dtype=tt, device=DEV) for n, h in zip("qkv", (H, Hkv, Hkv))}
    lpp.lpp_rotary_qkv(rotary, tree, code, *[ins[n] if n in parts else None for n in "qkv"], None if first is None else dev(first),
                       None if row_len is None else dev(row_len), B, H, Hkv, M, Dh, *[outs[n] if n in parts else None for n in "qkv"])
    theta, m = rotary_angles(dim, base=base or 10000.0, scaling=scaling, **extra)
    step = np.arange(M) if tree is None else np.asarray(tree_depths(tree.parent))
    pos = (np.zeros(B, dtype=np.int64) if first is None else first)[:, None] + step[None]
    rows = np.full(B, M) if row_len is None else np.clip(row_len, 0, M)
    for n, x in zip("qkv", np.split(qkv.float().numpy(), [H, H + Hkv], axis=2)):
        y = outs[n].float().cpu().numpy()
        for b in range(B):
            assert np.all(y[b, :, rows[b]:] == 7.0)     # rows behind the last stay as they were
            if n not in parts:
                assert np.all(y[b] == 7.0)
                continue
            got, src = y[b, :, :rows[b]], x[b, :rows[b]].transpose(1, 0, 2)
            if n == "v":
                assert np.array_equal(got, src)
            else:
                _check(src, got, pos[b, :rows[b]][None], theta, m, layout, 2.0 ** -8 if dtype == "bf16" else 0.0)


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_chunks_far_and_ragged(scaling, layout, dtype):
    _run(3, 37, 6, 2, 128, 64, layout, scaling, dtype, np.array([0, 131000, 1 << 22], dtype=np.int32),
         np.array([37, 0, 11], dtype=np.int32))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("Dh,dim,M,H,Hkv", [(64, 64, 1, 1, 1), (64, 16, 300, 3, 3), (128, 128, 33, 32, 8), (80, 32, 20, 5, 1), (256, 256, 9, 4, 4),
                                            (16, 16, 257, 9, 3), (112, 96, 5, 2, 2)])
def test_heads_and_parts(Dh, dim, M, H, Hkv, layout):
    _run(2, M, H, Hkv, Dh, dim, layout, "none", "bf16", np.array([5, 70], dtype=np.int32))
    _run(2, M, H, Hkv, Dh, dim, layout, "none", "f32", None, base=500000.0)


@pytest.mark.parametrize("N,branching", [(15, (4, 2, 1, 1)), (128, (8, 4, 2, 2, 1, 1, 1, 1))])
def test_tree_rows_stand_at_their_depth(N, branching):
    tree = lpp.Tree(static_tree(branching, N))
    _run(3, N + 1, 4, 2, 64, 64, "half", "none", "f32", np.array([0, 1000, 77], dtype=np.int32), tree=tree)


def test_a_chain_of_the_most_rows():
    tree = lpp.Tree(np.arange(-1, 255))                 # depths up to 255, ancestors in four words
    _run(1, 256, 2, 1, 64, 32, "interleaved", "none", "f32", np.array([3], dtype=np.int32), tree=tree)


def test_positions_before_the_first_turn_backwards():
    _run(2, 4, 1, 1, 64, 64, "half", "none", "f32", np.array([-3, -1000], dtype=np.int32))


@pytest.mark.parametrize("parts", ["q", "k", "qk", "v"])
def test_parts_alone(parts):
    _run(2, 9, 5, 2, 64, 64, "half", "linear", "bf16", np.array([5, 9], dtype=np.int32), parts=parts)


def test_in_place_on_the_output_layout():
    rng = np.random.default_rng(4)
    B, H, M, Dh = 2, 3, 21, 128
    x = rng.standard_normal((B, H, M, Dh), dtype=np.float32)
    t = dev(x)
    rotary = lpp.Rotary(128)
    first = dev(np.array([40, 4], dtype=np.int32))
    lpp.lpp_rotary_qkv(rotary, None, lpp.LPP_F32, t.permute(0, 2, 1, 3), None, None, first, None, B, H, 1, M, Dh, t, None, None)
    theta, m = rotary_angles(128)
    y = t.cpu().numpy()
    for b, f in enumerate((40, 4)):
        _check(x[b], y[b], (f + np.arange(M))[None], theta, m, "half", 0.0)
