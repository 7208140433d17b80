"""GPU: adjusted logits and token counts against the oracle.

Tolerance: guidance rounds three times (difference, product, sum), the penalties four (quotient or product, frequency times n,
two differences), the bias once: 8 * 2^-24 of the sum of the magnitudes that go into a value."""
import math

import numpy as np
import pytest
import torch

import paper_2502_06352_amd as lpp
from oracle import adjust_logits
from workloads import static_tree
from gpu_common import DEV, dev

pytestmark = pytest.mark.gpu


def _bits(mask):
    """bool [..., V] -> int32 words [..., ceil(V/32)]; bits behind V are set at random places."""
    V = mask.shape[-1]
    words = -(-V // 32)
    full = np.zeros(mask.shape[:-1] + (words * 32,), dtype=np.uint8)
    full[..., :V] = mask
    full[..., V:] = 1
    return np.packbits(full, axis=-1, bitorder="little").view(np.int32)


def _run(parent, B, V, off=0, pad=0, dtype="f32", guided=False, path=True, counts=True, penalties=True, bias=1, mask=3, seed=0, cond=None,
         in_place=False, few=False):
    rng = np.random.default_rng(seed)
    tree = lpp.Tree(parent)
    M, ldv = tree.M, V + off + pad
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def rows():
        x = np.full((B, M, ldv), 55.0, dtype=np.float32)            # columns outside: not -inf, so that a read shows
        x[..., off:off + V] = rng.standard_normal((B, M, V)) * 3
        return torch.from_numpy(x).to(tt)

    c, u = rows(), rows() if guided else None
    if cond is not None:
        c[..., off:off + V] = torch.from_numpy(cond).to(tt)
    kw, dv = {}, {}
    if path:
        kw["tokens"] = rng.integers(0, min(V, 5) if few else V, (B, M)).astype(np.int32)
        kw["tokens"][:, -1] = V + 3                                # clamped, as in verification
    if counts:
        kw["counts"] = (rng.random((B, V)) < 0.3) * rng.integers(1, 300, (B, V)).astype(np.int32)
    if penalties:
        kw.update(repetition=(0.7 + rng.random(B)).astype(np.float32), frequency=rng.random(B).astype(np.float32),
                  presence=(rng.random(B) - 0.5).astype(np.float32))
    if bias:
        kw["bias"] = rng.standard_normal((B, V)[2 - bias:], dtype=np.float32)
    dv = {n: dev(v.astype(np.int32) if n in ("tokens", "counts") else v) for n, v in kw.items()}
    allowed = None
    if mask:
        shape = {1: (V,), 2: (B, V), 3: (B, M, V)}[mask]
        allowed = rng.random(shape) < 0.5
        if mask == 3:
            allowed[0, 0] = False                                  # a row that allows nothing
        dv["mask"] = dev(_bits(allowed))
        allowed = allowed[:, None] if mask == 2 else allowed
    d_c, d_u = c.to(DEV), None if u is None else u.to(DEV)
    out = d_c if in_place else torch.full((B, M, ldv), 99.0, device=DEV)
    lpp.lpp_adjust_logits(tree, lpp.LPP_BF16 if dtype == "bf16" else lpp.LPP_F32, d_c, ldv, off, V, B, out, uncond_logits=d_u,
                          cfg_scale=2.5 if guided else 0.0, **dv)
    y = out.cpu().numpy()
    want, size = adjust_logits(parent, c.float().numpy()[..., off:off + V], None if u is None else u.float().numpy()[..., off:off + V], 2.5,
                               mask=allowed, **kw)
    got = y[..., off:off + V]
    with np.errstate(over="ignore"):                                # (beyond float32's largest number: an infinity)
        rounded = want.astype(np.float32)
    odd = ~np.isfinite(rounded)
    assert np.array_equal(got[odd], rounded[odd], equal_nan=True)
    assert np.all(np.abs(got[~odd] - want[~odd]) <= 8 * 2.0 ** -24 * size[~odd])
    left = 55.0 if in_place else 99.0
    assert np.all(y[..., :off] == left) and np.all(y[..., off + V:] == left)      # columns outside: as they were


SMALL = static_tree((4, 2, 1, 1), 15)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,off,pad", [(1, 0, 0), (3, 1, 0), (31, 0, 2), (64, 4, 0), (4095, 7, 1), (4097, 0, 0), (16384, 0, 0), (8192, 4, 500)])
def test_sizes_and_offsets(V, off, pad, dtype):
    _run(SMALL, 2, V, off, pad, dtype)
    _run(SMALL, 1, V, off, pad, dtype, guided=True)


@pytest.mark.parametrize("kw", [dict(path=False), dict(counts=False), dict(penalties=False), dict(bias=0), dict(bias=2), dict(mask=0), dict(mask=1),
                                dict(mask=2), dict(few=True), dict(in_place=True), dict(in_place=True, guided=True, few=True),
                                dict(path=False, counts=False, penalties=False, bias=0, mask=0)])
def test_each_part_alone(kw):
    _run(SMALL, 3, 1000, 3, 2, seed=1, **kw)


def test_a_chain_of_one_token_and_the_root_alone():
    _run(np.arange(-1, 255), 1, 300, seed=2, few=True)              # up to 255 tokens on a path, most of them the same few
    _run(np.array([-1]), 2, 5000, seed=3)


def test_infinities_and_nan():
    cond = np.random.default_rng(4).standard_normal((2, 16, 200)).astype(np.float32)
    cond[:, :, ::7], cond[:, :, 1::7], cond[:, :, 2::7] = -math.inf, math.inf, math.nan
    cond[:, :, 3::7] = np.finfo(np.float32).min
    _run(SMALL, 2, 200, cond=cond)
    _run(SMALL, 2, 200, cond=cond, guided=True, mask=2, seed=5)


@pytest.mark.parametrize("B,T,V", [(1, 1, 1), (3, 0, 50), (4, 5000, 1000), (2, 700, 16384), (2, 3000, 40000), (5, 64, 32768)])
def test_token_counts(B, T, V):
    rng = np.random.default_rng(T)
    tokens = rng.integers(-2, V + 2, (B, T)).astype(np.int32)
    length = rng.integers(-1, T + 3, B).astype(np.int32)
    for given in (None, length):
        out = torch.full((B, V), -9, dtype=torch.int32, device=DEV)
        lpp.lpp_token_counts(dev(tokens), None if given is None else dev(given), B, V, out)
        for b, got in enumerate(out.cpu().numpy()):
            t = tokens[b, :T if given is None else min(max(given[b], 0), T)]
            assert np.array_equal(got, np.bincount(t[(t >= 0) & (t < V)], minlength=V))


def test_commit_counts():
    rng = np.random.default_rng(6)
    parent = np.arange(-1, 99)                                      # paths longer than a wave
    tree, B, V = lpp.Tree(parent), 4, 30
    tokens = rng.integers(0, V, (B, 100)).astype(np.int32)
    tokens[2, 5] = V + 50                                           # clamped
    path = np.tile(np.arange(1, 100, dtype=np.int32), (B, 1))
    accept, final = np.array([99, 0, 70, -1], dtype=np.int32), np.array([3, 4, 5, -1], dtype=np.int32)
    start = rng.integers(0, 9, (B, V)).astype(np.int32)
    counts = dev(start)
    lpp.lpp_commit_counts(tree, dev(tokens), dev(path), dev(accept), dev(final), B, V, counts)
    want = start.copy()
    for b in range(3):
        for x in tokens[b, 1:1 + accept[b]].clip(0, V - 1).tolist() + [int(final[b])]:
            want[b, x] += 1
    assert np.array_equal(counts.cpu().numpy(), want)


WIDE = static_tree((8, 4, 2, 2, 1, 1, 1, 1), 128)


@pytest.mark.parametrize("kw", [dict(), dict(guided=True), dict(dtype="bf16"), dict(dtype="bf16", guided=True, bias=2, mask=2),
                                dict(in_place=True, guided=True, few=True)])
def test_many_rows(kw):
    """4 x 129 rows in pieces of 2048 tokens, the last of one token: blocks of two groups of four tokens a lane, which are taken where
    they are four a compute unit (here 1548 blocks)."""
    assert 4 * 129 * 3 >= 4 * torch.cuda.get_device_properties(0).multi_processor_count
    _run(WIDE, 4, 4097, 5, 3, seed=7, **kw)


def test_tokens_far_outside_count_nowhere():
    tokens = np.array([[-2 ** 31, 2 ** 31 - 1, 39999, 32768, -1, 40000, 32767, -2 ** 31 + 5, 39999]], dtype=np.int32)
    out = torch.full((1, 40000), -9, dtype=torch.int32, device=DEV)
    lpp.lpp_token_counts(dev(tokens), None, 1, 40000, out)
    got = out.cpu().numpy()[0]
    assert got.sum() == 4 and got[39999] == 2 and got[32768] == 1 and got[32767] == 1


def test_penalties_that_go_by_different_counts():
    """Repetition by prompt and output, then frequency and presence by the output alone: two calls, the second in place."""
    rng = np.random.default_rng(8)
    tree, B, V = lpp.Tree(SMALL), 2, 700
    x = rng.standard_normal((B, tree.M, V), dtype=np.float32) * 3
    tokens = rng.integers(0, 9, (B, tree.M)).astype(np.int32)
    output = (rng.random((B, V)) < 0.2) * rng.integers(1, 5, (B, V))
    both = output + (rng.random((B, V)) < 0.3)
    rep, freq, pres = (np.array(v, dtype=np.float32) for v in ([1.3, 0.8], [0.25, 0.5], [-0.5, 1.0]))
    out = torch.empty(B, tree.M, V, device=DEV)
    lpp.lpp_adjust_logits(tree, lpp.LPP_F32, dev(x), V, 0, V, B, out, tokens=dev(tokens), counts=dev(both.astype(np.int32)), repetition=dev(rep))
    lpp.lpp_adjust_logits(tree, lpp.LPP_F32, out, V, 0, V, B, out, tokens=dev(tokens), counts=dev(output.astype(np.int32)), frequency=dev(freq),
                          presence=dev(pres))
    first, size = adjust_logits(SMALL, x, tokens=tokens, counts=both, repetition=rep)
    want, size = adjust_logits(SMALL, first, tokens=tokens, counts=output, frequency=freq, presence=pres)
    assert np.all(np.abs(out.cpu().numpy() - want) <= 8 * 2.0 ** -24 * size)
