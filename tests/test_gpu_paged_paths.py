"""GPU: paged attention on every path that a plan may take (tests/paged_paths.py), against the oracle.  Tolerances are those of
test_gpu_paged_attention."""
import numpy as np
import pytest
import torch

import paged_paths
from gpu_common import DEV
from test_gpu_paged_attention import TINY, WIDE, XXL, Case
import paper_2502_06352_amd as lpp

pytestmark = pytest.mark.gpu

PARENTS = {1: [-1], 16: TINY, 61: XXL, 129: WIDE}


def _case(path, seed):
    """Items of all lengths, the longest neither first nor last, ties, empty ones and ones without rows among them; where there are
    rows enough an infinity and a NaN among the new values, and a new key of NaN that its own row alone sees."""
    dtype, Dh, _, _, _, form, B, H, Hkv, M, S, page = path
    lens = np.random.default_rng(seed).integers(0, S + 1, B)
    lens[B // 2] = S
    if B > 2:
        lens[0], lens[-1] = 0, lens[1]
    if form == "tree":
        c = Case(B, H, Hkv, Dh, page, lens.tolist(), parent=PARENTS[M], S=S, dtype=dtype, seed=seed)
    else:
        rows = [(M, M - 1, M // 2 + 1, M + 5, 1, 0, -3)[(b - B // 2) % 7] for b in range(B)]
        c = Case(B, H, Hkv, Dh, page, lens.tolist(), M=M, rows=rows, S=S, dtype=dtype, seed=seed)
    if M > 4:
        b = B // 2                                         # (has all M rows)
        c.vn[b, 0, 2 * M // 3, 3], c.vn[b, Hkv - 1, M - 2, Dh - 1] = np.inf, np.nan
        c.kn[b, 0, M - 1, 5] = np.nan
    return c


def _bits(t):
    return t.view(torch.int16 if t.dtype is torch.bfloat16 else torch.int32)


@pytest.mark.parametrize("i", range(len(paged_paths.PATHS)))
def test_paths(i):
    """Three calls on one handle and workspace, the outputs filled anew: the oracle's result, and the same bits each time."""
    path = paged_paths.PATHS[i]
    print(path, flush=True)
    c = _case(path, seed=100 + i)
    t = c.upload()
    first = c.call(t).clone()
    c.check(first)
    for _ in range(2):
        t["out"].fill_(7.0)
        t["ws"].fill_(255)
        assert torch.equal(_bits(c.call(t)), _bits(first))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_calls_that_the_last_block_joins(dtype):
    """Two graphs on one handle and workspace, replayed in turn with eager calls in between."""
    cases = [Case(len(lens), 8, 2, 128, 16, lens, parent=[-1], dtype=dtype, seed=60 + i) for i, lens in enumerate(paged_paths.TOKENS)]
    n_pages, states = max(c.n_pages for c in cases), [c.upload() for c in cases]
    ws = torch.full((max(t["ws"].numel() for t in states),), 255, dtype=torch.uint8, device=DEV)
    cache = lpp.PagedCache(states[0]["cache"].dtype, 2, 128, 16, n_pages)
    for c, t in zip(cases, states):
        t["kp"], t["vp"] = (torch.cat([x, x.new_zeros(n_pages - c.n_pages, 2, 16, 128)]) for x in (t["kp"], t["vp"]))
        t.update(ws=ws, cache=cache)
    eager = [c.call(t).clone() for c, t in zip(cases, states)]
    for c, out in zip(cases, eager):
        c.check(out)
    side, graphs = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    for c, t in zip(cases, states):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.stream(side):
            with torch.cuda.graph(graphs[-1], stream=side):
                c.call(t, side)
    for which in (0, 1, 1, 0, 0):
        for t in states:
            t["out"].fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[which].replay()
            cases[1 - which].call(states[1 - which], side)
        side.synchronize()
        for t, want in zip(states, eager):
            assert torch.equal(t["out"], want)


@pytest.mark.parametrize("dtype,H,Hkv,Dh,largest,calls", [
    ("bf16", 32, 8, 128, (64, 1, 900), [(64, 900), (1, 900), (3, 700), (2, 0), (64, 31)]),
    ("f32", 16, 16, 64, (60, 16, 700), [(2, 600), (60, 700), (1, 699)])])
def test_one_workspace_for_calls_of_all_sizes(dtype, H, Hkv, Dh, largest, calls):
    """Made for the largest batch; smaller ones are cut into more ranges.  Nothing is written behind it."""
    B, M, S = largest
    parent = PARENTS[M]
    cache = lpp.PagedCache(lpp.LPP_BF16 if dtype == "bf16" else lpp.LPP_F32, Hkv, Dh, 32, 1)
    n = lpp.lpp_paged_attention_workspace(cache, B, H, M, S)
    whole = torch.full((n + 4096,), 165, dtype=torch.uint8, device=DEV)
    for i, (items, most) in enumerate(calls):
        lens = [most * (b + 1) // items for b in range(items)]
        c = Case(items, H, Hkv, Dh, 32, lens, parent=parent, dtype=dtype, seed=70 + i)
        t = c.upload()
        t["ws"] = whole[:n]
        c.check(c.call(t))
        assert bool((whole[n:] == 165).all())


def test_outputs_and_workspaces_over_inputs_are_refused():
    """Tensors that are parts of one buffer: what lies in an input, or out and the workspace in each other, is not enqueued."""
    c = Case(1, 8, 2, 128, 16, [3000], parent=TINY, seed=80)
    t = c.upload()
    want, n = c.call(t).clone(), t["out"].numel()

    def status(**kw):
        with pytest.raises(lpp.LppError) as e:
            c.call(dict(t, **kw))
        return e.value.status

    one = torch.zeros(2 * n, dtype=torch.bfloat16, device=DEV)
    one[:n] = t["q"].view(-1)
    q = one[:n].view(t["q"].shape)
    for at in (0, 8, n - 8):
        assert status(q=q, out=one[at:at + n].view(q.shape)) == lpp.LPP_EINVAL
    for name in ("kp", "vp"):
        assert status(out=t[name].view(-1)[64:64 + n].view(q.shape)) == lpp.LPP_EINVAL
    parts, pool = t["ws"].numel(), t["kp"].view(-1).view(torch.uint8)
    long = torch.cat([pool, torch.zeros(parts, dtype=torch.uint8, device=DEV)])
    kp = long[:pool.numel()].view(torch.bfloat16).view(t["kp"].shape)
    assert status(kp=kp, ws=long[256:256 + parts]) == lpp.LPP_EINVAL
    both = torch.zeros(parts + 2 * n, dtype=torch.uint8, device=DEV)
    assert status(ws=both[:parts], out=both[:2 * n].view(torch.bfloat16).view(q.shape)) == lpp.LPP_EINVAL
    out = both[parts:].view(torch.bfloat16).view(q.shape)
    assert torch.equal(c.call(dict(t, q=q, ws=both[:parts], out=out)), want)          # side by side
    assert torch.equal(c.call(dict(t, q=q, out=one[n:].view(q.shape))), want)


def test_rotary_outputs_over_inputs_are_refused():
    tree, rotary = lpp.Tree(TINY), lpp.Rotary(64)
    B, M, H, Hkv, Dh = 2, 16, 4, 2, 64
    qkv = torch.randn(B, M, H + 2 * Hkv, Dh, device=DEV)
    q, k, v = qkv.split([H, Hkv, Hkv], 2)
    outs = [torch.full((B, h, M, Dh), 7.0, device=DEV) for h in (H, Hkv, Hkv)]
    over = qkv.view(-1)[H * Dh:H * Dh + B * H * M * Dh].view(B, H, M, Dh)
    for bad in ((over, outs[1], outs[2]), (outs[0], outs[1], outs[1]), (outs[0], outs[0].view(-1)[:B * Hkv * M * Dh], outs[2])):
        with pytest.raises(lpp.LppError) as e:
            lpp.lpp_rotary_qkv(rotary, tree, lpp.LPP_F32, q, k, v, None, None, B, H, Hkv, M, Dh, *bad)
        assert e.value.status == lpp.LPP_EINVAL
    torch.cuda.synchronize()
    assert all(bool((o == 7.0).all()) for o in outs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("parent,rows,sign,big,scale", [(TINY, None, 1, 15, 0.5), (XXL, None, -1, 15, 0.5), (None, [140, 77], 1, 15, 0.5),
                                                       (TINY, None, -1, 50, 2.0 ** -71), (XXL, None, -1, 50, 2.0 ** -71),
                                                       (None, [140, 77], -1, 50, 2.0 ** -71), (XXL, None, 1, -40, 2.0 ** 109)])
def test_scores_of_nearly_ten_to_the_ninth(parent, rows, sign, big, scale, dtype):
    """One number of a head makes the score, so that products are exact and scores differ by millions or not at all: a row's
    result is the mean of the values whose score is the largest that it sees."""
    c = Case(2, 4, 2, 64, 16, [400, 130], M=140, parent=parent, rows=rows, dtype=dtype, seed=81)
    rng = np.random.default_rng(82)
    for x in (c.kp, c.kn):
        x[..., 1:][~np.isnan(x[..., 1:])] = 0.0
        steps = 1.0 + rng.integers(0, 100, x[..., 0].shape) / 128.0
        x[..., 0] = np.where(np.isnan(x[..., 0]), np.nan, sign * steps * 2.0 ** big)
    c.q[..., 1:], c.q[..., 0] = 0.0, 2.0 ** big
    t = c.upload()
    c.check(c.call(t, scale=scale), scale=scale)


@pytest.mark.parametrize("dtype,kw", [
    ("f32", dict(B=2, H=4, Hkv=2, Dh=128, page=32, lens=[900, 333], M=700, rows=[700, 413])),
    ("f32", dict(B=3, H=3, Hkv=3, Dh=64, page=64, lens=[500, 0, 77], M=520, rows=[129, 520, 300])),
    ("bf16", dict(B=2, H=4, Hkv=2, Dh=128, page=32, lens=[900, 333], M=700, rows=[700, 413])),
    ("bf16", dict(B=3, H=3, Hkv=3, Dh=64, page=64, lens=[500, 0, 77], M=520, rows=[129, 520, 300]))])
def test_long_chunks(dtype, kw):
    """Several blocks of rows, the last not whole, over keys of which most blocks see a part."""
    Case(dtype=dtype, seed=90, **kw).run()
