"""GPU: attention of new tokens over a paged cache against the oracle.

Tolerances.  A = sum of weights times |values|, what a relative error of the weights is multiplied by.
bf16: every weight is rounded by at most 2^-8, numerator and sum alike (2 * 2^-8 of A, 2% for second order), float32 scores of
magnitudes up to 30 move weights by less than 2^-10, and the output is rounded by at most 2^-8 of itself.  Root mean squares: a
rounding's is at most 2^-8 / sqrt(3); the output's and the weights' together stay below 2^-8.
float32: a score is a chain of Dh / 4 sums of four products and some additions (Dh / 4 + 8 roundings of its magnitude, the
reference's likewise), sums run over a wave's tiles, waves and ranges (n / 8 + 100 roundings of A).  Root mean square below 2^-17."""
import numpy as np
import pytest
import torch

import paper_2502_06352_amd as lpp
from oracle import gather_pages, paged_attention
from workloads import bf16_round, static_tree
from gpu_common import DEV, dev

pytestmark = pytest.mark.gpu

WIDE = static_tree((8, 4, 2, 2, 1, 1, 1, 1), 128)
XXL = static_tree((6, 3, 2, 2, 1, 1), 60)
TINY = static_tree((4, 2, 1, 1), 15)


class Case:
    """Inputs on the host; what no row sees holds NaN: slots behind the lengths, pages of nobody, rows behind the last."""

    def __init__(self, B, H, Hkv, Dh, page, lens, M=0, parent=None, rows=None, S=None, dtype="bf16", size=1.0, seed=0):
        rng = np.random.default_rng(seed)
        self.__dict__.update(B=B, H=H, Hkv=Hkv, Dh=Dh, page=page, parent=parent, dtype=dtype)
        self.M = M = len(parent) if parent is not None else M
        self.lens, self.rows = np.asarray(lens, dtype=np.int32), None if rows is None else np.asarray(rows, dtype=np.int32)
        self.S = max(lens) if S is None else S
        stride = max(-(-self.S // page), 1) + 1
        self.n_pages = B * stride + 2

        def normal(*shape):
            x = rng.standard_normal(shape, dtype=np.float32)
            return bf16_round(x) if dtype == "bf16" else x

        self.q, self.kn, self.vn = normal(B, H, M, Dh) * np.float32(size), normal(B, Hkv, M, Dh), normal(B, Hkv, M, Dh)
        self.kp, self.vp = normal(self.n_pages, Hkv, page, Dh), normal(self.n_pages, Hkv, page, Dh)
        self.table = rng.permutation(self.n_pages)[:B * stride].reshape(B, stride).astype(np.int32)
        used = np.zeros((self.n_pages, page), dtype=bool)
        for b in range(B):
            n = min(max(int(self.lens[b]), 0), self.S)
            at = np.arange(n)
            used[self.table[b, at // page], at % page] = True
            self.table[b, -(-n // page):] = [1 << 30, -5][b % 2]
            if rows is not None:
                self.kn[b, :, max(rows[b], 0):], self.vn[b, :, max(rows[b], 0):] = np.nan, np.nan
        for x in (self.kp, self.vp):
            x.transpose(0, 2, 1, 3)[~used] = np.nan

    def upload(self):
        tt = torch.bfloat16 if self.dtype == "bf16" else torch.float32
        t = {n: dev(getattr(self, n)).to(tt) for n in ("q", "kn", "vn", "kp", "vp")}
        t.update(table=dev(self.table), lens=dev(self.lens), rows=None if self.rows is None else dev(self.rows))
        t["cache"] = lpp.PagedCache(lpp.LPP_BF16 if self.dtype == "bf16" else lpp.LPP_F32, self.Hkv, self.Dh, self.page, self.n_pages)
        t["tree"] = None if self.parent is None else lpp.Tree(self.parent)
        t["out"] = torch.full((self.B, self.H, self.M, self.Dh), 7.0, dtype=tt, device=DEV)
        ws = lpp.lpp_paged_attention_workspace(t["cache"], self.B, self.H, self.M, self.S)
        t["ws"] = torch.full((ws,), 255, dtype=torch.uint8, device=DEV)          # (NaN in any type)
        return t

    def call(self, t, stream=None, scale=0.0):
        seq = t["lens"]
        if t["tree"] is not None:
            lpp.lpp_paged_tree_attention(t["cache"], t["tree"], t["q"], t["kp"], t["vp"], t["table"], t["kn"], t["vn"], seq, self.B, self.H,
                                         self.S, scale, t["out"], t["ws"], stream)
        else:
            lpp.lpp_paged_chunk_attention(t["cache"], t["q"], t["kp"], t["vp"], t["table"], t["kn"], t["vn"], seq, t["rows"], self.B,
                                          self.H, self.M, self.S, scale, t["out"], t["ws"], stream)
        return t["out"]

    def check(self, out, scale=None):
        got = out.float().cpu().numpy()
        lens = np.clip(self.lens, 0, self.S)
        rows = None if self.rows is None else np.clip(self.rows, 0, self.M)
        args = (self.table, self.kn)
        want = paged_attention(self.q, self.kp, self.vp, *args, self.vn, lens, self.parent, rows, scale)
        A = paged_attention(self.q, self.kp, np.abs(self.vp), *args, np.abs(self.vn), lens, self.parent, rows, scale)
        for b in range(self.B):
            n = self.M if rows is None else rows[b]
            assert np.all(got[b, :, n:] == 7.0), "rows behind the last were written"
            g, w, a = got[b, :, :n], want[b, :, :n], A[b, :, :n]
            odd = ~np.isfinite(w)
            assert np.array_equal(np.isfinite(g), ~odd)
            if not n or odd.all():
                continue
            if self.dtype == "bf16":
                tol = (1.02 * 2.0 ** -7 + 2.0 ** -10) * a
                tol, rms = tol + 2.0 ** -8 * (np.abs(w) + tol), 2.0 ** -8
            else:
                # magnitude of a score: sum of |q| |k| by the norms
                K = np.concatenate([gather_pages(self.kp, self.table, b, int(lens[b])), self.kn[b, :, :n]], axis=1)
                top = np.linalg.norm(self.q[b, :, :n], axis=-1).max() * np.nanmax(np.linalg.norm(K, axis=-1)) * (scale or self.Dh ** -0.5)
                tol, rms = a * (2 * (self.Dh / 4 + 8) * top + (lens[b] + n) / 8 + 100) * 2.0 ** -24, 2.0 ** -17
            err, tol, norm = np.abs(g[~odd] - w[~odd]), tol[~odd], np.linalg.norm(w[~odd])
            assert np.all(err <= tol), f"item {b}: {np.max(err / tol)} of the tolerance"
            assert np.linalg.norm(err) <= rms * max(norm, np.linalg.norm(a[~odd]) * 0.5), f"item {b}: {np.linalg.norm(err) / norm}"

    def run(self):
        t = self.upload()
        print(self.dtype, self.B, self.H, self.Hkv, self.Dh, self.page, self.S, self.M, flush=True)
        self.check(self.call(t))
        return t


TREES = [
    # one token: alone, with an empty cache, over page and tile ends, with shared heads
    dict(B=1, H=1, Hkv=1, Dh=64, page=16, lens=[0], parent=[-1]),
    dict(B=3, H=8, Hkv=2, Dh=128, page=16, lens=[1, 17, 0], parent=[-1]),
    dict(B=2, H=32, Hkv=8, Dh=128, page=64, lens=[700, 31], parent=[-1]),
    dict(B=2, H=24, Hkv=1, Dh=64, page=256, lens=[257, 512], parent=[-1]),
    dict(B=1, H=40, Hkv=1, Dh=64, page=32, lens=[65], parent=[-1]),
    # trees: one tile of rows, two, four, and more blocks; rows past a mask word
    dict(B=2, H=4, Hkv=4, Dh=64, page=16, lens=[256, 33], parent=TINY),
    dict(B=1, H=4, Hkv=2, Dh=128, page=32, lens=[127], parent=TINY),
    dict(B=2, H=3, Hkv=3, Dh=64, page=64, lens=[64, 0], parent=XXL),
    dict(B=1, H=2, Hkv=2, Dh=128, page=16, lens=[333], parent=XXL),
    dict(B=2, H=6, Hkv=2, Dh=64, page=128, lens=[500, 129], parent=WIDE),
    dict(B=1, H=3, Hkv=1, Dh=128, page=64, lens=[200], parent=WIDE),
    dict(B=1, H=2, Hkv=1, Dh=64, page=16, lens=[40], parent=np.arange(-1, 255)),
    dict(B=9, H=2, Hkv=1, Dh=64, page=16, lens=[5, 0, 16, 31, 32, 33, 64, 100, 1], parent=TINY),
    # a bound above the lengths, and lengths out of range
    dict(B=3, H=4, Hkv=2, Dh=64, page=32, lens=[90, -4, 500], S=300, parent=TINY),
]
CHUNKS = [
    dict(B=1, H=1, Hkv=1, Dh=64, page=16, lens=[0], M=1, rows=[1]),
    dict(B=3, H=4, Hkv=1, Dh=64, page=16, lens=[100, 0, 47], M=5, rows=[5, 1, 0]),
    dict(B=4, H=4, Hkv=4, Dh=64, page=16, lens=[256, 85, 16, 3], M=37, rows=[37, 12, -2, 99]),
    dict(B=2, H=8, Hkv=2, Dh=128, page=32, lens=[300, 64], M=64, rows=[64, 33]),
    dict(B=2, H=2, Hkv=1, Dh=128, page=64, lens=[0, 190], M=200, rows=[200, 129]),
    dict(B=1, H=3, Hkv=1, Dh=64, page=256, lens=[70], M=321, rows=None),
    dict(B=2, H=2, Hkv=2, Dh=64, page=32, lens=[0, 0], S=0, M=130, rows=[130, 65]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("i", range(len(TREES)))
def test_trees(i, dtype):
    Case(dtype=dtype, seed=i, **TREES[i]).run()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("i", range(len(CHUNKS)))
def test_chunks(i, dtype):
    Case(dtype=dtype, seed=i, **CHUNKS[i]).run()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("parent,M", [(TINY, 0), (XXL, 0), (None, 140)])
def test_large_scores_and_a_scale(parent, M, dtype):
    """Scores of spread 8, so that references move; and a scale of the caller's."""
    c = Case(2, 4, 2, 64, 16, [400, 130], M=M, parent=parent, rows=None if parent is not None else [140, 77], dtype=dtype, size=8.0, seed=3)
    t = c.upload()
    c.check(c.call(t, scale=0.11), scale=0.11)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("parent,M,rows,H", [(TINY, 0, None, 2), (XXL, 0, None, 4), (WIDE, 0, None, 2), (None, 150, [150, 40], 2)])
def test_what_a_row_does_not_see_plays_no_part(parent, M, rows, H, dtype):
    """Infinities and NaN among the new keys and values: rows that see them get them, the others nothing."""
    c = Case(2, H, 2, 64, 16, [70, 0], M=M, parent=parent, rows=rows, dtype=dtype, seed=4)
    c.vn[0, 0, 5, 3], c.vn[0, 1, 2, 60], c.vn[1, 0, 9, :], c.vn[1, 1, 1, 7] = np.inf, np.nan, -np.inf, np.inf
    c.kn[1, 1, 11], c.kn[0, 0, 14, 2] = np.nan, np.nan
    c.run()


def test_an_infinity_in_the_cache_is_seen_by_all():
    c = Case(1, 2, 2, 64, 16, [50], parent=TINY, seed=5)
    c.vp[c.table[0, 1], 0, 3, 9] = np.inf
    c.run()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_beyond_four_gigabytes(dtype):
    """The items' pages lie at the end of a pool of more than 2^32 bytes (and of more than 2^31 elements in bf16)."""
    c = Case(2, 8, 8, 128, 256, [300, 513], parent=TINY, dtype=dtype, seed=6)
    t = c.upload()
    each = 8 * 256 * 128
    n = (5 << 30) // (each * t["kp"].element_size())
    far = n - c.n_pages
    for name in ("kp", "vp"):
        pool = torch.empty((n, 8, 256, 128), dtype=t[name].dtype, device=DEV)
        pool[far:] = t[name]
        t[name] = pool
    c_table = np.where((c.table >= 0) & (c.table < c.n_pages), c.table + far, c.table)
    t["table"], t["cache"] = dev(c_table), lpp.PagedCache(t["cache"].dtype, 8, 128, 256, n)
    c.check(c.call(t))


def test_two_runs_give_the_same_bits_and_leave_the_handle_clean():
    """Key ranges joined by the block that finishes last; other sizes on the same handle and workspace in between."""
    c = Case(1, 8, 2, 128, 16, [3000], parent=TINY, seed=7)
    t = c.upload()
    assert t["ws"].numel() > 256
    first = c.call(t).clone()
    d = Case(1, 8, 2, 128, 16, [90], M=70, rows=[70], seed=8)
    u = d.upload()
    u["cache"] = t["cache"]
    u["kp"], u["vp"] = (torch.cat([x, x.new_zeros(c.n_pages - d.n_pages, 2, 16, 128)]) for x in (u["kp"], u["vp"]))
    for _ in range(3):
        u["out"].fill_(7.0)
        d.check(d.call(u))
        t["ws"].fill_(127)
        t["out"].fill_(7.0)
        assert torch.equal(c.call(t), first)
    c.check(first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(B=1, H=2, Hkv=1, Dh=128, page=64, lens=[9000], parent=XXL),
                                dict(B=2, H=4, Hkv=2, Dh=64, page=16, lens=[7000, 300], M=33, rows=[33, 20]),
                                dict(B=3, H=1, Hkv=1, Dh=64, page=256, lens=[20000, 5, 9999], parent=[-1])])
def test_many_ranges(kw, dtype):
    """Long caches of few heads: ranges added up by the last block or in a launch of their own, items of one range beside others."""
    t = Case(dtype=dtype, seed=10, **kw).run()
    assert t["ws"].numel() > 256


def test_a_short_workspace_is_refused():
    c = Case(1, 8, 2, 128, 16, [3000], parent=TINY)
    t = c.upload()
    assert t["ws"].numel() > 256                                    # (the keys are cut in ranges here)
    for ws in (t["ws"][:-256], None):
        t["ws"] = ws
        with pytest.raises(lpp.LppError) as e:
            c.call(t)
        assert e.value.status == lpp.LPP_ENOWORKSPACE


@pytest.mark.parametrize("kw", [dict(parent=XXL), dict(M=100, rows=[100, 31])])
def test_captured_on_a_side_stream(kw):
    c = Case(2, 8, 2, 64, 32, [450, 77], seed=9, **kw)
    t = c.upload()
    eager = c.call(t).clone()
    other = {n: t[n].clone() for n in ("q", "lens")}
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            c.call(t, side)
    for _ in range(3):
        t["out"].fill_(7.0)
        t["q"].neg_()
        t["lens"].fill_(20)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert not torch.equal(t["out"], eager)
        t["q"].copy_(other["q"])
        t["lens"].copy_(other["lens"])
        t["out"].fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(t["out"], eager)
    c.check(eager)


def _lens(B, most, seed):
    lens = np.random.default_rng(seed).integers(0, most + 1, B)
    lens[seed % B], lens[(seed + 1) % B] = most, 0
    return lens.tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [
    dict(B=64, H=2, Hkv=1, Dh=64, page=16, lens=_lens(64, 3000, 20), parent=[-1]),
    dict(B=65, H=1, Hkv=1, Dh=64, page=16, lens=_lens(65, 3000, 21), parent=[-1]),
    dict(B=7, H=8, Hkv=1, Dh=128, page=32, lens=_lens(7, 6000, 22), M=12, rows=[12, 0, 1, 12, 7, -3, 40]),
    dict(B=5, H=2, Hkv=2, Dh=64, page=64, lens=[0] * 5, S=6000, parent=XXL),
    dict(B=6, H=2, Hkv=1, Dh=64, page=64, lens=[0, 1, 0, 9000, 0, 0], parent=TINY),
    dict(B=3, H=3, Hkv=1, Dh=128, page=128, lens=[50, 14000, 700], M=40, rows=[40, 40, 40]),
])
def test_ranges_cut_by_the_items_lengths(kw, dtype):
    """Items in any order of their lengths, empty ones among them, bounds far above all lengths; batches of 64 and more."""
    t = Case(dtype=dtype, seed=30, **kw).run()
    assert t["ws"].numel() > 256


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [
    dict(B=64, H=8, Hkv=8, Dh=64, page=16, lens=_lens(64, 90, 23), parent=[-1]),
    dict(B=40, H=8, Hkv=8, Dh=64, page=32, lens=_lens(40, 130, 24), parent=TINY),
    dict(B=12, H=24, Hkv=8, Dh=128, page=16, lens=_lens(12, 100, 25), M=24, rows=[24, 1, 0, 24, 13, 2, -1, 30, 24, 24, 5, 8]),
    dict(B=70, H=4, Hkv=4, Dh=64, page=16, lens=_lens(70, 60, 26), parent=[-1]),
])
def test_more_items_than_fit_at_once(kw, dtype):
    """More blocks than compute units, of items in any order of their lengths."""
    Case(dtype=dtype, seed=31, **kw).run()


def test_other_lengths_between_two_runs():
    """The ranges of one call leave nothing behind for the next, whatever its lengths."""
    c = Case(4, 4, 1, 128, 16, [6000, 100, 3000, 0], parent=TINY, seed=32)
    t = c.upload()
    assert t["ws"].numel() > 256
    first = c.call(t).clone()
    c.check(first)
    for lens in ([0, 0, 0, 0], [1, 100, 2000, 0], [6000, 0, 0, 0], [5999, 90, 2999, 0]):
        t["lens"].copy_(dev(np.asarray(lens, dtype=np.int32)))
        c.call(t)
        t["lens"].copy_(dev(c.lens))
        assert torch.equal(c.call(t), first)


def test_tensors_of_the_host_are_refused():
    """Nothing is enqueued with an address that the kernels cannot read."""
    c = Case(2, 4, 2, 64, 16, [40, 3], parent=TINY, seed=33)
    for name in ("ws", "q", "kn", "table", "lens", "out", "kp"):
        t = c.upload()
        t[name] = t[name].cpu()
        with pytest.raises(lpp.LppError) as e:
            c.call(t)
        assert e.value.status == lpp.LPP_EINVAL
    c.run()


def test_two_graphs_share_a_handle_and_a_workspace():
    """Captured one after the other, replayed in turn on one stream, with eager calls on the same handle in between."""
    cases = [Case(3, 8, 2, 128, 16, [3000, 40, 1700], parent=TINY, seed=34), Case(2, 8, 2, 128, 16, [90, 5000], M=70, rows=[70, 31], seed=35)]
    n_pages, states = max(c.n_pages for c in cases), [c.upload() for c in cases]
    ws = torch.full((max(t["ws"].numel() for t in states),), 255, dtype=torch.uint8, device=DEV)
    cache = lpp.PagedCache(lpp.LPP_BF16, 2, 128, 16, n_pages)
    for c, t in zip(cases, states):
        assert t["ws"].numel() > 256
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
    for which in (0, 1, 1, 0, 1, 0):
        states[which]["out"].fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[which].replay()
            other = states[1 - which]
            other["out"].fill_(7.0)
            cases[1 - which].call(other, side)
        side.synchronize()
        assert torch.equal(states[which]["out"], eager[which]) and torch.equal(other["out"], eager[1 - which])


def test_two_streams_with_a_handle_each():
    """Calls that may overlap: what they leave in their handles and workspaces is their own."""
    cases = [Case(2, 8, 2, 128, 16, [4000, 2500], parent=TINY, seed=s) for s in (36, 37)]
    states, streams = [c.upload() for c in cases], [torch.cuda.Stream(), torch.cuda.Stream()]
    want = [c.call(t).clone() for c, t in zip(cases, states)]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, t, s in zip(cases, states, streams):
            c.call(t, s)
    torch.cuda.synchronize()
    for c, t, w in zip(cases, states, want):
        assert torch.equal(t["out"], w)
        c.check(w)
