"""Host-only checks of the calls over a paged cache, of rotary positions and of adjusted logits: what they refuse, before
anything is enqueued (no kernel runs here)."""
import ctypes as C
import math
import os

import pytest
import torch

import paper_2502_06352_amd as lpp

FAKE = 0x1000          # 16-byte aligned; never dereferenced
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="valid arguments end in LPP_EHIP only without a device")


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lpp.LIB_PATH):
        from paper_2502_06352_amd.build import build_library
        build_library(verbose=False)
    return lpp.lib()


def _refusals(call, good, bad):
    """call(**good) with one argument after the other replaced: (changes, status)."""
    for change, status in bad:
        got = call(**dict(good, **change))
        assert got == status, f"{change}: {got}"


EINVAL, EUNSUP, EHIP = lpp.LPP_EINVAL, lpp.LPP_EUNSUPPORTED, lpp.LPP_EHIP


def test_paged_handle(L):
    def create(dtype=lpp.LPP_BF16, Hkv=8, Dh=128, page=64, n=10):
        h = C.c_void_p()
        st = L.lpp_paged_create(dtype, Hkv, Dh, page, n, C.byref(h))
        assert (st == lpp.LPP_OK) == bool(h.value)
        L.lpp_paged_destroy(h)
        return st

    assert create() == lpp.LPP_OK
    for page in (16, 32, 128, 256):
        assert create(page=page) == lpp.LPP_OK
    _refusals(create, {}, [(dict(dtype=2), EUNSUP), (dict(Hkv=0), EINVAL), (dict(Hkv=4097), EUNSUP), (dict(Dh=0), EINVAL),
                           (dict(Dh=96), EUNSUP), (dict(page=0), EINVAL), (dict(page=8), EUNSUP), (dict(page=48), EUNSUP),
                           (dict(page=512), EUNSUP), (dict(n=0), EINVAL)])
    assert L.lpp_paged_create(1, 8, 128, 64, 10, None) == EINVAL
    assert L.lpp_paged_destroy(None) == lpp.LPP_OK


@no_gpu
def test_paged_writes_refuse(L):
    cache, tree = lpp.PagedCache(lpp.LPP_BF16, 2, 64, 16, 4), lpp.Tree([-1, 0, 0])

    def commit(c=cache.handle, t=tree.handle, k=FAKE, v=FAKE, path=FAKE, acc=FAKE, table=FAKE, stride=3, seq=FAKE, B=2, kp=FAKE,
               vp=FAKE, new=None):
        return L.lpp_paged_commit_kv(c, t, k, v, path, acc, table, stride, seq, B, kp, vp, new, None)

    shared = [(dict(c=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(table=None), EINVAL),
              (dict(stride=0), EINVAL), (dict(seq=None), EINVAL), (dict(B=0), EINVAL), (dict(kp=None), EINVAL),
              (dict(vp=None), EINVAL), (dict(new=FAKE), EINVAL), (dict(k=FAKE + 8), EINVAL), (dict(vp=FAKE + 2), EINVAL),
              (dict(stride=1 << 28), EUNSUP), ({}, EHIP)]
    _refusals(commit, {}, shared + [(dict(t=None), EINVAL), (dict(path=None), EINVAL), (dict(acc=None), EINVAL)])

    def append(c=cache.handle, k=FAKE, v=FAKE, rows=None, table=FAKE, stride=3, seq=FAKE, B=2, M=5, kp=FAKE, vp=FAKE, new=None):
        return L.lpp_paged_append_kv(c, k, v, rows, table, stride, seq, B, M, kp, vp, new, None)

    for other in ("acc", "path", "table", "seq"):
        _refusals(commit, {}, [({other: 2 * FAKE}, EHIP), ({other: 2 * FAKE, "new": 2 * FAKE}, EINVAL)])
    for other in ("rows", "table", "seq"):
        _refusals(append, {}, [({other: 2 * FAKE}, EHIP), ({other: 2 * FAKE, "new": 2 * FAKE}, EINVAL)])
    _refusals(append, {}, shared + [(dict(M=0), EINVAL), (dict(M=0x7FFFFFFF), EUNSUP), (dict(rows=FAKE), EHIP)])


@no_gpu
def test_paged_attention_refuses(L):
    cache, tree = lpp.PagedCache(lpp.LPP_BF16, 2, 64, 16, 4), lpp.Tree([-1, 0, 0])

    def trees(c=cache.handle, t=tree.handle, q=FAKE, kp=FAKE, vp=FAKE, table=FAKE, stride=3, kn=FAKE, vn=FAKE, seq=None, B=2, H=4, S=40,
              scale=0.0, out=2 * FAKE, ws=FAKE, n=1 << 30):
        return L.lpp_paged_tree_attention(c, t, q, kp, vp, table, stride, kn, vn, seq, B, H, S, scale, out, ws, n, None)

    shared = [({}, EHIP), (dict(seq=FAKE), EHIP), (dict(c=None), EINVAL), (dict(q=None), EINVAL), (dict(kp=None), EINVAL), (dict(vp=None), EINVAL),
              (dict(table=None), EINVAL), (dict(stride=0), EINVAL), (dict(stride=2), EINVAL), (dict(kn=None), EINVAL), (dict(vn=None), EINVAL),
              (dict(B=0), EINVAL), (dict(H=0), EINVAL), (dict(H=3), EINVAL), (dict(S=-1), EINVAL), (dict(S=49), EINVAL),
              (dict(S=0, kp=None, vp=None, table=None, stride=0), EHIP), (dict(scale=-1.0), EINVAL), (dict(scale=math.nan), EINVAL),
              (dict(scale=math.inf), EINVAL), (dict(out=None), EINVAL), (dict(out=FAKE), EINVAL), (dict(q=FAKE + 4), EINVAL), (dict(out=FAKE + 8), EINVAL),
              (dict(kp=FAKE + 2), EINVAL), (dict(B=1 << 24), EUNSUP), (dict(S=1 << 30, stride=1 << 26), EUNSUP)]
    _refusals(trees, {}, shared + [(dict(t=None), EINVAL)])
    need = L.lpp_paged_attention_workspace(cache.handle, 1, 4, 3, 4000)
    assert need > 256
    for ws, n in ((None, need), (FAKE, need - 1), (FAKE + 4, need)):
        assert trees(B=1, S=4000, stride=250, ws=ws, n=n) == lpp.LPP_ENOWORKSPACE
    assert trees(B=1, S=4000, stride=250, n=need) == EHIP

    def chunks(c=cache.handle, q=FAKE, kp=FAKE, vp=FAKE, table=FAKE, stride=3, kn=FAKE, vn=FAKE, seq=None, rows=None, B=2, H=4, M=9, S=40,
               scale=0.0, out=2 * FAKE, ws=FAKE, n=1 << 30):
        return L.lpp_paged_chunk_attention(c, q, kp, vp, table, stride, kn, vn, seq, rows, B, H, M, S, scale, out, ws, n, None)

    _refusals(chunks, {}, shared + [(dict(rows=FAKE), EHIP), (dict(M=0), EINVAL), (dict(M=1 << 24), EUNSUP)])
    assert L.lpp_paged_attention_workspace(None, 1, 4, 3, 40) == 0
    for args in ((0, 4, 3, 40), (1, 3, 3, 40), (1, 4, 0, 40), (1, 4, 3, -1)):
        assert L.lpp_paged_attention_workspace(cache.handle, *args) == 0


def test_rotary_handle(L):
    def create(**kw):
        c = lpp.binding.RotaryConfig(**dict(dict(dim=64), **kw))
        h = C.c_void_p()
        st = L.lpp_rotary_create(C.byref(c), C.byref(h))
        assert (st == lpp.LPP_OK) == bool(h.value)
        L.lpp_rotary_destroy(h)
        return st

    yarn = dict(scaling=3, factor=4.0, original_len=4096)
    for good in ({}, dict(dim=16), dict(dim=256), dict(layout=1), dict(scaling=1, factor=1.0), dict(scaling=2, factor=8.0), yarn,
                 dict(base=500000.0), dict(magnitude=1.5)):
        assert create(**good) == lpp.LPP_OK, good
    _refusals(create, {}, [(dict(dim=0), EINVAL), (dict(dim=24), EUNSUP), (dict(dim=272), EUNSUP), (dict(layout=2), EINVAL),
                           (dict(scaling=4), EINVAL), (dict(scaling=-1), EINVAL), (dict(scaling=1), EINVAL),
                           (dict(scaling=1, factor=0.5), EINVAL), (dict(scaling=1, factor=math.nan), EINVAL),
                           (dict(base=1.0), EINVAL), (dict(base=math.inf), EINVAL), (dict(magnitude=-1.0), EINVAL),
                           (dict(magnitude=math.nan), EINVAL)])
    _refusals(create, yarn, [(dict(original_len=0), EINVAL), (dict(fast=1.0), EINVAL), (dict(slow=-1.0), EINVAL),
                             (dict(fast=math.inf), EINVAL)])
    assert L.lpp_rotary_create(None, C.byref(C.c_void_p())) == EINVAL
    assert L.lpp_rotary_destroy(None) == lpp.LPP_OK


def _rows(data=FAKE, item=640, row=128, head=64):
    return lpp.binding._pack_rows(data, item, row, head)


@no_gpu
def test_rotary_refuses(L):
    rotary, tree = lpp.Rotary(64), lpp.Tree([-1, 0, 0, 1, 1])

    def call(r=rotary.handle, t=tree.handle, dtype=lpp.LPP_BF16, q=_rows(), k=_rows(), v=_rows(), first=FAKE, rows=None, B=2, H=4,
             Hkv=2, M=5, Dh=64, qo=FAKE * 2, ko=FAKE * 3, vo=FAKE * 4):
        return L.lpp_rotary_qkv(r, t, dtype, q, k, v, first, rows, B, H, Hkv, M, Dh, qo, ko, vo, None)

    _refusals(call, {}, [({}, EHIP), (dict(r=None), EINVAL), (dict(q=None, k=None, v=None, qo=None, ko=None, vo=None), EINVAL),
                         (dict(q=None), EINVAL), (dict(vo=None), EINVAL), (dict(k=None, ko=None), EHIP), (dict(dtype=7), EUNSUP),
                         (dict(B=0), EINVAL), (dict(H=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(M=4), EINVAL), (dict(t=None, M=0), EINVAL),
                         (dict(Dh=48), EINVAL), (dict(Dh=72), EUNSUP), (dict(Dh=272), EUNSUP), (dict(q=_rows(data=0)), EINVAL),
                         (dict(q=_rows(data=FAKE + 2)), EINVAL), (dict(ko=FAKE + 8), EINVAL), (dict(q=_rows(row=-64)), EINVAL),
                         (dict(k=_rows(head=65)), EUNSUP), (dict(v=_rows(item=641)), EUNSUP),
                         # in place: only where every number stays where it is
                         (dict(qo=FAKE), EINVAL), (dict(q=_rows(item=4 * 5 * 64, row=64, head=5 * 64), qo=FAKE), EHIP)])


@no_gpu
def test_logits_refuse(L):
    tree = lpp.Tree([-1, 0, 0])

    def options(**kw):
        names = ("uncond", "tokens", "counts", "repetition", "frequency", "presence", "bias", "mask", "bias_stride", "mask_item",
                 "mask_row", "scale")
        return lpp.binding._pack_logits(*[kw.get(n, 0) for n in names])

    def call(t=tree.handle, dtype=lpp.LPP_F32, logits=FAKE, ldv=100, off=4, V=90, B=2, opts=options(), out=FAKE):
        return L.lpp_adjust_logits(t, dtype, logits, ldv, off, V, B, opts, out, None)

    _refusals(call, {}, [({}, EHIP), (dict(t=None), EINVAL), (dict(logits=None), EINVAL), (dict(opts=None), EINVAL), (dict(out=None), EINVAL),
                         (dict(dtype=3), EUNSUP), (dict(V=0), EINVAL), (dict(B=0), EINVAL), (dict(off=-1), EINVAL), (dict(off=11), EINVAL),
                         (dict(dtype=lpp.LPP_BF16), EINVAL), (dict(dtype=lpp.LPP_BF16, out=FAKE * 2), EHIP),
                         (dict(dtype=lpp.LPP_BF16, out=FAKE * 2, opts=options(uncond=FAKE * 2)), EINVAL),
                         (dict(opts=options(scale=math.nan)), EINVAL), (dict(opts=options(bias_stride=-1)), EINVAL),
                         (dict(opts=options(mask_item=-1)), EINVAL), (dict(opts=options(mask_row=-1)), EINVAL),
                         (dict(B=1 << 30), EUNSUP)])

    def counts(tokens=FAKE, length=None, B=2, T=7, V=90, out=FAKE):
        return L.lpp_token_counts(tokens, length, B, T, V, out, None)

    _refusals(counts, {}, [({}, EHIP), (dict(tokens=None), EINVAL), (dict(tokens=None, T=0), EHIP), (dict(B=0), EINVAL), (dict(T=-1), EINVAL),
                           (dict(V=0), EINVAL), (dict(out=None), EINVAL)])

    def commit(t=tree.handle, tokens=FAKE, path=FAKE, acc=FAKE, final=FAKE, B=2, V=90, out=FAKE):
        return L.lpp_commit_counts(t, tokens, path, acc, final, B, V, out, None)

    _refusals(commit, {}, [({}, EHIP)] + [({n: None}, EINVAL) for n in ("t", "tokens", "path", "acc", "final", "out")] +
              [(dict(B=0), EINVAL), (dict(V=0), EINVAL)])


def _status(call, *args, **kw):
    with pytest.raises(lpp.LppError) as e:
        call(*args, **kw)
    return e.value.status


@no_gpu
def test_the_binding_refuses_tensors_of_other_sizes_types_and_strides():
    """Host tensors here: with no device they pass for the current device's, and a right call ends in LPP_EHIP."""
    B, Hkv, M, Dh, n = 2, 2, 3, 64, 4
    cache, tree = lpp.PagedCache(lpp.LPP_F32, Hkv, Dh, 16, n), lpp.Tree([-1, 0, 0])
    new, pool = torch.zeros(B, Hkv, M, Dh), torch.zeros(n, Hkv, 16, Dh)
    i32 = dict(dtype=torch.int32)
    table, lens, path = torch.zeros(B, 2, **i32), torch.zeros(B, **i32), torch.zeros(B, tree.depth, **i32)

    def commit(k=new, p=path, a=lens, t=table, s=lens, kp=pool, nl=None):
        return _status(lpp.lpp_paged_commit_kv, cache, tree, k, new, p, a, t, s, B, kp, pool, nl)

    assert commit() == EHIP
    for bad in (dict(k=new[:1]), dict(k=new.bfloat16()), dict(k=new.transpose(2, 3).contiguous().transpose(2, 3)), dict(kp=pool[:3]),
                dict(t=table[0]), dict(t=table.long()), dict(s=lens[:1]), dict(p=path[:, :0]), dict(a=lens.float())):
        assert commit(**bad) == EINVAL, bad

    def attend(q=torch.zeros(B, 4, M, Dh), ws=torch.zeros(1 << 16, dtype=torch.uint8), s=lens):
        return _status(lpp.lpp_paged_tree_attention, cache, tree, q, pool, pool, table, new, new, s, B, 4, 20, 0.0, torch.zeros(B, 4, M, Dh), ws)

    assert attend() == EHIP
    for bad in (dict(q=new), dict(ws=torch.zeros(1 << 17, dtype=torch.uint8)[::2]), dict(s=lens[:1])):
        assert attend(**bad) == EINVAL, bad

    qkv = torch.zeros(B, M, 8, Dh)
    rotary = lpp.Rotary(32)
    q, k, v = qkv.split([4, 2, 2], 2)
    out = [torch.zeros(B, h, M, Dh) for h in (4, 2, 2)]

    def turn(q=q, o=out[0], first=lens):
        return _status(lpp.lpp_rotary_qkv, rotary, tree, lpp.LPP_F32, q, k, v, first, None, B, 4, 2, M, Dh, o, out[1], out[2])

    assert turn() == EHIP
    for bad in (dict(q=qkv), dict(q=q.bfloat16()), dict(q=torch.zeros(B, M, 4, 2 * Dh)[..., ::2]), dict(o=out[1]), dict(first=lens.long())):
        assert turn(**bad) == EINVAL, bad

    x = torch.zeros(B, M, 40)

    def logits(x=x, out=x, **kw):
        return _status(lpp.lpp_adjust_logits, tree, lpp.LPP_F32, x, 40, 0, 40, B, out, **kw)

    one = torch.zeros(B)
    assert logits(tokens=torch.zeros(B, M, **i32), repetition=one, bias=torch.zeros(40), mask=torch.zeros(B, M, 2, **i32)) == EHIP
    assert logits(bias=torch.zeros(B, 40), mask=torch.zeros(B, 2, **i32)) == EHIP
    for bad in (dict(x=x[:, :2]), dict(out=x.bfloat16()), dict(tokens=torch.zeros(B, M)), dict(counts=torch.zeros(B, 39, **i32)),
                dict(repetition=one[:1]), dict(bias=torch.zeros(39)), dict(mask=torch.zeros(B, M, 1, **i32))):
        assert logits(**bad) == EINVAL, bad


@no_gpu
def test_a_workspace_serves_smaller_calls(L):
    """Two items of 512 rows over up to 3264 positions, then less of each: more ranges of keys, in the same workspace."""
    cache = lpp.PagedCache(lpp.LPP_BF16, 8, 128, 16, 4)
    n = lpp.lpp_paged_attention_workspace(cache, 2, 32, 512, 3264)

    def chunk(B, M, S, n):
        return L.lpp_paged_chunk_attention(cache.handle, FAKE, FAKE, FAKE, FAKE, 204, FAKE, FAKE, None, None, B, 32, M, S, 0.0, 2 * FAKE, FAKE, n,
                                           None)

    for B, M, S in ((2, 512, 3200), (1, 512, 3264), (1, 1, 3264), (2, 100, 2000), (1, 40, 900), (2, 512, 3264)):
        assert lpp.lpp_paged_attention_workspace(cache, B, 32, M, S) <= n
        assert chunk(B, M, S, n) == EHIP
    assert chunk(1, 1, 3264, lpp.lpp_paged_attention_workspace(cache, 1, 32, 1, 3264) - 1) == lpp.LPP_ENOWORKSPACE


@no_gpu
def test_rotary_refuses_outputs_over_inputs_and_each_other(L):
    """A fused projection [B, M, H + 2 Hkv, Dh] in bf16 at `at`; without a tree, so that nothing but the launch is left."""
    rotary = lpp.Rotary(64)
    B, M, H, Hkv, Dh, at = 2, 5, 4, 2, 64, 1 << 20
    item, row, width = M * (H + 2 * Hkv) * Dh, (H + 2 * Hkv) * Dh, 2 * Dh
    end = at + B * item * 2

    def call(qo=2 << 20, ko=3 << 20, vo=4 << 20, q=_rows(at, item, row, Dh), k=_rows(at + H * width, item, row, Dh),
             v=_rows(at + (H + Hkv) * width, item, row, Dh), B=B, M=M):
        return L.lpp_rotary_qkv(rotary.handle, None, lpp.LPP_BF16, q, k, v, None, None, B, H, Hkv, M, Dh, qo, ko, vo, None)

    big, small = B * H * M * width, B * Hkv * M * width             # bytes of q_out, and of k_out and v_out
    packed = _rows(2 << 20, H * M * Dh, Dh, M * Dh)
    _refusals(call, {}, [
        ({}, EHIP), (dict(qo=end), EHIP), (dict(qo=at - big), EHIP), (dict(vo=at - small), EHIP), (dict(ko=(2 << 20) + big), EHIP),
        (dict(qo=at + H * width), EINVAL), (dict(qo=at + 16), EINVAL), (dict(qo=end - 16), EINVAL), (dict(qo=at - big + 16), EINVAL),
        (dict(ko=at), EINVAL), (dict(vo=at + H * width), EINVAL), (dict(ko=end - 16), EINVAL), (dict(ko=end - small), EINVAL),
        (dict(ko=2 << 20), EINVAL), (dict(vo=3 << 20), EINVAL), (dict(ko=(2 << 20) + big - 16), EINVAL), (dict(vo=(2 << 20) - small + 16), EINVAL),
        # in place, and one's own neighbours
        (dict(q=packed), EHIP), (dict(q=packed, ko=(2 << 20) + big - 16), EINVAL), (dict(q=packed, qo=(2 << 20) + 16), EINVAL),
        # one row of one item is laid out as its output is: all three in place
        (dict(B=1, M=1, qo=at, ko=at + H * width, vo=at + (H + Hkv) * width), EHIP),
        (dict(B=1, M=1, qo=at, ko=at + (H + Hkv) * width, vo=at + H * width), EINVAL)])
    # an output between an input's rows touches none of them
    assert call(q=None, qo=None, k=None, ko=None, v=_rows(at, 1 << 16, 1 << 15, Dh), vo=at + Hkv * width, M=1, B=1) == EHIP
    wide = _rows(at, 1 << 14, 1 << 13, Dh)
    assert call(q=None, qo=None, k=None, ko=None, v=wide, vo=at + Hkv * width) == EHIP
    assert call(q=None, qo=None, k=None, ko=None, v=wide, vo=at + Hkv * width - 16) == EINVAL


@no_gpu
def test_attention_over_its_pages_is_refused(L):
    cache, tree = lpp.PagedCache(lpp.LPP_BF16, 2, 64, 16, 4), lpp.Tree([-1, 0, 0])
    for kp, vp, status in ((3 * FAKE, 4 * FAKE, EHIP), (2 * FAKE, 4 * FAKE, EINVAL), (3 * FAKE, 2 * FAKE, EINVAL)):
        assert L.lpp_paged_tree_attention(cache.handle, tree.handle, FAKE, kp, vp, FAKE, 3, FAKE, FAKE, None, 2, 4, 40, 0.0, 2 * FAKE, FAKE,
                                          1 << 20, None) == status


@no_gpu
def test_a_scale_that_overflows_in_base_two_is_refused(L):
    cache, tree = lpp.PagedCache(lpp.LPP_BF16, 2, 64, 16, 4), lpp.Tree([-1, 0, 0])
    for scale, status in ((3e38, EINVAL), (2.01e38, EINVAL), (2e38, EHIP), (1e-45, EHIP)):
        assert L.lpp_paged_tree_attention(cache.handle, tree.handle, FAKE, 3 * FAKE, 3 * FAKE, FAKE, 3, FAKE, FAKE, None, 2, 4, 40, scale, 2 * FAKE,
                                          FAKE, 1 << 20, None) == status


@no_gpu
def test_launches_of_more_lanes_than_can_be_numbered_are_refused(L):
    """2^32 lanes and more, and the largest number of items below."""
    cache, tree, rotary = lpp.PagedCache(lpp.LPP_BF16, 2, 64, 16, 4), lpp.Tree([-1, 0, 0]), lpp.Rotary(64)
    far = [n << 44 for n in range(1, 7)]

    def commit(B):                                                 # two kept rows an item
        return L.lpp_paged_commit_kv(cache.handle, tree.handle, FAKE, FAKE, FAKE, FAKE, FAKE, 3, FAKE, B, FAKE, FAKE, None, None)

    def append(B):                                                 # two heads of one block
        return L.lpp_paged_append_kv(cache.handle, FAKE, FAKE, None, FAKE, 3, FAKE, B, 5, FAKE, FAKE, None, None)

    def turn(B):                                                   # eight heads, two a block
        return L.lpp_rotary_qkv(rotary.handle, None, lpp.LPP_BF16, _rows(far[0]), _rows(far[1]), _rows(far[2]), None, None, B, 4, 2, 5, 64, far[3],
                                far[4], far[5], None)

    opts = lpp.binding._pack_logits(*[0] * 12)

    def logits(B):                                                 # three rows
        return L.lpp_adjust_logits(tree.handle, lpp.LPP_F32, FAKE, 100, 4, 90, B, opts, FAKE, None)

    def counts(B):
        return L.lpp_token_counts(FAKE, None, B, 7, 90, FAKE, None)

    def commit_counts(B):
        return L.lpp_commit_counts(tree.handle, FAKE, FAKE, FAKE, FAKE, B, 90, FAKE, None)

    for call, first in ((commit, 1 << 23), (append, 1 << 23), (turn, 1 << 22), (logits, (1 << 24) // 3 + 1), (counts, 1 << 22),
                        (commit_counts, 1 << 26)):
        assert call(first) == EUNSUP and call(0x7FFFFFFF) == EUNSUP, call
        assert call(first - 1) == EHIP, call

    def chunk(B):                                                  # two heads of 200 rows, blocks of at least 256 lanes
        return L.lpp_paged_chunk_attention(cache.handle, FAKE, FAKE, FAKE, FAKE, 3, FAKE, FAKE, None, None, B, 4, 100, 40, 0.0, 2 * FAKE, FAKE, 1 << 30,
                                           None)

    assert chunk(1 << 22) == EUNSUP and chunk(1 << 18) == EHIP


@no_gpu
def test_sizes_whose_numbers_would_not_fit_are_refused(L):
    tree, rotary, far = lpp.Tree([-1, 0, 0]), lpp.Rotary(16), [n << 44 for n in range(1, 7)]
    opts = lpp.binding._pack_logits(*[0] * 12)
    for n, status in (((1 << 30) - 1, EHIP), (1 << 30, EUNSUP), (0x7FFFFFFF, EUNSUP)):
        row = _rows(far[0], 0, 16, 0)
        assert L.lpp_rotary_qkv(rotary.handle, None, lpp.LPP_BF16, row, None, None, None, None, 1, 2, 2, n, 16, far[3], None, None, None) == status
        assert L.lpp_adjust_logits(tree.handle, lpp.LPP_F32, FAKE, 1 << 31, 0, n, 1, opts, FAKE, None) == status
        assert L.lpp_token_counts(FAKE, None, 1, n, 90, FAKE, None) == status
        assert L.lpp_token_counts(FAKE, None, 1, 7, n, FAKE, None) == status


def test_a_rotary_magnitude_is_a_float32(L):
    for magnitude, status in ((1e39, EINVAL), (1e-60, EINVAL), (math.inf, EINVAL), (3e38, lpp.LPP_OK), (1e-30, lpp.LPP_OK)):
        h = C.c_void_p()
        assert L.lpp_rotary_create(C.byref(lpp.binding.RotaryConfig(dim=64, magnitude=magnitude)), C.byref(h)) == status
        L.lpp_rotary_destroy(h)


@no_gpu
def test_the_binding_refuses_what_is_missing():
    B, Hkv, M, Dh, n = 2, 2, 3, 64, 4
    cache, tree = lpp.PagedCache(lpp.LPP_F32, Hkv, Dh, 16, n), lpp.Tree([-1, 0, 0])
    new, pool, q = torch.zeros(B, Hkv, M, Dh), torch.zeros(n, Hkv, 16, Dh), torch.zeros(B, 4, M, Dh)
    i32 = dict(dtype=torch.int32)
    table, lens, path, tokens = torch.zeros(B, 2, **i32), torch.zeros(B, **i32), torch.zeros(B, tree.depth, **i32), torch.zeros(B, M, **i32)
    x, counts, ws = torch.zeros(B, M, 40), torch.zeros(B, 40, **i32), torch.zeros(1 << 16, dtype=torch.uint8)
    calls = [(lpp.lpp_paged_commit_kv, [cache, tree, new, new, path, lens, table, lens, B, pool, pool, None]),
             (lpp.lpp_paged_append_kv, [cache, new, new, None, table, lens, B, M, pool, pool, None]),
             (lpp.lpp_paged_tree_attention, [cache, tree, q, pool, pool, table, new, new, None, B, 4, 20, 0.0, q.clone(), ws]),
             (lpp.lpp_paged_chunk_attention, [cache, q, pool, pool, table, new, new, None, None, B, 4, M, 20, 0.0, q.clone(), ws]),
             (lpp.lpp_adjust_logits, [tree, lpp.LPP_F32, x, 40, 0, 40, B, x]), (lpp.lpp_token_counts, [tokens, None, B, 40, counts]),
             (lpp.lpp_commit_counts, [tree, tokens, path, lens, lens, B, 40, counts])]
    for call, args in calls:
        assert _status(call, *args) == EHIP
        for i, a in enumerate(args):
            if torch.is_tensor(a) and a is not ws:
                assert _status(call, *args[:i], None, *args[i + 1:]) == EINVAL, (call, i)
    # nothing is cached: neither pages nor a table
    for pages, t in ((None, None), (None, table), (pool, table)):
        assert _status(lpp.lpp_paged_tree_attention, cache, tree, q, pages, pages, t, new, new, None, B, 4, 0, 0.0, q.clone(), ws) == EHIP
