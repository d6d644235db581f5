"""Host side of the norm, of 4-bit weights with group scales and of the gradients' norm (no GPU call): exported symbols, sizes,
and every refusal of the C ABI."""
import ctypes
import os
import re

import pytest
import torch

from paper_2010_11305_amd import clip, dense_lib, rmsnorm, w4
from paper_2010_11305_amd import emb_cache as ec

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ENOMEM = ec.EMB_EINVAL, ec.EMB_ENOMEM
FAKE = 1 << 20    # an aligned address that no call dereferences: the checks come first
FAR = 1 << 30     # others, apart from it


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(ec.LIB_PATH):
        from paper_2010_11305_amd import build
        build.build()
    return dense_lib.load()


def test_every_declared_symbol_is_exported(L):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "emb_dense.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(emb_(?:rmsnorm|rows8|w4|clip)_\w+)\s*\(", text)))
    assert len(names) == 18
    for n in names:
        assert ctypes.cast(getattr(L, n), ctypes.c_void_p).value


def norm(L, **kw):
    a = dict(x=FAKE, type=1, rows=4, cols=40, ldx=40, r=FAR, ldr=40, g=2 * FAR, gt=0, eps=1e-6, h=3 * FAR, ldh=40, y=4 * FAR, ldy=40, inv=5 * FAR)
    a.update(kw)
    return L.emb_rmsnorm_forward(*(a[k] for k in ("x", "type", "rows", "cols", "ldx", "r", "ldr", "g", "gt", "eps", "h", "ldh", "y", "ldy", "inv")), None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(x=FAKE + 1), dict(type=3), dict(rows=-1), dict(cols=0), dict(cols=-1), dict(ldx=39), dict(r=FAR + 1), dict(ldr=39),
    dict(g=2 * FAR + 2), dict(gt=2), dict(gt=1, g=2 * FAR + 1), dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-39), dict(eps=float("nan")),
    dict(eps=float("inf")), dict(h=3 * FAR + 1), dict(ldh=39), dict(y=None), dict(y=4 * FAR + 1), dict(ldy=39), dict(inv=5 * FAR + 2),
    dict(r=None), dict(rows=2**31), dict(cols=2**31), dict(ldx=2**62), dict(ldy=2**62),
    # shared memory other than x or the residual exactly
    dict(y=FAKE + 2), dict(y=FAKE, ldy=41), dict(h=FAKE + 80), dict(h=FAR, ldh=80), dict(y=3 * FAR), dict(inv=FAKE), dict(inv=4 * FAR + 8),
    dict(y=2 * FAR + 156), dict(h=2 * FAR), dict(inv=2 * FAR), dict(y=FAR - 2),
])
def test_norm_refusals(L, bad):
    assert norm(L, **bad) == EINVAL


def test_norm_of_nothing(L):
    assert norm(L, rows=0, x=None, r=None, h=None, y=None, inv=None) == 0


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(codes=None), dict(scales=None), dict(scales=5 * FAR + 2), dict(ldc=39), dict(codes=FAKE), dict(codes=FAR + 319), dict(scales=4 * FAR),
    dict(scales=FAKE), dict(eps=0.0), dict(cols=0), dict(h=4 * FAR), dict(ldc=2**62),
])
def test_norm8_refusals(L, bad):
    a = dict(x=FAKE, r=FAR, h=3 * FAR, cols=40, eps=1e-6, codes=4 * FAR, ldc=40, scales=5 * FAR)
    a.update(bad)
    assert L.emb_rmsnorm_forward8(a["x"], 1, 4, a["cols"], 40, a["r"], 40, 2 * FAR, 0, a["eps"], a["h"], 40, a["codes"], a["ldc"], a["scales"], None) == EINVAL


@pytest.mark.parametrize("bad", [dict(c=None), dict(s=None), dict(x=None), dict(s=FAR + 1), dict(ldc=39), dict(ldx=39), dict(t=3), dict(rows=-1), dict(cols=-1),
                                 dict(x=FAKE), dict(x=FAR - 4), dict(rows=2**31)])
def test_rows8_refusals(L, bad):
    a = dict(c=FAKE, rows=4, cols=40, ldc=40, s=FAR, x=2 * FAR, t=0, ldx=40)
    a.update(bad)
    assert L.emb_rows8_dequantize(a["c"], a["rows"], a["cols"], a["ldc"], a["s"], a["x"], a["t"], a["ldx"], None) == EINVAL


def test_norm_backward_refusals(L):
    n = ctypes.c_size_t()
    for type, rows, cols in ((1, 4, 40), (0, 300, 1), (2, 100000, 8192), (1, 100000, 20000), (0, 10**6, 64), (1, 0, 5)):
        assert L.emb_rmsnorm_backward_workspace(type, rows, cols, ctypes.byref(n)) == 0
        # at most 4 teams of 256 rows share a part, and there are no more parts than rows
        assert n.value % 256 == 0 and n.value >= rows // 1024 * cols * 4 and n.value <= 4 * rows * cols + 255
    for type, rows, cols, want in ((1, 16, 2048, 0), (1, 17, 2048, 3 * 2048 * 4), (1, 4, 8192, 0), (0, 1, 5, 0), (0, 2, 3, 256), (1, 1, 20000, 80128)):
        assert L.emb_rmsnorm_backward_workspace(type, rows, cols, ctypes.byref(n)) == 0 and n.value == want
    assert L.emb_rmsnorm_backward_workspace(1, 4, 40, None) == EINVAL
    assert L.emb_rmsnorm_backward_workspace(1, 4, 0, ctypes.byref(n)) == EINVAL and L.emb_rmsnorm_backward_workspace(3, 4, 40, ctypes.byref(n)) == EINVAL
    assert L.emb_rmsnorm_backward_workspace(1, 40, 40, ctypes.byref(n)) == 0 and n.value

    def call(**kw):
        a = dict(dy=FAKE, type=1, rows=40, cols=40, lddy=40, h=FAR, ldh=40, inv=2 * FAR, g=3 * FAR, gt=0, ds=4 * FAR, ldds=40, dx=5 * FAR, lddx=40,
                 dg=6 * FAR, ws=7 * FAR, wsb=n.value)
        a.update(kw)
        return L.emb_rmsnorm_backward(*a.values(), None)

    for bad in (dict(dy=None), dict(dy=FAKE + 1), dict(type=3), dict(rows=-1), dict(cols=0), dict(lddy=39), dict(h=None), dict(ldh=39), dict(inv=None),
                dict(inv=2 * FAR + 2), dict(g=3 * FAR + 2), dict(gt=2), dict(ds=4 * FAR + 1), dict(ldds=39), dict(dx=None), dict(lddx=39), dict(dg=6 * FAR + 2),
                dict(ws=None), dict(ws=7 * FAR + 8), dict(dx=FAKE + 2), dict(dx=FAR, lddx=80), dict(dx=2 * FAR), dict(dx=3 * FAR), dict(dg=FAKE), dict(dg=3 * FAR),
                dict(ws=FAKE), dict(dg=5 * FAR), dict(dg=7 * FAR), dict(ws=5 * FAR)):
        assert call(**bad) == EINVAL, bad
    assert call(wsb=n.value - 1) == ENOMEM


@pytest.mark.parametrize("rows,cols", [(1, 1), (16, 128), (17, 129), (4096, 12800), (5, 513), (2**31 - 1, 1), (1, 2**31 - 1)])
def test_w4_bytes(L, rows, cols):
    n = ctypes.c_size_t()
    rt, kt = -(-rows // 16), -(-cols // 128)
    for g in (32, 64, 128):
        assert L.emb_w4_query_bytes(rows, cols, g, ctypes.byref(n)) == 0 and n.value == rt * kt * 1024 + rt * (kt * 128 // g) * 64


def test_w4_refusals(L):
    n = ctypes.c_size_t(7)
    for rows, cols in ((0, 5), (5, 0)):
        assert L.emb_w4_query_bytes(rows, cols, 32, ctypes.byref(n)) == 0 and n.value == 0
    for rows, cols, g in ((-1, 4, 32), (4, -1, 32), (2**31, 1, 32), (4, 4, 16), (4, 4, 0), (4, 4, 256), (2**30, 2**30, 32)):
        assert L.emb_w4_query_bytes(rows, cols, g, ctypes.byref(n)) == EINVAL
    assert L.emb_w4_query_bytes(4, 4, 32, None) == EINVAL
    for f in (L.emb_w4_quantize, lambda x, t, r, c, ld, g, q, s: L.emb_w4_dequantize(q, r, c, g, x, t, ld, s)):
        good = (FAKE, 1, 4, 40, 40, 32, FAR, None)
        for i, v in ((0, None), (0, FAKE + 1), (1, 3), (2, -1), (3, -1), (4, 39), (5, 33), (6, None), (6, FAR + 16), (6, FAKE), (0, FAR + 1020)):
            bad = list(good)
            bad[i] = v
            assert f(*bad) == EINVAL, (i, v)
        assert f(None, 1, 0, 40, 40, 32, None, None) == 0
    for f in (L.emb_w4_pack, lambda c, s, b, r, k, g, q, st: L.emb_w4_unpack(q, r, k, g, c, s, b, st)):
        good = (FAKE, 2 * FAKE, 3 * FAKE, 4, 40, 32, FAR, None)
        for i, v in ((0, None), (1, None), (1, 2 * FAKE + 1), (2, None), (2, 3 * FAKE + 1), (3, -1), (4, -1), (5, 1), (6, None), (6, FAR + 8)):
            bad = list(good)
            bad[i] = v
            assert f(*bad) == EINVAL, (i, v)


def test_w4_linear_refusals(L):
    n = ctypes.c_size_t()
    for bad in ((4, 1, 8, 40, 32), (-1, 1, 8, 40, 32), (1, -1, 8, 40, 32), (1, 1, -8, 40, 32), (1, 1, 8, 2**24 + 1, 32), (1, 1, 8, 40, 31), (1, 2**31, 8, 40, 32)):
        assert L.emb_w4_linear_workspace(*bad, ctypes.byref(n)) == EINVAL
    assert L.emb_w4_linear_workspace(1, 1, 8, 40, 32, None) == EINVAL
    assert L.emb_w4_linear_workspace(1, 0, 8, 40, 32, ctypes.byref(n)) == 0 and n.value == 0

    def call(**kw):
        a = dict(x=FAKE, type=1, scales=None, m=4, k=40, ldx=40, w=FAR, n=8, group=32, bias=2 * FAR, relu=1, y=3 * FAR, yt=1, ldy=8, ws=4 * FAR, wsb=1 << 29)
        a.update(kw)
        return L.emb_w4_linear(*a.values(), None)

    for bad in (dict(x=None), dict(x=FAKE + 1), dict(type=4), dict(type=3), dict(scales=5 * FAR), dict(m=-1), dict(k=-1), dict(ldx=39), dict(w=None), dict(w=FAR + 8),
                dict(n=-1), dict(group=48), dict(bias=2 * FAR + 1), dict(y=None), dict(y=3 * FAR + 1), dict(yt=3), dict(ldy=7), dict(k=2**24 + 1),
                dict(y=FAKE), dict(y=FAKE + 80, ldy=40), dict(y=2 * FAR), dict(y=FAR + 1024), dict(type=3, scales=5 * FAR + 2), dict(type=3, scales=5 * FAR, y=5 * FAR + 8),
                dict(type=3, scales=5 * FAR, ldx=2**62)):
        assert call(**bad) == EINVAL, bad
    assert call(m=0, x=None, y=None) == 0 and call(n=0, w=None, y=None) == 0


def config(sizes=(5, 33), type=0, types=None):
    c = dense_lib.ClipConfig()
    keep = ((ctypes.c_int64 * len(sizes))(*sizes), (ctypes.c_int32 * len(types))(*types) if types else None)
    c.num_tensors, c.type, c.sizes = len(sizes), type, keep[0]
    if types:
        c.types = keep[1]
    return c, keep


def test_clip_refusals(L):
    s, h = dense_lib.ClipSizes(), ctypes.c_void_p(1)
    for sizes, kw in (((5, -1), {}), ((5,), dict(type=3)), ((5, 5), dict(types=[0, 4])), ((2**41,), {}), ((2**40, 2**40), {})):
        c, keep = config(sizes, **kw)
        assert L.emb_clip_query_sizes(ctypes.byref(c), ctypes.byref(s)) == EINVAL
        assert L.emb_clip_create(ctypes.byref(c), FAKE, 1 << 40, None, ctypes.byref(h)) == EINVAL and not h.value
    c, keep = config()
    c.num_tensors = 0
    assert L.emb_clip_query_sizes(ctypes.byref(c), ctypes.byref(s)) == EINVAL and L.emb_clip_query_sizes(None, ctypes.byref(s)) == EINVAL
    c, keep = config((5, 33), 9, [0, 2])     # the common type is not looked at
    assert L.emb_clip_query_sizes(ctypes.byref(c), None) == EINVAL
    assert L.emb_clip_query_sizes(ctypes.byref(c), ctypes.byref(s)) == 0 and s.state_bytes > 0 and s.workspace_bytes % 256 == 0
    for state, nbytes, want in ((None, s.state_bytes, EINVAL), (FAKE + 8, s.state_bytes, EINVAL), (FAKE, s.state_bytes - 1, ENOMEM)):
        assert L.emb_clip_create(ctypes.byref(c), state, nbytes, None, ctypes.byref(h)) == want and not h.value
    assert L.emb_clip_norm(None, FAKE, 1.0, FAKE, FAKE, 1 << 20, None) == EINVAL
    assert L.emb_clip_scale(None, FAKE, FAKE, None) == EINVAL
    assert L.emb_clip_apply(None, FAKE, 1.0, FAKE, FAKE, 1 << 20, None) == EINVAL
    assert L.emb_clip_destroy(None) == 0


def test_bindings_refuse_host_tensors():
    x = torch.zeros(4, 40)
    for bad in (lambda: rmsnorm.norm(x), lambda: rmsnorm.norm8(x), lambda: rmsnorm.backward(x, x, x[:, 0]), lambda: w4.quantize(x), lambda: clip.GradClip([x]),
                lambda: rmsnorm.Rows8(x.to(torch.int8), x[:, 0]), lambda: w4.from_codes(x.to(torch.uint8), x.half(), x.half(), 80)):
        with pytest.raises(ValueError):
            bad()
