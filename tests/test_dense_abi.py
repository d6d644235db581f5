"""Host side of the dense operators (no GPU call): exported symbols, buffer sizes, and every
refusal of the C ABI and of the bindings' checks."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import dense_ref as ref
from paper_2010_11305_amd import adamw, dense_lib, mx4
from paper_2010_11305_amd import emb_cache as ec

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ENOMEM = ec.EMB_EINVAL, ec.EMB_ENOMEM
FAKE = 1 << 20    # an aligned address that no call dereferences: the checks come first


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(ec.LIB_PATH):
        from paper_2010_11305_amd import build
        build.build()
    return dense_lib.load()


def test_every_declared_symbol_is_exported(L):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "emb_dense.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(emb_(?:mx4|adamw)_\w+)\s*\(", text)))
    assert len(names) == 18
    for n in names:
        assert ctypes.cast(getattr(L, n), ctypes.c_void_p).value


@pytest.mark.parametrize("rows,cols", [(1, 1), (16, 128), (17, 129), (4096, 12800), (1000, 1999), (5, 513), (2**31 - 1, 1), (1, 2**31 - 1)])
def test_mx4_bytes(L, rows, cols):
    n = ctypes.c_size_t()
    assert L.emb_mx4_query_bytes(rows, cols, ctypes.byref(n)) == 0
    rt, kt = -(-rows // 16), -(-cols // 128)
    assert n.value == rt * kt * 1024 + rt * -(-kt // 4) * 256


def test_mx4_bytes_of_nothing_and_refusals(L):
    n = ctypes.c_size_t(7)
    for rows, cols in ((0, 5), (5, 0), (0, 0)):
        assert L.emb_mx4_query_bytes(rows, cols, ctypes.byref(n)) == 0 and n.value == 0
    for rows, cols in ((-1, 4), (4, -1), (2**31, 1), (1, 2**31), (2**30, 2**30)):
        assert L.emb_mx4_query_bytes(rows, cols, ctypes.byref(n)) == EINVAL
    assert L.emb_mx4_query_bytes(1, 1, None) == EINVAL


def test_quantize_refusals(L):
    good = dict(x=FAKE, type=0, rows=4, cols=40, ld=40, r=FAKE, c=None, rounding=0)

    def call(**kw):
        a = dict(good, **kw)
        return L.emb_mx4_quantize(a["x"], a["type"], a["rows"], a["cols"], a["ld"], a["r"], a["c"], a["rounding"], 1, 0,
                                  None)

    for bad in (dict(x=None), dict(x=FAKE + 2), dict(type=3), dict(type=-1), dict(rows=-1), dict(cols=-1), dict(ld=39),
                dict(r=None), dict(r=FAKE + 16), dict(c=FAKE + 16), dict(rounding=2), dict(rows=2**31),
                dict(ld=2**62), dict(x=FAKE + 1, type=1)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=0, x=None) == 0 and call(cols=0, x=None) == 0   # nothing to do


def test_dequantize_pack_unpack_refusals(L):
    assert L.emb_mx4_dequantize(None, 4, 4, FAKE, 0, 4, None) == EINVAL
    assert L.emb_mx4_dequantize(FAKE + 8, 4, 4, FAKE, 0, 4, None) == EINVAL
    assert L.emb_mx4_dequantize(FAKE, 4, 4, None, 0, 4, None) == EINVAL
    assert L.emb_mx4_dequantize(FAKE, 4, 4, FAKE, 5, 4, None) == EINVAL
    assert L.emb_mx4_dequantize(FAKE, 4, 4, FAKE, 0, 3, None) == EINVAL
    assert L.emb_mx4_dequantize(FAKE, 0, 4, None, 0, 4, None) == 0
    for f in (lambda c, s, q: L.emb_mx4_pack(c, s, 4, 4, q, None), lambda c, s, q: L.emb_mx4_unpack(q, 4, 4, c, s, None)):
        assert f(None, FAKE, FAKE) == EINVAL and f(FAKE, None, FAKE) == EINVAL
        assert f(FAKE, FAKE, None) == EINVAL and f(FAKE, FAKE, FAKE + 1) == EINVAL


def test_matmul_and_linear_refusals(L):
    def mm(a=FAKE, b=FAKE, m=4, n=8, k=40, c=FAKE, type=1, ldc=8):
        return L.emb_mx4_matmul(a, b, m, n, k, c, type, ldc, None)

    for bad in (dict(a=None), dict(b=None), dict(c=None), dict(a=FAKE + 4), dict(b=FAKE + 4), dict(c=FAKE + 1), dict(m=-1),
                dict(n=-1), dict(k=-1), dict(ldc=7), dict(type=9), dict(m=2**31), dict(k=2**24 + 1)):
        assert mm(**bad) == EINVAL, bad
    assert mm(m=0, c=None) == 0 and mm(n=0, c=None) == 0

    def lin(x=FAKE, type=1, m=4, k=40, ldx=40, w=FAKE, n=8, y=FAKE, ldy=8, ws=FAKE, wsb=1 << 40):
        return L.emb_mx4_linear(x, type, m, k, ldx, w, n, y, ldy, ws, wsb, None)

    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(x=FAKE + 1), dict(w=FAKE + 4), dict(y=FAKE + 1), dict(m=-1),
                dict(ldx=39), dict(ldy=7), dict(type=7), dict(n=2**31)):
        assert lin(**bad) == EINVAL, bad
    assert lin(m=0, x=None, y=None) == 0


def test_training_call_refusals(L):
    n = ctypes.c_size_t()
    assert L.emb_mx4_linear_train_workspace(40, 64, 128, ctypes.byref(n)) == 0 and n.value == 3 * 1024 + 3 * 256
    assert L.emb_mx4_linear_train_workspace(0, 64, 128, ctypes.byref(n)) == 0 and n.value == 0
    assert L.emb_mx4_linear_grad_workspace(40, 64, 128, ctypes.byref(n)) == 0 and n.value == (3 + 4) * 1280

    def train(x=FAKE, type=1, m=40, k=128, ldx=128, w=FAKE, n=64, y=FAKE, ldy=64, saved=FAKE, rounding=0, ws=FAKE,
              wsb=1 << 30):
        return L.emb_mx4_linear_train(x, type, m, k, ldx, w, n, y, ldy, saved, rounding, 0, 0, ws, wsb, None)

    for bad in (dict(x=None), dict(x=FAKE + 1), dict(type=3), dict(m=-1), dict(k=-1), dict(ldx=127), dict(w=None), dict(w=FAKE + 8),
                dict(y=None), dict(ldy=63), dict(saved=None), dict(saved=FAKE + 8), dict(rounding=3), dict(ws=None),
                dict(ws=FAKE + 8), dict(k=2**24 + 1)):
        assert train(**bad) == EINVAL, bad
    assert train(wsb=3839) == ENOMEM

    def grad(dy=FAKE, type=1, m=40, n=64, ldy=64, w=FAKE, k=128, saved=FAKE, dx=FAKE, ldx=128, dw=FAKE, dwt=0, ldw=128,
             rounding=1, ws=FAKE, wsb=1 << 30):
        return L.emb_mx4_linear_grad(dy, type, m, n, ldy, w, k, saved, dx, ldx, dw, dwt, ldw, rounding, 0, 0, ws, wsb, None)

    for bad in (dict(dy=None), dict(type=3), dict(m=-1), dict(n=-1), dict(ldy=63), dict(w=None), dict(w=FAKE + 8), dict(saved=None),
                dict(saved=FAKE + 8), dict(dx=None), dict(ldx=127), dict(dw=None), dict(dwt=3), dict(dw=FAKE + 2), dict(ldw=127),
                dict(rounding=3), dict(ws=None), dict(ws=FAKE + 8), dict(m=2**24 + 1)):
        assert grad(**bad) == EINVAL, bad
    assert grad(wsb=7 * 1280 - 1) == ENOMEM


def test_workspace_is_checked(L):
    """The workspace that a linear layer needs must be there, aligned and large enough."""
    n = ctypes.c_size_t()
    call = lambda ws, b: L.emb_mx4_linear(FAKE, 1, 40, 12800, 12800, FAKE, 64, FAKE, 64, ws, b, None)  # noqa: E731
    assert L.emb_mx4_linear_workspace(40, 64, 12800, ctypes.byref(n)) == 0 and n.value
    assert call(None, n.value) == EINVAL
    assert call(FAKE + 8, n.value) == EINVAL
    assert call(FAKE, n.value - 1) == ENOMEM
    assert L.emb_mx4_linear_workspace(-1, 64, 128, ctypes.byref(n)) == EINVAL
    assert L.emb_mx4_linear_workspace(4, 64, 128, None) == EINVAL
    assert L.emb_mx4_linear_workspace(4, 0, 128, ctypes.byref(n)) == 0 and n.value == 0


def adamw_config(of=(5, 33), **kw):
    c = dense_lib.AdamwConfig()
    keep = (ctypes.c_int64 * len(of))(*of)
    c.num_tensors, c.sizes = len(of), keep
    c.param_type, c.grad_type, c.state_bits, c.rounding = 0, 0, 32, 0
    c.beta1, c.beta2, c.eps, c.weight_decay, c.seed = 0.9, 0.999, 1e-8, 0.01, 1
    for k, v in kw.items():
        setattr(c, k, v)
    return c, keep


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_layout(L, bits):
    c, keep = adamw_config((5, 0, 33, 4097), state_bits=bits)
    s = dense_lib.AdamwSizes()
    assert L.emb_adamw_query_sizes(ctypes.byref(c), ctypes.byref(s)) == 0
    assert s.elements == 32 + 0 + 64 + 4128
    each = 4 if bits == 32 else 1
    assert s.first_offset == 0 and s.second_offset >= s.elements * each and s.second_offset % 256 == 0
    if bits == 8:
        assert s.second_scale_offset - s.first_scale_offset >= s.elements // 32
    assert s.state_bytes >= 2 * s.elements * each


@pytest.mark.parametrize("bad", [
    dict(num_tensors=0), dict(sizes=None), dict(param_type=2), dict(param_type=9), dict(grad_type=3), dict(state_bits=16),
    dict(rounding=2), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.5), dict(beta2=float("nan")), dict(eps=-1.0),
    dict(eps=float("inf")), dict(weight_decay=float("nan")),
])
def test_adamw_config_refusals(L, bad):
    c, keep = adamw_config(**bad)
    s = dense_lib.AdamwSizes()
    assert L.emb_adamw_query_sizes(ctypes.byref(c), ctypes.byref(s)) == EINVAL
    h = ctypes.c_void_p(1)
    assert L.emb_adamw_create(ctypes.byref(c), FAKE, 1 << 40, None, ctypes.byref(h)) == EINVAL and not h.value


def test_adamw_handle_refusals(L):
    c, keep = adamw_config((5, -1))
    s = dense_lib.AdamwSizes()
    assert L.emb_adamw_query_sizes(ctypes.byref(c), ctypes.byref(s)) == EINVAL
    assert L.emb_adamw_query_sizes(None, ctypes.byref(s)) == EINVAL
    c, keep = adamw_config()
    assert L.emb_adamw_query_sizes(ctypes.byref(c), None) == EINVAL
    assert L.emb_adamw_query_sizes(ctypes.byref(c), ctypes.byref(s)) == 0
    h = ctypes.c_void_p(1)
    assert L.emb_adamw_create(ctypes.byref(c), None, s.state_bytes, None, ctypes.byref(h)) == EINVAL
    assert L.emb_adamw_create(ctypes.byref(c), FAKE + 8, s.state_bytes, None, ctypes.byref(h)) == EINVAL
    assert L.emb_adamw_create(ctypes.byref(c), FAKE, s.state_bytes - 1, None, ctypes.byref(h)) == ENOMEM
    assert not h.value
    n = ctypes.c_uint64()
    assert L.emb_adamw_step(None, None, None, 0.1, None, None) == EINVAL
    assert L.emb_adamw_get_step(None, ctypes.byref(n)) == EINVAL and L.emb_adamw_set_step(None, 1) == EINVAL
    assert L.emb_adamw_destroy(None) == 0


def test_bindings_refuse_host_tensors():
    x = torch.zeros(4, 40)
    with pytest.raises(ValueError):
        dense_lib.matrix(x, "x")
    with pytest.raises(ValueError):
        adamw.AdamW([x])
    with pytest.raises(ValueError):
        adamw.AdamW([])
    with pytest.raises(ValueError):
        dense_lib.rounding_of("up")
    with pytest.raises(ValueError):
        dense_lib.type_of(torch.float64)
    with pytest.raises(ec.EmbCacheError):
        mx4.Mx4Matrix(-1, 4, "cpu")


# ---- the references themselves ------------------------------------------------------------------
def test_reference_e4m3_grid_is_torch():
    """The 127 magnitudes of the reference's E4M3 grid are torch's."""
    e = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(e, ref.GRID8)


def test_reference_philox_known_answers():
    """The known answers that the stochastic rounding of the tables is pinned to hold here too."""
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "golden", "philox4x32_10_kat.txt")
    seen = 0
    for line in open(path):
        v = line.split("#")[0].split()
        if len(v) != 10:
            continue
        n = [int(x, 16) for x in v]
        got = ref.philox(*[np.array([x]) for x in n[:4]], n[4] | n[5] << 32)
        assert [int(g[0]) for g in got] == n[6:]
        seen += 1
    assert seen >= 1


def test_reference_block_scale():
    """floor(log2 a) - 2 from powers of two and their neighbours; the smallest and the largest."""
    x = np.zeros((6, 32))
    x[:, 3] = [1.0, np.nextafter(1.0, 0), 7.9, 2.0**-149, 2.0**127 * 1.5, 0.0]
    code, scale = ref.mx4_quantize(x)
    assert scale[:, 0].tolist() == [125, 124, 127, 0, 252, 0]
    assert code[:, 3].tolist() == [6, 7, 7, 0, 7, 0]   # 4, 8 saturates to 6, 7.9 likewise, 2^-22, 6, 0
