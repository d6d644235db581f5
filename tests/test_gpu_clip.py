"""The norm of many gradients and their scaling against 64 bits: types and their mixtures, empty and missing tensors, many
tensors, odd addresses, values whose squares leave FP32 or that are not finite, the optimizer, graphs."""
import numpy as np
import pytest

from layers_ref import DTYPES, U, f64

pytestmark = pytest.mark.gpu
SIZES = {"one": [1], "few": [3, 1000, 77], "empty": [0, 5, 0], "parts": [2048, 2049, 10000, 1], "many": [7 * k % 531 for k in range(1000)],
         "large": [5_000_000, 123_457]}


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2010_11305_amd import dense_lib
    dense_lib.load()
    return t


def gradients(torch, sizes, dtypes, seed=0):
    r = np.random.default_rng(seed)
    return [torch.from_numpy(r.standard_normal(n) * 0.1).to(DTYPES[dtypes[k % len(dtypes)]]).cuda() for k, n in enumerate(sizes)]


def exact(grads):
    return np.sqrt(sum(float((f64(g) ** 2).sum()) for g in grads if g is not None))


@pytest.mark.parametrize("dtypes", [["fp32"], ["bf16"], ["fp16"], ["fp32", "bf16", "fp16"]])
@pytest.mark.parametrize("name", SIZES)
def test_norm_and_clipping(torch, name, dtypes):
    """Squares and sums in FP64, then one rounding to FP32 of the norm and of the factor.  The products are FP32 ones,
    rounded to the type."""
    from paper_2010_11305_amd.clip import GradClip

    grads = gradients(torch, SIZES[name], dtypes)
    want = exact(grads)
    for max_norm in (want / 3 + 1e-30, want * 3 + 1e-30, float("inf")):
        c = GradClip(grads, max_norm=max_norm)
        norm, factor = c.norm(grads)
        assert abs(float(norm) - want) <= 1.01 * U * want
        limit = min(1.0, max_norm / want) if want else 1.0
        assert abs(float(factor) - limit) <= 1.01 * U * limit
        t = [g.clone() for g in grads]
        norm2, factor2 = c.clip_(t)
        assert norm2 == norm and factor2 == factor
        for a, g in zip(t, grads):
            assert torch.equal(a, (g.float() * factor).to(g.dtype))
        t = [g.clone() for g in grads]
        c.scale_(t, factor)
        for a, g in zip(t, grads):
            assert torch.equal(a, (g.float() * factor).to(g.dtype))


def test_missing_gradients_and_views(torch):
    from paper_2010_11305_amd.clip import GradClip

    flat = torch.randn(5001, device="cuda").bfloat16()
    grads = list(flat[1:].split([1001, 999, 3000]))
    c = GradClip(grads, max_norm=0.5)
    grads[1] = None
    before = flat.clone()
    norm, factor = c.clip_(grads)
    want = exact([before[1:1002], before[2001:]])
    assert abs(float(norm) - want) <= 1.01 * U * want
    assert torch.equal(flat[1002:2001], before[1002:2001]) and flat[0] == before[0]
    assert torch.equal(flat[2001:], (before[2001:].float() * factor).bfloat16())
    norm, factor = c.norm([None] * 3)
    assert norm == 0 and factor == 1


def test_values_whose_squares_leave_fp32(torch):
    from paper_2010_11305_amd.clip import GradClip

    for v in (1e30, 1e-30, 1e-44):
        g = [torch.full((3000,), v, device="cuda")]
        want = exact(g)
        norm, factor = GradClip(g, max_norm=want / 2).norm(g)
        # below the normal numbers FP32 has steps of 2^-149
        assert abs(float(norm) - want) <= 1.01 * U * want + 2.0**-150 and abs(float(factor) - 0.5) < 1e-6


def test_values_that_are_not_finite(torch):
    from paper_2010_11305_amd.clip import GradClip

    g = gradients(torch, [100, 5000], ["fp32"])
    c = GradClip(g)
    g[1][4999] = float("inf")
    norm, factor = c.norm(g)
    assert norm == float("inf") and factor == 0
    assert GradClip(g, max_norm=float("inf")).norm(g)[1] == 1
    g[0][3] = float("nan")
    norm, factor = c.clip_(g)
    assert torch.isnan(norm) and torch.isnan(factor) and torch.isnan(g[0]).all()


def test_with_the_optimizer(torch):
    """The factor as AdamW's grad_scale, and gradients scaled before: the same FP32 gradients, hence the same step."""
    from paper_2010_11305_amd.adamw import AdamW
    from paper_2010_11305_amd.clip import GradClip

    p = gradients(torch, [33, 4097], ["fp32"])
    q = [v.clone() for v in p]
    g = gradients(torch, [33, 4097], ["fp32"], 1)
    c = GradClip(p, max_norm=0.25)
    _, factor = c.norm(g)
    AdamW(p).step(g, grad_scale=factor)
    c.clip_(g)
    AdamW(q).step(g)
    assert all(torch.equal(a, b) for a, b in zip(p, q))


def test_graph_and_streams(torch):
    """One handle, two captured graphs replayed in turn and an eager call between: each call has its own workspace."""
    from paper_2010_11305_amd.clip import GradClip

    for sizes in ([1000, 3], [3_000_000, 17]):
        a, b = gradients(torch, sizes, ["fp32"], 1), gradients(torch, sizes, ["fp32"], 2)
        c = GradClip(a, max_norm=0.1)
        c.norm(a)
        torch.cuda.synchronize()
        graphs = []
        for t in (a, b):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                out = c.norm(t)
            graphs.append((g, t, out))
        for k in range(3):
            for g, t, out in graphs:
                t[0].mul_(1.5)
                g.replay()
                assert out[0] == c.norm(t)[0] and out[1] == c.norm(t)[1]
            torch.cuda.synchronize()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            x = c.norm(a)
        y = c.norm(b)
        torch.cuda.synchronize()
        assert x[0] == c.norm(a)[0] and y[0] == c.norm(b)[0]


def test_refusals(torch):
    from paper_2010_11305_amd.clip import GradClip

    g = gradients(torch, [40, 8], ["fp32"])
    c = GradClip(g)
    for bad in (lambda: GradClip([]), lambda: GradClip([torch.zeros(3)]), lambda: GradClip(g, max_norm=0.0), lambda: GradClip(g, max_norm=float("nan")),
                lambda: c.norm(g[:1]), lambda: c.norm([g[0], g[0]]), lambda: c.norm([g[0], g[1].half()]), lambda: c.norm([g[0].cpu(), g[1]]),
                lambda: c.norm([torch.zeros(80, device="cuda")[::2], g[1]]), lambda: GradClip([torch.zeros(3, device="cuda").double()])):
        with pytest.raises(ValueError):
            bad()
    same = torch.ones(50, device="cuda")
    shared = [same[:40], same[39:47]]
    assert abs(float(c.norm(shared)[0]) - 48**0.5) < 1e-6     # read only
    with pytest.raises(Exception, match="emb_clip_apply"):
        c.clip_(shared)
    with pytest.raises(Exception, match="emb_clip_scale"):
        c.scale_(shared, torch.zeros(1, device="cuda"))
    assert (same == 1).all()
    for bad in (torch.ones(1), torch.ones(2, device="cuda"), torch.ones(1, device="cuda").half()):
        with pytest.raises(ValueError):
            c.scale_(g, bad)


def test_written_tensors_count_as_changed(torch):
    from paper_2010_11305_amd.clip import GradClip

    g = [torch.ones(8, device="cuda")]
    z = (torch.ones(8, device="cuda", requires_grad=True) * g[0]).sum()
    GradClip(g).clip_(g)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()
