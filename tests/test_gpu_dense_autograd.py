"""Tensors that the dense operators write in place count as changed: a backward pass that kept one raises instead of
using the new values.  Results carry no history."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2010_11305_amd import dense_lib
    dense_lib.load()
    return t


def test_a_step_between_forward_and_backward(torch):
    from paper_2010_11305_amd.adamw import AdamW

    p, q = (torch.nn.Parameter(torch.ones(8, device="cuda")) for _ in range(2))
    opt = AdamW([p, q])
    x = torch.ones(8, device="cuda", requires_grad=True)
    for grads, seen in (([torch.ones_like(p), None], (p, q)), ([None, torch.ones_like(q)], (q, p))):
        changed, kept = (x * seen[0]).sum(), (x * seen[1]).sum()
        opt.step(grads)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            changed.backward()
        kept.backward()


def test_parameters_of_inference_mode(torch):
    from paper_2010_11305_amd.adamw import AdamW

    with torch.inference_mode():
        p = torch.ones(8, device="cuda")
    q, r = torch.ones(8, device="cuda"), torch.ones(8, device="cuda")
    AdamW([p, q]).step([torch.ones(8, device="cuda")] * 2)
    AdamW([r]).step([torch.ones(8, device="cuda")])
    assert torch.equal(p, r) and torch.equal(q, r) and (r != 1).all() and q._version == 1


def test_outputs_given(torch):
    from paper_2010_11305_amd import mx4

    x = torch.ones(4, 32, device="cuda", requires_grad=True)
    w4 = mx4.quantize(torch.ones(8, 32, device="cuda"))
    x4 = mx4.quantize(x)
    out, wide = torch.zeros(4, 8, device="cuda"), torch.zeros(8, 32, device="cuda")
    for call, o in ((lambda: mx4.linear(x, w4, out=out), out), (lambda: mx4.matmul(x4, w4, out=out), out),
                    (lambda: w4.dequantize(out=wide), wide)):
        z = (torch.ones_like(o, requires_grad=True) * o).sum()
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            z.backward()
    assert not mx4.linear(x, w4).requires_grad
    with torch.inference_mode():
        mx4.linear(x, w4, out=torch.zeros(4, 8, device="cuda"))
