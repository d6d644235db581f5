"""Parameters of AdamW whose memory or type changes between steps."""
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


def make(torch, **kw):
    from paper_2010_11305_amd.adamw import AdamW

    params = [torch.nn.Parameter(torch.randn(s, device="cuda")) for s in ((7,), (40, 30), (33,))]
    return params, AdamW(params, lr=1e-2, grad_dtype=torch.bfloat16, **kw)


def grads_of(torch, params):
    return [torch.ones(p.shape, dtype=torch.bfloat16, device="cuda") for p in params]


@pytest.mark.parametrize("change", ["type", "half type", "size", "order", "device"])
def test_a_changed_parameter_is_refused(torch, change):
    """Gradients still fit (they have a type of their own); the parameter no longer does, and nothing is written."""
    params, opt = make(torch)
    opt.step(grads_of(torch, params))
    p = params[1]
    grads = grads_of(torch, params)
    if change == "type":
        p.data = p.data.bfloat16()
    elif change == "half type":
        p.data = p.data.half()
    elif change == "size":
        p.data = torch.zeros(20, 30, device="cuda")
    elif change == "order":
        p.data = p.data.t()
    else:
        p.data = p.data.cpu()
    before = [q.detach().clone() for q in params]
    for _ in range(2):
        with pytest.raises(ValueError):
            opt.step(grads)
    assert opt.step_count == 1 and all(torch.equal(a, b) for a, b in zip(before, params))


def test_other_memory_of_the_same_kind_is_taken(torch):
    params, opt = make(torch)
    other, same = make(torch)
    for p, q in zip(params, other):
        q.data.copy_(p.data)
    for step in range(3):
        if step:
            params[1].data = params[1].data.clone()
        old = params[1].data
        opt.step(grads_of(torch, params))
        same.step(grads_of(torch, other))
        assert all(torch.equal(p, q) for p, q in zip(params, other))
        assert params[1].data_ptr() == old.data_ptr()


def test_shared_memory_is_refused(torch):
    """Two tensors in one memory would be updated by two workgroups at once."""
    from paper_2010_11305_amd.adamw import AdamW

    base = torch.zeros(100, device="cuda")
    p, other = torch.zeros(10, device="cuda"), torch.zeros(64, device="cuda")
    for bad in ([p, other, p], [base[:51], p, base[50:]], [base, base[10:20].view(5, 2)]):
        with pytest.raises(ValueError):
            AdamW(bad)
    params = [base[:50], base[50:], p]
    opt = AdamW(params + [base[7:7]])
    params[2].data = base[20:30]
    with pytest.raises(ValueError):
        opt.step([torch.ones(n, device="cuda") for n in (50, 50, 10, 0)])
    assert (base == 0).all()


def test_steps_that_a_counter_may_hold(torch):
    """A negative number wraps round to a huge one, and 2^64 - 1 is followed by step 0, whose corrections divide by 0."""
    from paper_2010_11305_amd.emb_cache import EmbCacheError

    params, opt = make(torch)
    for bad in (-1, -5, 2**63):
        with pytest.raises(EmbCacheError):
            opt.step_count = bad
        assert opt.step_count == 0
    for good in (2**63 - 1, 10**12, 1000):
        opt.step_count = good
        opt.step(grads_of(torch, params))
        assert opt.step_count == good + 1 and all(torch.isfinite(p).all() for p in params)


@pytest.mark.parametrize("off", [1, 2, 3])
def test_a_factor_at_an_odd_address_is_refused(torch, off):
    from array import array

    from paper_2010_11305_amd import dense_lib
    from paper_2010_11305_amd.emb_cache import EmbCacheError

    params, opt = make(torch)
    scale, grads = torch.ones(2, device="cuda"), grads_of(torch, params)
    p, g = (array("Q", [t.data_ptr() for t in ts]) for ts in (params, grads))
    with pytest.raises(EmbCacheError):
        dense_lib.call("emb_adamw_step", opt.device, opt._h, p.buffer_info()[0], g.buffer_info()[0], 1e-3, scale.data_ptr() + off)
    assert opt.step_count == 0


@pytest.mark.parametrize("elsewhere", ["cpu", "empty", "type"])
def test_a_parameter_without_a_gradient_may_be_elsewhere(torch, elsewhere):
    """Nothing of it is read or written; once it has a gradient it must be what it was."""
    params, opt = make(torch)
    other, same = make(torch)
    for p, q in zip(params, other):
        q.data.copy_(p.data)
    home = params[1].data
    params[1].data = {"cpu": home.cpu, "empty": lambda: home[:0, :0], "type": home.half}[elsewhere]()
    grads = grads_of(torch, other)
    for _ in range(2):
        opt.step([grads[0], None, grads[2]])
        same.step([grads[0], None, grads[2]])
    with pytest.raises(ValueError):
        opt.step(grads)
    params[1].data = home
    opt.step(grads)
    same.step(grads)
    assert opt.step_count == same.step_count == 3
    assert all(torch.equal(p, q) for p, q in zip(params, other))
