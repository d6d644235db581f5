"""A handle dropped while another stream still has its calls to run: its tables are not given to anyone before."""
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


@pytest.mark.parametrize("call", ["norm", "clip_", "scale_"])
def test_dropped_while_another_stream_runs(torch, call):
    """Nothing is written to the memory in question; only whose it is is looked at."""
    from paper_2010_11305_amd.clip import GradClip

    grads = [torch.full((5000,), 2.0, device="cuda"), torch.ones(77, device="cuda")]
    c = GradClip(grads, max_norm=1e9)
    at, n = c._state.data_ptr(), c._state.numel()
    one = torch.ones(1, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)     # some 0.1 s
        out = c.scale_(grads, one) if call == "scale_" else getattr(c, call)(grads)
    del c
    late = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(8)]
    running = not s.query()
    assert running, "the call ended before its handle was dropped"
    assert all(t.data_ptr() != at for t in late)
    s.synchronize()
    if call != "scale_":
        assert abs(float(out[0]) - (4 * 5000 + 77) ** 0.5) < 1e-3


def test_dropped_on_its_own_stream(torch):
    """The stream itself keeps the order: the memory may be given on at once."""
    from paper_2010_11305_amd.clip import GradClip

    grads = [torch.ones(5000, device="cuda")]
    c = GradClip(grads)
    out = c.norm(grads)
    at, n = c._state.data_ptr(), c._state.numel()
    del c
    late = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(8)]
    assert any(t.data_ptr() == at for t in late)
    assert abs(float(out[0]) - 5000**0.5) < 1e-4
