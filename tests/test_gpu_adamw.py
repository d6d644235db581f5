"""The AdamW step through its binding, against the formula in 64 bits (dense_ref).

FP32 bounds: one step is a dozen FP32 operations on constants that are themselves rounded, so
m and v are within 4 2^-23 of the magnitudes summed for them (m's may cancel), and the parameter
within 4 2^-24 of its magnitude plus 24 2^-24 of the step that those magnitudes would give.
8 bits: a stored moment is a neighbour on its grid of the exact one: within half a step
(nearest) or below a whole one (stochastic), with 2^-17 of a step for the error of the FP32 value
that was rounded.  BF16 parameters: half or a whole of their step, likewise."""
import numpy as np
import pytest

import dense_ref as ref

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS = 1e-2, 0.9, 0.999, 1e-8
SIZES = [1, 31, 32, 33, 7, 0, 4095, 4096, 4097, 100, 3, 20000]


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2010_11305_amd import dense_lib
    dense_lib.load()
    return t


def tensors(torch, sizes, dtype, seed, scale):
    """Views at odd offsets of one buffer, with a value before and behind each."""
    r = np.random.default_rng(seed)
    flat = torch.full((sum(sizes) + 3 * len(sizes) + 3,), 7.0, dtype=dtype, device="cuda")
    out, at = [], 1
    for n in sizes:
        v = flat[at:at + n]
        v.copy_(torch.from_numpy(r.standard_normal(n) * scale * np.exp2(r.integers(-6, 7, n))))
        out.append(v)
        at += n + 3
    return flat, out


def plain(t):
    return t.double().cpu().numpy()


def places(sizes):
    at, out = 0, []
    for n in sizes:
        out.append(at + np.arange(n))
        at += -(-n // 32) * 32
    return out


def second(state, bits):
    if bits == 32:
        return plain(state["exp_avg"]), plain(state["exp_avg_sq"])
    m = ref.e4m3_values(state["exp_avg"].view(state["exp_avg_scale"].dtype).cpu().numpy(),
                        state["exp_avg_scale"].cpu().numpy())
    r = ref.e4m3_values(state["exp_avg_root"].view(state["exp_avg_scale"].dtype).cpu().numpy(),
                        state["exp_avg_root_scale"].cpu().numpy())
    return m, r * r


def check_moment(got, exact, block_max, rounding, keep):
    """Stored values of whole blocks against exact ones."""
    s = ref.e4m3_scale(block_max)
    # on the edge of a scale either byte is right: the coarser step bounds both
    s = s + (np.abs(block_max / np.exp2(s - 127.0) / 448 - 1) < 1e-6)
    unit = np.repeat(np.exp2(s - 127.0), 32)
    y = np.abs(exact) / unit
    e = np.maximum(np.frexp(y)[1] - 1, -6)
    step = np.exp2(e - 3.0) * unit
    slack = 1.0 if rounding == "stochastic" else 0.5
    bound = step * (slack + 2.0**-17)
    if keep:
        low = (exact > 0) & (y < 2.0**-9)
        bound = np.where(low, 2.0**-9 * unit, bound)
        assert (got[exact > 0] > 0).all()
    assert (np.abs(got - exact) <= bound).all()


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [("float32", "float32"), ("float32", "bfloat16"), ("float32", "float16"),
                                        ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("bfloat16", "float16")])
def test_steps(torch, param, grad, bits, rounding):
    from paper_2010_11305_amd.adamw import AdamW

    print("adamw", param, grad, bits, rounding, flush=True)
    pt, gt = getattr(torch, param), getattr(torch, grad)
    flat, params = tensors(torch, SIZES, pt, 1, 0.05)
    decays = [0.0 if n < 32 else 0.1 for n in SIZES]
    opt = AdamW(params, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=decays, grad_dtype=gt, state_bits=bits,
                rounding=rounding, seed=99)
    at = places(SIZES)
    total = sum(-(-n // 32) * 32 for n in SIZES)
    scale = torch.tensor(0.25, device="cuda")
    for t in range(1, 5):
        before_m, before_v = second(opt.state(), bits)
        before_p = [plain(p) for p in params]
        _, grads = tensors(torch, SIZES, gt, 10 + t, 1e-2)
        opt.step(grads, lr=LR / t, grad_scale=scale)
        assert opt.step_count == t
        m, v = second(opt.state(), bits)
        want_m, want_v = np.zeros(total), np.zeros(total)
        for k, n in enumerate(SIZES):
            if not n:
                continue
            g = plain(grads[k]) * 0.25
            p, pm, pv = ref.adamw(before_p[k], g, before_m[at[k]], before_v[at[k]], t, LR / t, B1, B2, EPS, decays[k])
            want_m[at[k]], want_v[at[k]] = pm, pv
            # the step if the two parts of m had one sign
            moved = np.abs(ref.adamw(0.0, np.abs(g), np.abs(before_m[at[k]]), before_v[at[k]], t, LR / t, B1, B2, EPS, 0.0)[0])
            bound = 4 * 2.0**-24 * np.abs(before_p[k]) + 24 * 2.0**-24 * moved + 2.0**-149
            if param == "bfloat16":
                e = np.exp2(np.frexp(np.abs(p) + bound)[1] - 8.0)
                bound = bound + e * (1.0 if rounding == "stochastic" else 0.5)
            assert (np.abs(plain(params[k]) - p) <= bound).all(), (t, k)
        if bits == 32:
            for k in range(len(SIZES)):
                g = np.abs(plain(grads[k])) * 0.25
                assert (np.abs(m - want_m)[at[k]] <= 4 * 2.0**-23 * (np.abs(before_m[at[k]]) + g)).all()
                assert (np.abs(v - want_v)[at[k]] <= 4 * 2.0**-23 * (before_v[at[k]] + g * g) + 2.0**-149).all()
        else:
            root = np.sqrt(want_v)
            check_moment(m, want_m, np.abs(want_m).reshape(-1, 32).max(1), rounding, False)
            check_moment(np.sqrt(v), root, root.reshape(-1, 32).max(1), rounding, True)
        pads = np.ones(total, dtype=bool)
        pads[np.concatenate(at)] = False
        assert (m[pads] == 0).all() and (v[pads] == 0).all()
    # nothing beside the tensors was written
    keep = torch.ones(flat.numel(), dtype=torch.bool)
    o = 1
    for n in SIZES:
        keep[o:o + n] = False
        o += n + 3
    assert (flat.cpu()[keep] == 7.0).all()


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", ["float32", "bfloat16"])
def test_bits_of_one_step(torch, param, bits, rounding):
    """The step is defined operation by operation in FP32, and its roundings by given bits: numpy's FP32 operations
    (IEEE, as the kernel's) and the grids give every stored bit."""
    from paper_2010_11305_amd.adamw import AdamW

    n, t, seed = 5003, 8, 1234
    _, (p,) = tensors(torch, [n], getattr(torch, param), 5, 0.05)
    _, (g,) = tensors(torch, [n], torch.float32, 6, 1e-2)
    g[::7] = 0.0
    opt = AdamW([p], lr=LR, betas=(B1, B2), eps=EPS, weight_decay=0.1, grad_dtype=torch.float32, state_bits=bits,
                rounding=rounding, seed=seed)
    for _ in range(t - 1):
        opt.step([g])
        g = g.flip(0).contiguous()
    m, v = (x[:n].astype(np.float32) for x in second(opt.state(), bits))
    if bits == 8:      # v is the square of the root that is kept, in FP32
        r = np.sqrt(second(opt.state(), 8)[1][:n]).astype(np.float32)
        v = r * r
    before, grad = p.float().cpu().numpy(), g.cpu().numpy()
    opt.step([g])
    f = np.float32
    m = m * f(B1) + grad * f(1 - B1)
    v = v * f(B2) + (grad * grad) * f(1 - B2)
    root = np.sqrt(v)
    want = before * f(1 - LR * 0.1) - (m / (root * f(1 / np.sqrt(1 - B2**t)) + f(EPS))) * f(LR / (1 - B1**t))
    um, ur, up = ref.adam_random_bits(np.arange(n), t, seed)
    if param == "bfloat16":
        b = want.view(np.uint32).astype(np.uint64)
        if rounding == "stochastic":
            b = (b + up.astype(np.uint64)) >> np.uint64(16)
            assert np.array_equal(p.view(torch.int16).cpu().numpy().view(np.uint16), b.astype(np.uint16))
        else:
            assert torch.equal(p.cpu(), torch.from_numpy(want).bfloat16())
    else:
        assert np.array_equal(p.cpu().numpy().view(np.uint32), want.view(np.uint32))
    state = {k: x.view(torch.uint8).cpu().numpy() for k, x in opt.state().items()}
    if bits == 32:
        assert np.array_equal(state["exp_avg"].view(np.float32)[:n], m)
        assert np.array_equal(state["exp_avg_sq"].view(np.float32)[:n], v)
        return
    for name, x, u in (("exp_avg", m, um), ("exp_avg_root", root, ur)):
        block = np.zeros(-(-n // 32) * 32)
        block[:n] = np.abs(x)
        s = ref.e4m3_scale(block.reshape(-1, 32).max(1))
        assert np.array_equal(state[name + "_scale"], s)
        y = np.abs(x.astype(np.float64)) / np.repeat(np.exp2(s - 127.0), 32)[:n]
        code = ref.on_grid(y, ref.GRID8, u if rounding == "stochastic" else None)
        if name == "exp_avg_root":
            code = np.where(x > 0, np.maximum(code, 1), code)
        assert np.array_equal(state[name][:n], code + 128 * np.signbit(x))


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(torch, bits):
    """More tensors than one launch carries, each as if it were alone (rounding to nearest: no draw by place)."""
    from paper_2010_11305_amd.adamw import AdamW

    r = np.random.default_rng(4)
    sizes = [int(n) for n in r.integers(0, 300, 450)] + [9000]
    _, params = tensors(torch, sizes, torch.float32, 2, 0.1)
    _, grads = tensors(torch, sizes, torch.float32, 3, 1e-2)
    alone = [p.clone() for p in params]
    opt = AdamW(params, lr=LR, state_bits=bits)
    for _ in range(2):
        opt.step(grads)
    for k in (0, 100, 191, 192, 193, 239, 240, 241, 383, 384, 449, 450):
        one = AdamW([alone[k]], lr=LR, state_bits=bits)
        for _ in range(2):
            one.step([grads[k]])
        assert torch.equal(alone[k], params[k]), k


@pytest.mark.parametrize("bits", [32, 8])
def test_a_missing_gradient_leaves_its_tensor(torch, bits):
    from paper_2010_11305_amd.adamw import AdamW

    sizes = [100, 70, 64]
    _, params = tensors(torch, sizes, torch.float32, 2, 0.1)
    _, grads = tensors(torch, sizes, torch.float32, 3, 1e-2)
    opt = AdamW(params, lr=LR, state_bits=bits)
    opt.step(grads)
    before, state = params[1].clone(), {k: v.view(torch.uint8).clone() for k, v in opt.state().items()}
    opt.step([grads[0], None, grads[2]])
    assert torch.equal(params[1], before)
    for name, v in opt.state().items():
        per = v.view(torch.uint8).numel() // (128 + 96 + 64)
        part = slice(128 * per, (128 + 96) * per) if per else slice(4, 7)
        assert torch.equal(v.view(torch.uint8)[part], state[name][part])
        assert not torch.equal(v.view(torch.uint8), state[name])


def test_stochastic_moments_follow_what_nearest_ones_miss(torch):
    """A constant gradient: v should approach g^2 with 1 - beta2^t.  The change of r = sqrt(v) in one step is below half
    a step of the grid, so nearest rounding stops; stochastic rounding follows on average (tolerance: 6 sigma
    of the mean over 8192 elements, a walk of at most t roundings with 1/16 of the value each)."""
    from paper_2010_11305_amd.adamw import AdamW

    n, steps = 8192, 200
    want = np.sqrt(1 - B2**steps)
    got = {}
    for rounding in ("nearest", "stochastic"):
        p = torch.zeros(n, device="cuda")
        opt = AdamW([p], lr=0.0, betas=(B1, B2), state_bits=8, rounding=rounding, seed=3)
        for _ in range(steps):
            opt.step([torch.ones(n, device="cuda")])
        m, v = second(opt.state(), 8)
        got[rounding] = np.sqrt(v).mean()
    assert abs(got["stochastic"] / want - 1) < 6 * np.sqrt(steps) / 16 / np.sqrt(n) + 0.02
    assert got["nearest"] < 0.8 * want


@pytest.mark.parametrize("bits", [32, 8])
def test_values_that_are_not_finite(torch, bits):
    """A gradient that is not finite spoils its element (32 bits) or its block (8 bits), and no other."""
    from paper_2010_11305_amd.adamw import AdamW

    for value in (float("nan"), -float("nan"), float("inf")):
        p = torch.ones(100, device="cuda")
        opt = AdamW([p], lr=LR, state_bits=bits)
        g = torch.full((100,), 0.5, device="cuda")
        g[40] = value
        opt.step([g])
        assert torch.isnan(p).nonzero().flatten().tolist() == [40]
        assert all(v.view(torch.uint8)[40 // 32] == 255 for k, v in opt.state().items() if "scale" in k)
    opt.step([torch.full((100,), 0.5, device="cuda")])
    bad = torch.isnan(p).nonzero().flatten().tolist()
    assert bad == ([40] if bits == 32 else list(range(32, 64)))


def test_small_second_moments_stay_above_zero(torch):
    """An element far below its block's largest keeps a root above 0, so that its step stays bounded."""
    from paper_2010_11305_amd.adamw import AdamW

    p = torch.zeros(32, device="cuda")
    opt = AdamW([p], lr=1.0, state_bits=8, weight_decay=0.0)
    g = torch.full((32,), 1e-9, device="cuda")
    g[0] = 1.0
    for _ in range(3):
        opt.step([g])
    assert (p.abs() < 5).all()


def test_resume_stream_and_refusals(torch):
    from paper_2010_11305_amd.adamw import AdamW
    from paper_2010_11305_amd.emb_cache import EmbCacheError

    _, params = tensors(torch, [50, 3000], torch.bfloat16, 2, 0.1)
    _, grads = tensors(torch, [50, 3000], torch.bfloat16, 3, 1e-2)
    other = [p.clone() for p in params]
    make = lambda ps: AdamW(ps, lr=LR, state_bits=8, rounding="stochastic", seed=8)  # noqa: E731
    a = make(params)
    for _ in range(4):
        a.step(grads)
    b = make(other)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.step(grads)
        b.step(grads)
    torch.cuda.current_stream().wait_stream(s)
    c = make(other)      # from the state as it was saved
    for k, v in b.state().items():
        c.state()[k].copy_(v)
    c.step_count = b.step_count
    c.step(grads)
    c.step(grads)
    for x, y in zip(params, other):
        assert torch.equal(x, y)
    for bad in (lambda: a.step(grads[:1]), lambda: a.step([g.float() for g in grads]), lambda: a.step([grads[0], grads[0]]),
                lambda: a.step(grads, grad_scale=torch.ones(2, device="cuda")), lambda: AdamW([params[0], params[0].float()]),
                lambda: AdamW(params, weight_decay=[0.1]), lambda: AdamW([torch.zeros(4, 4, device="cuda").t()[:2]]),
                lambda: AdamW(params, rounding="up"), lambda: AdamW([torch.zeros(4, device="cuda").double()])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: AdamW(params, state_bits=4), lambda: AdamW(params, betas=(1.0, 0.9)), lambda: a.step(grads, lr=float("nan")),
                lambda: AdamW([params[0].half()])):
        with pytest.raises(EmbCacheError):
            bad()
