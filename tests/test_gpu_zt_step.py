"""The global gradient norm, clipping and the AdamW step on the GPU against the formulas in 64 bits."""
import math

import numpy as np
import pytest

from oracle import zt_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zt():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2409_02423_amd import zt
    zt.lib()
    return zt


def _dtypes():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _tensors(seed, sizes, types, std=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    names = list(types) if not isinstance(types, str) else [types]
    return [(torch.randn(n, generator=g, dtype=torch.float64) * std).to(_dtypes()[names[i % len(names)]]).cuda() for i, n in enumerate(sizes)]


def _squares(tensors):
    """Exactly rounded: squares of what 24 bits hold are exact in 53."""
    return math.fsum(float(v) for t in tensors for v in (t.double().cpu().numpy() ** 2).ravel()) if sum(t.numel() for t in tensors) < 200000 else \
        sum(float((t.double() ** 2).sum()) for t in tensors)


# sums of n doubles in any order are off by less than n 2^-53 of the sum, in chunks and a tree by far less
EXACT = 1e-12

SIZES = ([1], [0], [], [5, 0, 3], [8191], [8192], [8193], [8192 * 3 + 1, 1, 8192, 7], [1000003], [3] * 111, [3] * 112, [3] * 113, [17] * 224, [1, 0] * 150,
         [300000] * 5 + [11] * 200 + [70001])


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%d_tensors_%d" % (len(s), sum(s)))
@pytest.mark.parametrize("types", ("f32", "bf16", "f16", ("f32", "bf16", "f16")), ids=str)
def test_sum_of_squares(zt, sizes, types):
    tensors = _tensors(1, sizes, types)
    slots = zt.zt_sum_squares(tensors)
    want = _squares(tensors)
    assert abs(float(slots.sum()) - want) <= EXACT * want
    norm = zt.zt_norm(slots, scale=0.25)
    assert abs(float(norm) - 0.25 * math.sqrt(want)) <= 2.0 ** -23 * math.sqrt(want)
    # added to what is there, as gradients of other types or other calls are
    twice = zt.zt_sum_squares(tensors, d_slots=slots, accumulate=True)
    assert twice is slots and abs(float(slots.sum()) - 2 * want) <= 2 * EXACT * want


@pytest.mark.parametrize("types", ("f32", "bf16", ("bf16", "f32", "f16")), ids=str)
def test_lists_of_more_chunks_than_workgroups(zt, types):
    """Each workgroup goes from tensor to tensor several times, long ones and short ones by turns."""
    import torch
    print("lists of more chunks than workgroups", types, flush=True)
    sizes = [3 * 1025 * 1025, 3 * 1025, 1025 * 1025, 1025, 4 * 1025 * 1025, 4 * 1025, 1025, 8192, 16384 * 40 + 5] * 3
    g = torch.Generator(device="cuda").manual_seed(12)
    names = [types] if isinstance(types, str) else list(types)
    tensors = [torch.randn(n, generator=g, device="cuda").to(_dtypes()[names[i % len(names)]]) for i, n in enumerate(sizes)]
    want = sum(float((t.double() ** 2).sum()) for t in tensors)
    assert abs(float(zt.zt_sum_squares(tensors).sum()) - want) <= EXACT * want
    out = [torch.full((n,), 7.0, device="cuda") for n in sizes]
    norm = zt.zt_clip(tensors, 2.0, d_out=out)
    assert abs(float(norm) - math.sqrt(want)) <= 2.0 ** -23 * math.sqrt(want)
    for t, o in zip(tensors, out):
        exact = t.double() * (2.0 / math.sqrt(want))
        assert bool(((o.double() - exact).abs() <= 2.0 ** -21 * exact.abs()).all())


def test_squares_neither_overflow_nor_vanish(zt):
    import torch
    for value in (3e38, 1e-30, 1.4e-45):
        t = torch.full((70000,), value, device="cuda")
        norm = zt.zt_norm(zt.zt_sum_squares([t]), scale=0.5)
        want = 0.5 * float(t[0].double()) * math.sqrt(70000)
        assert abs(float(norm) - want) <= 2.0 ** -23 * want + 2.0 ** -150 if want < 3.4e38 else float(norm) == math.inf
    small = torch.full((1000,), 2.0 ** -24, dtype=torch.float16, device="cuda")      # the smallest fp16
    assert abs(float(zt.zt_norm(zt.zt_sum_squares([small]))) - 2.0 ** -24 * math.sqrt(1000)) < 1e-12


@pytest.mark.parametrize("bad", (float("inf"), float("-inf"), float("nan")))
def test_norms_that_are_not_finite(zt, bad):
    import torch
    tensors = _tensors(2, [5000, 20000], "f32")
    tensors[1][19999] = bad
    norm = zt.zt_clip(tensors, 1.0, d_out=[torch.empty_like(t) for t in tensors])
    assert math.isnan(float(norm)) if math.isnan(bad) else float(norm) == math.inf


@pytest.mark.parametrize("types, outs", [(a, b) for a in ("f32", "bf16", "f16") for b in ("f32", "bf16", "f16")] + [(("f32", "bf16"), "f32"), (("f16", "f32"), ("bf16", "f32", "f16"))],
                         ids=str)
@pytest.mark.parametrize("max_norm", (0.5, 1e6, float("inf")))
def test_clip(zt, types, outs, max_norm):
    import torch
    sizes = [1, 8192, 8193, 0, 5, 100001, 31, 16384 * 2 + 7]
    tensors = _tensors(3, sizes, types, std=0.3)
    names = [outs] if isinstance(outs, str) else list(outs)
    names = [names[i % len(names)] for i in range(len(sizes))]
    # slices of a bucket of each type, one value apart: anything written outside its tensor would show
    out = [torch.full((n + 2,), 7.0, dtype=_dtypes()[k], device="cuda") for n, k in zip(sizes, names)]
    norm = zt.zt_clip(tensors, max_norm, scale=0.125, d_out=[o[1:-1] for o in out])
    want = 0.125 * math.sqrt(_squares(tensors))
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    factor = zt_ref.clip_factor(want, 0.125, max_norm)
    for t, o, k in zip(tensors, out, names):
        exact = factor * t.double().cpu().numpy()
        unit, tiny = zt_ref.STORED[k]
        assert np.all(np.abs(o[1:-1].double().cpu().numpy() - exact) <= (unit + 4 * zt_ref.U32) * np.abs(exact) + tiny)
        assert float(o[0]) == float(o[-1]) == 7.0


def test_clip_in_place_and_by_parts(zt):
    import torch
    sizes = [100003, 17, 8192]
    tensors = _tensors(4, sizes, ("f32", "bf16", "f16"))
    slots = zt.zt_sum_squares(tensors[:1])
    zt.zt_sum_squares(tensors[1:], d_slots=slots, accumulate=True)
    out = [torch.empty_like(t) for t in tensors]
    norm = zt.zt_clip(tensors, 2.0, d_out=out, d_slots=slots)
    whole = [torch.empty_like(t) for t in tensors]
    norm_whole = zt.zt_clip(tensors, 2.0, d_out=whole)
    assert abs(float(norm) - float(norm_whole)) <= 2.0 ** -23 * float(norm)
    assert all(torch.allclose(a.double(), b.double(), rtol=0.01, atol=0) for a, b in zip(out, whole))
    copies = [t.clone() for t in tensors]
    zt.zt_clip(copies, 2.0)
    assert all(torch.equal(a, b) for a, b in zip(copies, whole))
    # below the limit nothing changes, bit for bit
    same = [t.clone() for t in tensors]
    zt.zt_clip(same, 1e9)
    assert all(torch.equal(a, b) for a, b in zip(same, tensors))
    assert float(zt.zt_clip([], 1.0)) == 0.0


def test_many_tensors_in_several_launches(zt):
    import torch
    sizes = [(i * 37) % 900 for i in range(500)]
    tensors = _tensors(5, sizes, ("f32", "f16", "bf16"))
    copies = [t.clone() for t in tensors]
    want = math.sqrt(_squares(tensors))
    norm = zt.zt_clip(copies, 1.5)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    for t, c in zip(tensors, copies):
        exact = t.double() * (1.5 / want)
        assert bool(((c.double() - exact).abs() <= exact.abs() * (2.0 ** -8 if t.dtype == torch.bfloat16 else 2.0 ** -10 if t.dtype == torch.float16 else 2.0 ** -21) + 2.0 ** -25).all())


@pytest.mark.parametrize("n, grad, half", [(n, g, h) for n in (1, 2, 3, 4, 5, 1023, 1024, 1025, 70001) for g in ("f32", "bf16", "f16") for h in ("none", "bf16", "f16")] +
                         [((1 << 21) + 3, "f32", "bf16"), ((1 << 21) + 3, "bf16", "none")])
def test_adamw(zt, n, grad, half):
    import torch
    g = _tensors(6, [n], grad, std=0.2)[0]
    # slices that start one value behind their buffers' starts
    p, m = (torch.cat([t[:1], t])[1:] for t in _tensors(7, [n, n], "f32", std=0.5))
    v = torch.cat([torch.zeros(1, device="cuda"), _tensors(8, [n], "f32", std=0.3)[0] ** 2])[1:]
    h = None if half == "none" else torch.full((n + 2,), 7.0, dtype=_dtypes()[half], device="cuda")
    before = [t.double().cpu().numpy() for t in (g, p, m, v)]
    hyper = dict(lr=3e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=3)
    norm = zt.zt_adamw(g, p, m, v, d_half=None if h is None else h[1:-1], d_slots=zt.zt_sum_squares([g]), scale=0.5, max_norm=0.75, **hyper)
    exact_norm = 0.5 * math.sqrt(_squares([g]))
    assert abs(float(norm) - exact_norm) <= 2.0 ** -23 * exact_norm
    want, bound = zt_ref.adamw(*before, zt_ref.clip_factor(exact_norm, 0.5, 0.75), half="f32" if half == "none" else half, **hyper)
    for name, got, w, e in zip(("param", "m", "v"), (p, m, v), want, bound):
        off = np.abs(got.double().cpu().numpy() - w)
        assert np.all(off <= e), (name, float((off / e).max()))
    if h is not None:
        assert torch.equal(h[1:-1], p.to(h.dtype)) and float(h[0]) == float(h[-1]) == 7.0


def test_adamw_over_steps_without_clipping(zt):
    """Twenty steps from zero moments, gradients that change sign and vanish, against torch's optimizer in 64 bits."""
    import torch
    n = 5003
    start = _tensors(9, [n], "f32")[0]
    p, m, v = start.clone(), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    ref = start.double().cpu().requires_grad_()
    optimizer = torch.optim.AdamW([ref], lr=1e-2, betas=(0.9, 0.999), eps=1e-6, weight_decay=0.05, foreach=False)
    for step in range(1, 21):
        g = _tensors(20 + step, [n], "f32")[0]
        g[: n // 3] = 0.0
        assert zt.zt_adamw(g, p, m, v, 1e-2, 0.9, 0.999, 1e-6, 0.05, step, scale=0.5) is None
        ref.grad = 0.5 * g.double().cpu()
        optimizer.step()
    # each step's update is off by some roundings of lr, and the parameter by half a step of fp32
    off = (p.double().cpu() - ref.detach()).abs()
    assert float((off / (20 * (1e-2 * 64 * 2.0 ** -24 + ref.detach().abs() * 2.0 ** -23))).max()) <= 1.0


@pytest.mark.parametrize("bad", (float("inf"), float("nan")))
def test_adamw_leaves_everything_where_the_norm_is_not_finite(zt, bad):
    import torch
    g, p, m = _tensors(10, [3001, 3001, 3001], "f32")
    v = m ** 2
    g[1234] = bad
    kept = [t.clone() for t in (p, m, v)]
    h = torch.zeros(3001, dtype=torch.bfloat16, device="cuda")
    norm = zt.zt_adamw(g, p, m, v, 1e-2, 0.9, 0.95, 1e-8, 0.1, 1, d_half=h, d_slots=zt.zt_sum_squares([g]), max_norm=1.0)
    assert not math.isfinite(float(norm))
    assert all(torch.equal(a, b) for a, b in zip((p, m, v), kept)) and torch.equal(h, p.bfloat16())


def test_the_same_call_gives_the_same_bits(zt):
    import torch
    tensors = _tensors(11, [3000001, 77, 120000], ("f32", "bf16"))
    first = zt.zt_sum_squares(tensors)
    for _ in range(3):
        assert torch.equal(zt.zt_sum_squares(tensors), first)


def test_offsets_beyond_32_bits(zt):
    import torch
    n = (1 << 31) + 4099                       # 8.6 GB of fp32, more values than 31 bits count
    t = torch.zeros(n, device="cuda")
    places = [0, 1, (1 << 29) + 3, (1 << 30) + 1, (1 << 31) - 1, 1 << 31, (1 << 31) + 1, n - 1]
    t[places] = torch.arange(1.0, 9.0, device="cuda")
    norm = zt.zt_clip([t], 1.0)
    assert abs(float(norm) - math.sqrt(204.0)) < 1e-5
    assert np.allclose(t[places].cpu().numpy(), np.arange(1, 9) / math.sqrt(204.0), rtol=1e-6, atol=0) and int((t != 0).sum()) == 8
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    p = torch.zeros(n, device="cuda")
    zt.zt_adamw(t, p, m, v, 1e-2, 0.9, 0.95, 0.0 + 1e-8, 0.0, 1)
    assert int((p != 0).sum()) == 8 and np.allclose(p[places].cpu().numpy(), -1e-2, rtol=1e-5)


def test_another_stream_and_a_graph(zt):
    import torch
    inputs = [_tensors(30 + i, [60000, 33], "f32") for i in range(3)]
    x = [torch.empty_like(t) for t in inputs[0]]
    out = [torch.empty_like(t) for t in inputs[0]]
    slots, norm = torch.empty(zt.ZT_SLOTS, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")
    p, m, v = (torch.zeros(60000, device="cuda") for _ in range(3))
    start = _tensors(40, [60000] * 3, "f32")

    def sequence(stream):
        zt.zt_sum_squares(x, d_slots=slots, stream=stream)
        zt.zt_clip(x, 1.0, d_out=out, d_slots=slots, d_norm=norm, stream=stream)
        zt.zt_adamw(x[0], p, m, v, 1e-2, 0.9, 0.95, 1e-8, 0.1, 2, d_slots=slots, max_norm=1.0, d_norm=norm, stream=stream)

    def set_inputs(i):
        for a, b in zip(x + [p, m, v], inputs[i] + [start[0], start[1], start[2] ** 2]):
            a.copy_(b)
        torch.cuda.synchronize()

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (*out, norm, p, m, v)]

    eager, side = [], torch.cuda.Stream()
    for i in range(3):
        set_inputs(i)
        sequence(side if i == 1 else None)
        eager.append(results())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        sequence(None)
    for turn in (1, 2, 0, 2):
        print("graph replay with input", turn, flush=True)
        set_inputs(turn)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(results(), eager[turn])), turn


def test_refusals_of_the_binding(zt):
    import torch
    a, b = torch.zeros(8, device="cuda"), torch.zeros(9, device="cuda")
    with pytest.raises(TypeError):
        zt.zt_sum_squares([a.double()])
    with pytest.raises(TypeError):
        zt.zt_sum_squares([torch.zeros((4, 4), device="cuda").t()])
    with pytest.raises(ValueError):
        zt.zt_clip([a], 1.0, d_out=[b])
    with pytest.raises(ValueError):
        zt.zt_clip([a], 1.0, d_out=[a, a])
    with pytest.raises(zt.ZcError):
        zt.zt_clip([a], 0.0)
    c = torch.zeros(16, dtype=torch.float16, device="cuda")
    with pytest.raises(zt.ZcError):
        zt.zt_clip([c[:8]], 1.0, d_out=[c.view(torch.float32)])             # in place, but of another type
    with pytest.raises(ValueError):
        zt.zt_norm(torch.zeros(5, dtype=torch.float64, device="cuda"))
    with pytest.raises(ValueError):
        zt.zt_adamw(a, b, a, a, 1e-3, 0.9, 0.95, 1e-8, 0.0, 1)
    with pytest.raises(TypeError):
        zt.zt_adamw(a, a.half(), a, a, 1e-3, 0.9, 0.95, 1e-8, 0.0, 1)
    with pytest.raises(zt.ZcError):
        zt.zt_adamw(a, a, a, a, 1e-3, 0.9, 0.95, 1e-8, 0.0, 0)


@pytest.mark.parametrize("scale", (1.0, 0.5))
def test_adamw_is_left_out_where_the_norm_it_reports_is_not_finite(zt, scale):
    """70000 gradients of 3e38 have a norm that 64 bits hold and the reported value, of 32, does not: the caller is told that the step was
    left out."""
    import torch
    g = torch.full((70000,), 3e38, device="cuda")
    p, m = _tensors(50, [70000, 70000], "f32")
    v = m ** 2
    kept = [t.clone() for t in (p, m, v)]
    h = torch.zeros(70000, dtype=torch.bfloat16, device="cuda")
    norm = zt.zt_adamw(g, p, m, v, 1e-2, 0.9, 0.95, 1e-8, 0.1, 1, d_half=h, d_slots=zt.zt_sum_squares([g]), scale=scale, max_norm=1.0)
    assert float(norm) == math.inf
    assert all(torch.equal(a, b) for a, b in zip((p, m, v), kept)) and torch.equal(h, p.bfloat16())


def test_adamw_is_taken_at_the_largest_norms(zt):
    """Four gradients of 1.6e38: a norm of 3.2e38 is finite."""
    import torch
    g = torch.full((4,), 1.6e38, device="cuda")
    p, m, v = torch.ones(4, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda")
    norm = zt.zt_adamw(g, p, m, v, 1e-2, 0.9, 0.95, 1e-8, 0.0, 1, d_slots=zt.zt_sum_squares([g]), max_norm=1.0)
    assert abs(float(norm) / 3.2e38 - 1) < 1e-6
    assert np.allclose(m.cpu().numpy(), 0.1 * 0.5, rtol=1e-6) and np.allclose(p.cpu().numpy(), 1 - 1e-2, rtol=1e-6)


def test_clip_by_a_norm_that_32_bits_do_not_hold(zt):
    """The factor is made of the norm in 64 bits: 70000 gradients of 3e38 are clipped to 1 although the norm is reported as infinite."""
    import torch
    t = torch.full((70000,), 3e38, device="cuda")
    norm = zt.zt_clip([t], 1.0)
    assert float(norm) == math.inf
    # the factor is below fp32's normal numbers, 1 / 7.9e40: 2^-149 / 2 off at most, which 3e38 values of the same size make 2e-7 of them
    want = 1 / math.sqrt(70000)
    print("clipped", float(t[0]), "want", want, flush=True)
    assert bool(((t.double() - want).abs() <= 3e38 * 2.0 ** -150 + want * 2.0 ** -23).all())


def _state(lr, steps=0):
    import torch
    return torch.tensor([steps, lr, 0.0, 0.0], dtype=torch.float64, device="cuda")


@pytest.mark.parametrize("n, grad, half, clip", [(n, g, h, c) for n in (1, 5, 1025, 70001) for g, h in (("f32", "none"), ("bf16", "bf16"), ("f16", "f16")) for c in (True, False)])
def test_adamw_that_counts_its_steps(zt, n, grad, half, clip):
    """Steps with the count and the learning rate on the GPU, one of them left out and the rate changed on the way, each against the formula
    in 64 bits from where the one before it ended."""
    import torch
    p, m = _tensors(60, [n, n], "f32", std=0.5)
    v = _tensors(61, [n], "f32", std=0.3)[0] ** 2
    h = None if half == "none" else torch.empty(n, dtype=_dtypes()[half], device="cuda")
    fixed = dict(beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)
    state, taken = _state(3e-3), 0
    for turn, lr in enumerate((3e-3, 3e-3, 1e-3, 1e-3, 5e-4)):
        g = _tensors(62 + turn, [n], grad, std=0.2)[0]
        bad = clip and turn == 2
        if bad:
            g[n // 2] = math.inf
        before = [t.double().cpu().numpy() for t in (g, p, m, v)]
        kept = [t.clone() for t in (p, m, v)]
        state[1] = lr
        limit = dict(d_slots=zt.zt_sum_squares([g]), max_norm=0.75) if clip else {}
        norm = zt.zt_adamw(g, p, m, v, None, step=None, d_state=state, d_half=h, scale=0.5, **limit, **fixed)
        taken += 0 if bad else 1
        assert float(state[0]) == taken and float(state[1]) == lr
        if bad:
            assert float(norm) == math.inf and all(torch.equal(a, b) for a, b in zip((p, m, v), kept))
        else:
            factor = 0.5
            if clip:
                exact_norm = 0.5 * math.sqrt(_squares([g]))
                assert abs(float(norm) - exact_norm) <= 2.0 ** -23 * exact_norm
                factor = zt_ref.clip_factor(exact_norm, 0.5, 0.75)
            want, bound = zt_ref.adamw(*before, factor, lr=lr, step=taken, **fixed)
            for name, got, w, e in zip(("param", "m", "v"), (p, m, v), want, bound):
                off = np.abs(got.double().cpu().numpy() - w)
                assert np.all(off <= e), (turn, name, float((off / e).max()))
        if h is not None:
            assert torch.equal(h, p.to(h.dtype))


def test_a_captured_adamw_goes_on_from_step_to_step(zt):
    """Replays of one graph, a step among them that is left out, against eager calls with the same state, bit for bit, and against calls that
    are given the numbers of the steps."""
    import torch
    n, fixed = 60001, dict(beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
    grads = [_tensors(70 + i, [n], "f32")[0] for i in range(7)]
    grads[3][n - 1] = math.nan
    start = _tensors(80, [n, n], "f32")

    def fresh():
        return start[0].clone(), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")

    def step(g, t, norm, slots, stream=None, **numbers):
        zt.zt_sum_squares([g], d_slots=slots, stream=stream)
        zt.zt_adamw(g, *t, **numbers, d_slots=slots, max_norm=1.0, d_norm=norm, stream=stream, **fixed)

    def scratch():
        return torch.empty(1, device="cuda"), torch.empty(zt.ZT_SLOTS, dtype=torch.float64, device="cuda")

    eager, state, out = fresh(), _state(1e-2), scratch()
    numbered, count, out2 = fresh(), 0, scratch()
    after = []
    for i, g in enumerate(grads):
        step(g, eager, *out, lr=None, step=None, d_state=state)
        count += 0 if i == 3 else 1
        step(g, numbered, *out2, lr=1e-2, step=max(count, 1))
        torch.cuda.synchronize()
        assert float(state[0]) == count
        # the corrections are rounded once more or less: a step of fp32 of the update, and of the parameter
        assert float((eager[0] - numbered[0]).abs().max()) <= 8 * (i + 1) * (1e-2 * 2.0 ** -22 + 8 * 2.0 ** -24)
        after.append([t.clone() for t in (*eager, state, out[0])])
    x, live, state, (norm, slots), side = torch.empty(n, device="cuda"), fresh(), _state(1e-2), scratch(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(x, live, norm, slots, lr=None, step=None, d_state=state)
    for i, g in enumerate(grads):
        print("graph replay", i, flush=True)
        x.copy_(g)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip((*live, state, norm), after[i]):
            assert torch.equal(got, want) or (i == 3 and bool(got.isnan().all()) and bool(want.isnan().all())), i


def test_an_empty_shard_counts_its_steps(zt):
    import torch
    e, state = torch.empty(0, device="cuda"), _state(1e-2, 4)
    g = torch.ones(16, device="cuda")
    norm = zt.zt_adamw(e, e, e, e, None, 0.9, 0.95, 1e-8, 0.0, None, d_slots=zt.zt_sum_squares([g]), max_norm=1.0, d_state=state)
    assert float(norm) == 4.0 and float(state[0]) == 5.0
    g[3] = math.inf
    norm = zt.zt_adamw(e, e, e, e, None, 0.9, 0.95, 1e-8, 0.0, None, d_slots=zt.zt_sum_squares([g]), max_norm=1.0, d_state=state)
    assert float(norm) == math.inf and float(state[0]) == 5.0
    with pytest.raises(TypeError):
        zt.zt_adamw(g, g, g, g, None, 0.9, 0.95, 1e-8, 0.0, None, d_state=torch.zeros(4, device="cuda"))
    with pytest.raises(ValueError):
        zt.zt_adamw(g, g, g, g, None, 0.9, 0.95, 1e-8, 0.0, None, d_state=torch.zeros(3, dtype=torch.float64, device="cuda"))


@pytest.mark.parametrize("place", ("apart", "in place", "bf16"))
def test_what_clipping_writes_where_the_norm_is_not_finite(zt, place):
    """scale * max_norm / norm of an infinite norm is 0, which makes NaN of the infinite value alone; of a norm that is NaN, NaN of all."""
    import torch
    for bad in (math.inf, -math.inf, math.nan):
        tensors = _tensors(2, [5000, 20001], "f32")
        tensors[1][19999] = bad
        out = tensors if place == "in place" else [torch.full_like(t, 7.0, dtype=torch.bfloat16 if place == "bf16" else None) for t in tensors]
        norm = zt.zt_clip(tensors, 1.0, scale=0.5, d_out=out)
        if math.isnan(bad):
            assert math.isnan(float(norm)) and all(bool(o.isnan().all()) for o in out)
        else:
            assert float(norm) == math.inf
            assert bool(out[1][19999].isnan()) and sum(int((o == 0).sum()) for o in out) == 25000
        # no limit: scale alone, whatever the norm (NaN is not below it)
        tensors = _tensors(2, [5000, 20001], "f32")
        tensors[1][19999] = bad
        want = [0.5 * t for t in tensors]
        zt.zt_clip(tensors, math.inf, scale=0.5)
        if math.isnan(bad):
            assert all(bool(t.isnan().all()) for t in tensors)
        else:
            assert all(torch.equal(a, b) for a, b in zip(tensors, want))
