"""The residual join with the norms around a block on the GPU, forward and backward, against the formulas in 64 bits.  What a result may be
off by is oracle/zt_ref.py's bound for it."""
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


def _torch_dtype(dtype):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]


def _host(t):
    return None if t is None else t.double().cpu().numpy()


def _inputs(seed, rows, cols, dtype, layer, post, gate, mean=0.3):
    """Device tensors, and the same values as float64 on the host."""
    import torch
    g = torch.Generator().manual_seed(seed)

    def make(shape, std=1.0, at=0.0):
        return (torch.randn(shape, generator=g, dtype=torch.float64) * std + at).to(_torch_dtype(dtype)).cuda()

    d = {"x": make((rows, cols), 2.0, mean), "b": make((rows, cols), 0.7, -mean), "pre_weight": make(cols, 0.1, 1.0)}
    d["pre_bias"] = make(cols, 0.1) if layer else None
    d["post_weight"] = make(cols, 0.1, 1.0) if post else None
    d["post_bias"] = make(cols, 0.1) if post and layer else None
    d["gate"] = None if gate == "none" else make(cols if gate == "channel" else (rows, cols), 0.2, 0.5)
    d["dy"], d["dh"] = make((rows, cols), 0.3), make((rows, cols), 0.5)
    return d, {k: _host(v) for k, v in d.items()}


def _within(got, want, bound, what):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = np.abs(got - want)
    bad = ~(off <= bound)
    if bad.any():
        at = tuple(int(i) for i in np.argwhere(bad)[0])
        raise AssertionError("%s: %d of %d values are off, first at %s: got %r, want %r within %r" % (what, bad.sum(), bad.size, at, got[at], want[at], bound[at]))


def _forward_ref(h, layer, post, dtype, scale, eps=1e-5):
    return zt_ref.residual_norm(h["x"], h["b"], layer, post, h["pre_weight"], h["pre_bias"], h["post_weight"], h["post_bias"], h["gate"], scale, eps, dtype)


def _kind(zt, layer):
    return zt.ZT_LAYER if layer else zt.ZT_RMS


def _form(zt, d, layer, post, scale):
    return dict(kind=_kind(zt, layer), pre_weight=d["pre_weight"], pre_bias=d["pre_bias"], post=post, post_weight=d["post_weight"], post_bias=d["post_bias"],
                d_gate=d["gate"], residual_scale=scale)


def _stats_of(h, layer, post, y, eps=1e-5):
    import torch
    (_, _, stats), _ = zt_ref.residual_norm(y, np.zeros_like(y), layer, False, eps=eps)
    if post:
        (_, _, of_b), _ = zt_ref.residual_norm(h["b"], None, layer, False, eps=eps)
        stats[:, 0:2] = of_b[:, 2:4]
    return torch.tensor(stats, dtype=torch.float32).cuda()


def _check_forward(zt, seed, rows, cols, dtype, layer, post, gate, scale=0.7, mean=0.3):
    import torch
    d, h = _inputs(seed, rows, cols, dtype, layer, post, gate, mean)
    stats = torch.full((rows, 4), float("nan"), device="cuda")
    y, out = zt.zt_residual_norm(d["x"], d["b"], d_stats=stats, **_form(zt, d, layer, post, scale))
    (y_ref, h_ref, s_ref), (y_bound, h_bound, s_bound) = _forward_ref(h, layer, post, dtype, scale)
    _within(_host(y), y_ref, y_bound, "y")
    _within(_host(out), h_ref, h_bound, "h")
    _within(_host(stats), s_ref, s_bound + zt_ref.U32 * np.abs(s_ref), "stats")


def _check_backward(zt, seed, rows, cols, dtype, layer, post, gate, scale=0.7, with_dy=True):
    d, h = _inputs(seed, rows, cols, dtype, layer, post, gate)
    y, stats = d["x"], _stats_of(h, layer, post, h["x"])
    got = zt.zt_residual_norm_backward(d["dy"] if with_dy else None, d["dh"], y, d["b"], stats, **_form(zt, d, layer, post, scale))
    want, bound = zt_ref.residual_norm_backward(h["dy"] if with_dy else None, h["dh"], h["x"], h["b"], layer, post, h["pre_weight"], h["post_weight"],
                                                h["post_bias"], h["gate"], scale, dtype=dtype)
    for name, t in got.items():
        if t is None:
            assert d.get(name) is None, name
            continue
        key = "gate_sum" if name == "gate" and gate == "channel" else name
        _within(_host(t), want[key], bound[key], name)


FORMS = [(layer, post, gate) for layer in (False, True) for post in (False, True) for gate in ("none", "channel", "full")]
# every layout of a row over lanes, and both sides of the lines between them; odd ones; one value
COLS = (1, 2, 7, 8, 64, 255, 257, 511, 512, 513, 1000, 1024, 1025, 2047, 2048, 2049, 4096, 4097, 6144, 8191, 8192, 8193, 16384, 16391, 32768)


@pytest.mark.parametrize("dtype", ("f32", "bf16", "f16"))
@pytest.mark.parametrize("cols", COLS)
def test_forward_columns(zt, dtype, cols):
    print("forward", dtype, cols, flush=True)
    for i, (layer, post, gate) in enumerate(((False, True, "channel"), (True, True, "full"), (True, False, "none"))):
        _check_forward(zt, 100 + i, 5, cols, dtype, layer, post, gate)


@pytest.mark.parametrize("dtype", ("f32", "bf16", "f16"))
@pytest.mark.parametrize("cols", COLS)
def test_backward_columns(zt, dtype, cols):
    print("backward", dtype, cols, flush=True)
    for i, (layer, post, gate) in enumerate(((False, True, "channel"), (True, True, "full"), (True, True, "channel"), (False, False, "none"))):
        _check_backward(zt, 200 + i, 5, cols, dtype, layer, post, gate)


@pytest.mark.parametrize("layer, post, gate", FORMS)
@pytest.mark.parametrize("dtype", ("f32", "bf16", "f16"))
def test_every_form(zt, dtype, layer, post, gate):
    print("form", dtype, layer, post, gate, flush=True)
    for cols in (96, 777):
        _check_forward(zt, 300, 9, cols, dtype, layer, post, gate)
        _check_backward(zt, 301, 9, cols, dtype, layer, post, gate)
        _check_backward(zt, 302, 9, cols, dtype, layer, post, gate, with_dy=False)


@pytest.mark.parametrize("rows, cols", ((1, 6144), (2, 100), (3, 6144), (257, 65), (1023, 72), (2049, 24), (4100, 33), (700, 2000), (2600, 130)))
def test_rows(zt, rows, cols):
    print("rows", rows, cols, flush=True)
    _check_forward(zt, 400, rows, cols, "bf16", False, True, "channel")
    _check_forward(zt, 401, rows, cols, "f32", True, False, "none")
    _check_backward(zt, 402, rows, cols, "bf16", False, True, "channel")
    _check_backward(zt, 403, rows, cols, "f32", True, True, "channel")


# both sides of the lines where rows begin to share a wavefront, and where wide ones have other lanes or hold less
LINES = [("f32", cols) for cols in (3, 63, 65, 127, 129, 4097, 8189, 8193, 12291, 16381, 16385)]
LINES += [(dtype, cols) for dtype in ("bf16", "f16") for cols in (5, 127, 129, 255, 257, 8195, 12287, 12289, 16383, 16385)]


@pytest.mark.parametrize("layer, post, gate", FORMS)
@pytest.mark.parametrize("dtype, cols", LINES)
def test_every_form_at_the_lines_between_layouts(zt, dtype, cols, layer, post, gate):
    print("line", dtype, cols, layer, post, gate, flush=True)
    _check_forward(zt, 420, 3, cols, dtype, layer, post, gate)
    _check_backward(zt, 421, 3, cols, dtype, layer, post, gate)


# more rows than workgroups, so that each adds up several
@pytest.mark.parametrize("dtype, rows, cols", (("bf16", 13001, 100), ("f32", 12999, 50), ("f16", 6500, 200), ("f32", 6300, 101), ("f16", 3200, 300), ("f32", 4200, 250), ("bf16", 300, 5001), ("f32", 300, 5001),
                                               ("f32", 270, 9000), ("f16", 300, 8200), ("bf16", 300, 12289), ("bf16", 270, 16400)))
def test_workgroups_with_several_rows(zt, dtype, rows, cols):
    print("several rows", dtype, rows, cols, flush=True)
    _check_backward(zt, 422, rows, cols, dtype, False, True, "channel")
    _check_backward(zt, 423, rows, cols, dtype, True, True, "channel")
    _check_backward(zt, 424, rows, cols, dtype, True, False, "none")


def test_rows_far_from_zero(zt):
    """A mean a hundred times the deviation: the deviation comes of what is left when the mean is taken away."""
    _check_forward(zt, 410, 6, 1537, "f32", True, True, "none", mean=200.0)


def test_nothing_to_do_and_optional_parts(zt):
    import torch
    d, h = _inputs(500, 6, 300, "f32", False, False, "none")
    empty = torch.empty((0, 300), device="cuda")
    y, out = zt.zt_residual_norm(empty, empty)
    assert y.shape == out.shape == (0, 300)
    # no rows: sums over them are zero
    got = zt.zt_residual_norm_backward(empty, empty, empty, empty, torch.empty((0, 4), device="cuda"), pre_weight=d["pre_weight"])
    assert got["x"].shape == (0, 300) and bool((got["pre_weight"] == 0).all())
    # no block, no weight, y not wanted: a plain norm of x
    y, out = zt.zt_residual_norm(d["x"], want_y=False)
    (_, h_ref, _), (_, bound, _) = zt_ref.residual_norm(h["x"], None, False, False)
    assert y is None
    _within(_host(out), h_ref, bound, "plain norm")
    stats = _stats_of(h, False, False, h["x"])
    got = zt.zt_residual_norm_backward(None, d["dh"], d["x"], None, stats)
    want, bound = zt_ref.residual_norm_backward(None, h["dh"], h["x"], None, False, False)
    _within(_host(got["x"]), want["x"], bound["x"], "gradient of a plain norm")
    assert all(v is None for k, v in got.items() if k != "x")


def test_leading_dimensions(zt):
    d, h = _inputs(501, 6, 64, "f32", False, False, "none")
    y, out = zt.zt_residual_norm(d["x"].view(2, 3, 64), d["b"].view(2, 3, 64), pre_weight=d["pre_weight"])
    assert y.shape == out.shape == (2, 3, 64)
    y2, out2 = zt.zt_residual_norm(d["x"], d["b"], pre_weight=d["pre_weight"])
    assert bool((y.view(6, 64) == y2).all()) and bool((out.view(6, 64) == out2).all())
    y1, out1 = zt.zt_residual_norm(d["x"][0], d["b"][0], pre_weight=d["pre_weight"])      # one token as a vector
    assert y1.shape == (64,) and bool((out1 == out2[0]).all())


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("cols", (65, 640, 3001))
def test_strides_and_places(zt, dtype, cols):
    """Slices of wider tensors that start anywhere give what contiguous tensors give, and nothing outside them changes."""
    import torch
    rows = 7
    d, _ = _inputs(600, rows, cols, dtype, True, True, "full")
    stats = torch.empty((rows, 4), device="cuda")
    form = _form(zt, d, True, True, 0.7)
    y, h = zt.zt_residual_norm(d["x"], d["b"], d_stats=stats, **form)
    grads = zt.zt_residual_norm_backward(d["dy"], d["dh"], y, d["b"], stats, **form)

    def inside(t, left):
        wide = torch.full((rows, cols + left + 4), 7.0, dtype=t.dtype, device="cuda")
        wide[:, left:left + cols] = t
        return wide, wide[:, left:left + cols]

    def untouched(wide, left):
        return bool((wide[:, :left] == 7).all()) and bool((wide[:, left + cols:] == 7).all())

    _, x_s = inside(d["x"], 1)
    _, b_s = inside(d["b"], 2)
    _, g_s = inside(d["gate"], 3)
    _, dy_s = inside(d["dy"], 5)
    _, dh_s = inside(d["dh"], 1)
    y_w, y_s = inside(torch.zeros_like(y), 3)
    h_w, h_s = inside(torch.zeros_like(y), 1)
    dx_w, dx_s = inside(torch.zeros_like(y), 1)
    db_w, db_s = inside(torch.zeros_like(y), 2)
    stats2 = torch.empty_like(stats)
    form_s = dict(form, d_gate=g_s)
    for k in ("pre_weight", "pre_bias", "post_weight", "post_bias"):
        form_s[k] = torch.cat([form[k][:1], form[k]])[1:]             # one value further on
    zt.zt_residual_norm(x_s, b_s, d_y=y_s, d_h=h_s, d_stats=stats2, **form_s)
    got = zt.zt_residual_norm_backward(dy_s, dh_s, y_s, b_s, stats2, d_dx=dx_s, d_db=db_s, **form_s)
    assert torch.equal(y_s, y) and torch.equal(h_s, h) and torch.equal(stats2, stats)
    for k in grads:
        assert torch.equal(got[k], grads[k]), k
    assert untouched(y_w, 3) and untouched(h_w, 1) and untouched(dx_w, 1) and untouched(db_w, 2)


def test_outputs_in_place_of_inputs(zt):
    import torch
    d, _ = _inputs(601, 11, 1000, "bf16", False, True, "channel")
    form = _form(zt, d, False, True, 0.7)
    stats = torch.empty((11, 4), device="cuda")
    y, h = zt.zt_residual_norm(d["x"], d["b"], d_stats=stats, **form)
    x2, b2 = d["x"].clone(), d["b"].clone()
    zt.zt_residual_norm(x2, b2, d_y=x2, d_h=b2, **form)
    assert torch.equal(x2, y) and torch.equal(b2, h)
    want = zt.zt_residual_norm_backward(d["dy"], d["dh"], y, d["b"], stats, **form)
    dy2, dh2 = d["dy"].clone(), d["dh"].clone()
    zt.zt_residual_norm_backward(dy2, dh2, y, d["b"], stats, d_dx=dy2, d_db=dh2, **form)
    assert torch.equal(dy2, want["x"]) and torch.equal(dh2, want["b"])


@pytest.mark.parametrize("dtype, cols", (("f32", 3), ("bf16", 101), ("f32", 99), ("f16", 203), ("f32", 4999), ("bf16", 8203), ("f32", 9001), ("f16", 12299), ("bf16", 16397)))
def test_strides_and_places_of_short_and_wide_rows(zt, dtype, cols):
    print("places", dtype, cols, flush=True)
    test_strides_and_places(zt, dtype, cols)


@pytest.mark.parametrize("layer, post, gate", ((False, True, "channel"), (True, True, "channel"), (True, True, "full"), (True, False, "none"), (False, False, "channel")))
@pytest.mark.parametrize("dtype, cols", (("bf16", 5), ("f32", 99), ("bf16", 203), ("f32", 1001), ("f16", 6147), ("f32", 4999), ("bf16", 8203), ("f32", 9001), ("f16", 12299),
                                         ("f32", 16389), ("bf16", 16397)))
def test_outputs_in_place_at_odd_widths(zt, dtype, cols, layer, post, gate):
    """Where a row's last vector overlaps its neighbour, what it shares with it may have been overwritten by then."""
    import torch
    print("in place", dtype, cols, layer, post, gate, flush=True)
    rows = 300 if cols < 1000 else 5
    d, _ = _inputs(620, rows, cols, dtype, layer, post, gate)
    form = _form(zt, d, layer, post, 0.7)
    stats = torch.empty((rows, 4), device="cuda")
    y, h = zt.zt_residual_norm(d["x"], d["b"], d_stats=stats, **form)
    x2, b2 = d["x"].clone(), d["b"].clone()
    zt.zt_residual_norm(x2, b2, d_y=x2, d_h=b2, **form)
    assert torch.equal(x2, y) and torch.equal(b2, h)
    x2 = d["x"].clone()
    zt.zt_residual_norm(x2, d["b"], d_h=x2, want_y=False, **form)
    assert torch.equal(x2, h)
    want = zt.zt_residual_norm_backward(d["dy"], d["dh"], y, d["b"], stats, **form)
    for dx_is, db_is in (("dy", "dh"), ("dh", None)):
        t = {"dy": d["dy"].clone(), "dh": d["dh"].clone(), None: None}
        got = zt.zt_residual_norm_backward(t["dy"], t["dh"], y, d["b"], stats, d_dx=t[dx_is], d_db=t[db_is], **form)
        for k, v in want.items():
            assert v is None or torch.equal(got[k], v), (dx_is, k)


@pytest.mark.parametrize("cols", (300, 6144))
def test_what_is_not_a_number_stays_in_its_row(zt, cols):
    import torch
    d, _ = _inputs(602, 9, cols, "bf16", True, True, "none")
    form = _form(zt, d, True, True, 1.0)
    y, h = zt.zt_residual_norm(d["x"], d["b"], **form)
    x2, b2 = d["x"].clone(), d["b"].clone()
    x2[2, cols - 1], x2[4, 0], b2[6, 5] = float("nan"), float("inf"), float("nan")
    y2, h2 = zt.zt_residual_norm(x2, b2, **form)
    good = [0, 1, 3, 5, 7, 8]
    assert torch.equal(h2[good], h[good]) and torch.equal(y2[good], y[good])
    assert bool(h2[2].isnan().all()) and bool(h2[4].isnan().all()) and bool(h2[6].isnan().all())
    assert bool(y2[2, :-1].isfinite().all()) and bool(y2[6].isnan().all())


def test_a_row_of_zeros(zt):
    import torch
    x = torch.zeros((3, 500), dtype=torch.float16, device="cuda")
    c = torch.randn(500, device="cuda").half()
    stats = torch.empty((3, 4), device="cuda")
    y, h = zt.zt_residual_norm(x, x, kind=zt.ZT_LAYER, pre_bias=c, post=True, post_bias=None, d_stats=stats)
    assert bool((y == 0).all()) and torch.equal(h, c.expand(3, 500))
    got = zt.zt_residual_norm_backward(None, torch.ones_like(x), y, x, stats, kind=zt.ZT_LAYER, post=True)
    assert bool(got["x"].isfinite().all()) and bool(got["b"].isfinite().all())


def test_the_same_call_gives_the_same_bits(zt):
    import torch
    d, h = _inputs(603, 3000, 520, "bf16", True, True, "channel")
    stats = _stats_of(h, True, True, h["x"])
    form = _form(zt, d, True, True, 0.7)
    first = zt.zt_residual_norm_backward(d["dy"], d["dh"], d["x"], d["b"], stats, **form)
    for _ in range(3):
        again = zt.zt_residual_norm_backward(d["dy"], d["dh"], d["x"], d["b"], stats, **form)
        assert all(v is None or torch.equal(v, again[k]) for k, v in first.items())


@pytest.mark.parametrize("layer, post, gate", ((False, True, "channel"), (True, True, "full"), (True, False, "none")))
def test_gradients_against_differences(zt, layer, post, gate):
    """The backward kernel's gradients along a direction against central differences of the forward kernel, both in fp32 (differences summed
    in 64 bits): off by the forward pass's rounding over the step, and the step squared times the third derivative."""
    import torch
    rows, cols, step = 6, 200, 2.0 ** -7
    d, _ = _inputs(604, rows, cols, "f32", layer, post, gate)
    form = _form(zt, d, layer, post, 0.7)

    def loss(x, b, form):
        y, h = zt.zt_residual_norm(x, b, **form)
        return float((y.double() * d["dy"].double()).sum() + (h.double() * d["dh"].double()).sum())

    stats = torch.empty((rows, 4), device="cuda")
    y, _ = zt.zt_residual_norm(d["x"], d["b"], d_stats=stats, **form)
    got = zt.zt_residual_norm_backward(d["dy"], d["dh"], y, d["b"], stats, **form)
    g = torch.Generator().manual_seed(9)
    for name in ("x", "b", "gate", "pre_weight", "pre_bias", "post_weight", "post_bias"):
        if d[name] is None:
            continue
        along = torch.randn(d[name].shape, generator=g).cuda()
        at = {}
        for sign in (1, -1):
            moved = d[name] + sign * step * along
            args = {"x": d["x"], "b": d["b"], "form": dict(form)}
            if name in ("x", "b"):
                args[name] = moved
            else:
                args["form"]["d_gate" if name == "gate" else name] = moved
            at[sign] = loss(**args)
        slope = (at[1] - at[-1]) / (2 * step)
        want = float((got[name].double() * along.double()).sum())
        # 2400 terms of about one, rounded to 2^-24 each way; derivatives of about sqrt(2400) over a step of 2^-7
        assert abs(slope - want) < 2400 ** 0.5 * (16 * 2.0 ** -24 / step + 64 * step ** 2) + 1e-3 * abs(want), name


def test_offsets_beyond_32_bits(zt):
    import torch
    rows, cols, stride = 3, 1001, (1 << 31) + 5
    store = torch.empty(2 * stride + cols, dtype=torch.bfloat16, device="cuda")
    far = store.as_strided((rows, cols), (stride, 1))
    d, _ = _inputs(605, rows, cols, "bf16", False, False, "none")
    far.copy_(d["x"])
    y, h = zt.zt_residual_norm(d["x"], d["b"], pre_weight=d["pre_weight"])
    y2, h2 = zt.zt_residual_norm(far, d["b"], pre_weight=d["pre_weight"], d_y=far)
    assert torch.equal(far, y) and torch.equal(h2, h)


def test_more_rows_than_a_grid_has(zt):
    """2^21 workgroups are launched at most: rows beyond them are a launch of their own."""
    import torch
    rows, cols = (1 << 21) + 77, 16
    print("rows", rows, flush=True)
    g = torch.Generator(device="cuda").manual_seed(13)
    x, b, gate = (torch.randn((rows, cols), generator=g, device="cuda").bfloat16() for _ in range(3))
    stats = torch.empty((rows, 4), device="cuda")
    form = dict(post=True, residual_scale=0.5, d_gate=gate)
    y, h = zt.zt_residual_norm(x, b, d_stats=stats, **form)
    some = torch.cat([torch.arange(4), torch.arange((1 << 21) - 4, rows)]).cuda()
    stats2 = torch.empty((some.numel(), 4), device="cuda")
    y2, h2 = zt.zt_residual_norm(x[some], b[some], d_stats=stats2, **dict(form, d_gate=gate[some]))
    assert torch.equal(y[some], y2) and torch.equal(h[some], h2) and torch.equal(stats[some], stats2)
    weight = torch.ones(cols, device="cuda").bfloat16()
    got = zt.zt_residual_norm_backward(None, h, y, b, stats, pre_weight=weight, **form)
    want = zt.zt_residual_norm_backward(None, h2, y2, b[some], stats2, pre_weight=weight, **dict(form, d_gate=gate[some]))
    assert all(torch.equal(got[k][some], want[k]) for k in ("x", "b", "gate"))
    unit = y.double() * stats[:, 3:].double()
    # 2^21 terms, of which 1365 are added up one after the other
    assert bool(((got["pre_weight"].double() - (h.double() * unit).sum(0)).abs() <= 1365 * 2.0 ** -24 * (h.double() * unit).abs().sum(0)).all())


def test_another_stream_and_a_graph(zt):
    import torch
    d, _ = _inputs(606, 64, 700, "bf16", True, True, "channel")
    form = _form(zt, d, True, True, 0.7)
    x, b, dy, dh = (torch.empty_like(d[k]) for k in ("x", "b", "dy", "dh"))
    stats = torch.empty((64, 4), device="cuda")
    inputs = []
    for i in range(3):
        e, _ = _inputs(610 + i, 64, 700, "bf16", True, True, "channel")
        inputs.append([e[k] for k in ("x", "b", "dy", "dh")])
    y, h, dx, db = (torch.empty_like(x) for _ in range(4))
    kept = {}

    def sequence(stream):
        zt.zt_residual_norm(x, b, d_y=y, d_h=h, d_stats=stats, stream=stream, **form)
        kept.update(zt.zt_residual_norm_backward(dy, dh, y, b, stats, d_dx=dx, d_db=db, stream=stream, **form))

    def results():
        return [t.clone() for t in (y, h, stats, dx, db, kept["gate"], kept["pre_weight"], kept["pre_bias"], kept["post_weight"], kept["post_bias"])]

    eager = []
    side = torch.cuda.Stream()
    for i, tensors in enumerate(inputs):
        for t, v in zip((x, b, dy, dh), tensors):
            t.copy_(v)
        torch.cuda.synchronize()
        sequence(None if i != 1 else side)
        torch.cuda.synchronize()
        eager.append(results())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        sequence(None)
    for turn in (1, 2, 0, 2):
        print("graph replay with input", turn, flush=True)
        for t, v in zip((x, b, dy, dh), inputs[turn]):
            t.copy_(v)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, w) for a, w in zip(results(), eager[turn])), turn


def test_refusals_of_the_binding(zt):
    import torch
    x = torch.zeros((4, 32), device="cuda")
    with pytest.raises(ValueError):
        zt.zt_residual_norm(x, x[:3])
    with pytest.raises(TypeError):
        zt.zt_residual_norm(x, x.half())
    with pytest.raises(TypeError):
        zt.zt_residual_norm(x.t(), x.t())                                  # values of a row apart
    with pytest.raises(TypeError):
        zt.zt_residual_norm(x.double())
    with pytest.raises(TypeError):
        zt.zt_residual_norm(x, x[:1].expand(4, 32))
    with pytest.raises(ValueError):
        zt.zt_residual_norm(x, x, pre_weight=x[0, :31].contiguous())
    with pytest.raises(ValueError):
        zt.zt_residual_norm(x, x, post_weight=x[0])                        # without post
    with pytest.raises(ValueError):
        zt.zt_residual_norm(x, x, d_stats=torch.zeros(15, device="cuda"))
    with pytest.raises(zt.ZcError) as e:
        zt.zt_residual_norm(x, x, pre_bias=x[0])                           # RMS has no bias
    assert e.value.code == zt.ZC_ERR_ARG
    with pytest.raises(zt.ZcError):
        zt.zt_residual_norm(x, None, post=True)
    with pytest.raises(zt.ZcError):
        zt.zt_residual_norm(torch.zeros((1, zt.ZT_MAX_COLS + 1), device="cuda"))
    with pytest.raises(ValueError):
        zt.zt_residual_norm_backward(x, x, x, x, torch.zeros(3, device="cuda"))


def test_sums_over_rows_lose_no_more_than_a_tree_does(zt):
    """One row with gradient 1 and 511 with 2^-28, each in a workgroup of its own: added one after the other, what is small would be lost
    64 times over.  Eight partial sums a lane, then a tree of 64: no term goes through more than 13 additions."""
    import torch
    rows, cols = 512, 516
    print("sums over rows", rows, cols, flush=True)
    dh = torch.full((rows, cols), 2.0 ** -28, device="cuda")
    dh[0] = 1.0
    y, stats = torch.ones_like(dh), torch.tensor([0.0, 1.0, 0.0, 1.0], device="cuda").expand(rows, 4).contiguous()
    weight = torch.ones(cols, device="cuda")
    for kind, bias in ((zt.ZT_RMS, None), (zt.ZT_LAYER, torch.zeros(cols, device="cuda"))):
        got = zt.zt_residual_norm_backward(None, dh, y, None, stats, kind=kind, pre_weight=weight, pre_bias=bias)
        want = 1.0 + 511 * 2.0 ** -28
        for name in ("pre_weight", "pre_bias"):
            if got[name] is not None:
                assert float((got[name].double() - want).abs().max()) <= 13 * 2.0 ** -24 * want, name


# a form for each way in which the backward kernel lays rows out and holds them, with the sums that make it so
LAYOUTS = [("bf16", 5, 40), ("f32", 100, 40), ("bf16", 500, 12), ("f16", 1000, 5), ("bf16", 5003, 5), ("f16", 8191, 5), ("f32", 4099, 5), ("bf16", 12001, 4),
           ("f16", 16381, 4), ("f32", 8191, 4), ("f32", 16381, 3), ("f32", 16390, 3), ("bf16", 16397, 3)]


@pytest.mark.parametrize("layer, post, gate", ((False, True, "channel"), (True, True, "channel"), (True, True, "full"), (False, False, "full"), (True, False, "none")))
@pytest.mark.parametrize("dtype, cols, rows", LAYOUTS)
def test_outputs_that_are_not_wanted(zt, dtype, cols, rows, layer, post, gate):
    """The C call with each output left out in turn, and with all of them: the others are what they are with all of them, bit for bit, and
    a full gate's gradient may be a slice of wider rows."""
    import ctypes
    import torch
    print("outputs", dtype, cols, layer, post, gate, flush=True)
    d, h = _inputs(630, rows, cols, dtype, layer, post, gate)
    stats = _stats_of(h, layer, post, h["x"])
    form = zt.Residual(rows=rows, cols=cols, dtype=zt._DTYPES[_torch_dtype(dtype)], kind=_kind(zt, layer), post=int(post),
                       gate={"none": zt.ZT_GATE_NONE, "channel": zt.ZT_GATE_CHANNEL, "full": zt.ZT_GATE_FULL}[gate], residual_scale=0.7, eps=0.0)
    wide = cols + 5
    if gate == "full":
        form.stride_dgate = wide
    size = zt.lib().zt_residual_work_bytes(form)
    work = torch.empty(size, dtype=torch.uint8, device="cuda")
    names = ["x", "b"] + ["gate"] * (gate != "none") + ["pre_weight"] + ["pre_bias"] * layer + ["post_weight"] * post + ["post_bias"] * (layer and post)

    def call(without):
        out = {}
        for k in names:
            if k in without:
                continue
            if k in ("x", "b"):
                out[k] = torch.full((rows, cols), 7.0, dtype=d["x"].dtype, device="cuda")
            elif k == "gate" and gate == "full":
                out[k] = torch.full((rows, wide), 7.0, dtype=d["x"].dtype, device="cuda")
            else:
                out[k] = torch.full((cols,), 7.0, device="cuda")

        def at(t):
            return None if t is None else t.data_ptr()

        dgate = out.get("gate")
        if dgate is not None and gate == "full":
            dgate = dgate[:, 2:2 + cols]
        rc = zt.lib().zt_residual_norm_backward(form, at(d["dy"]), at(d["dh"]), at(d["x"]), at(d["b"]), at(d["gate"]), at(d["pre_weight"]), at(d["post_weight"]),
                                                at(d["post_bias"]), at(stats), at(out.get("x")), at(out.get("b")), at(dgate), at(out.get("pre_weight")),
                                                at(out.get("pre_bias")), at(out.get("post_weight")), at(out.get("post_bias")), at(work), size,
                                                ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == 0
        return out

    want = call(())
    through = zt.zt_residual_norm_backward(d["dy"], d["dh"], d["x"], d["b"], stats, **_form(zt, d, layer, post, 0.7))
    for k, t in want.items():
        if k == "gate" and gate == "full":
            assert bool((t[:, :2] == 7).all()) and bool((t[:, 2 + cols:] == 7).all())
            t = t[:, 2:2 + cols]
        assert torch.equal(t, through[k]), k
    for without in [(k,) for k in names] + [tuple(names), ("x", "b"), tuple(k for k in names if k not in ("x", "b"))]:
        got = call(without)
        for k, t in got.items():
            assert torch.equal(t, want[k]), (without, k)


@pytest.mark.parametrize("values", ("random", "the same"))
def test_sums_over_more_rows_than_a_grid_has(zt, values):
    """2^21 + 77 short rows, 16 to a workgroup, 768 workgroups.  A lane's 171 rows, each one multiplication and addition, and the two that
    make the normed value; 4 additions over a workgroup's lanes, 11 of partial sums, 6 in the tree over them: 194 roundings at most.
    Rows that are all the same one make roundings that all go the same way."""
    import torch
    rows, cols = (1 << 21) + 77, 16
    print("sums over rows", rows, values, flush=True)
    g = torch.Generator(device="cuda").manual_seed(14)
    y, dh = (torch.randn((rows, cols), generator=g, device="cuda").bfloat16() for _ in range(2))
    stats = torch.rand((rows, 4), generator=g, device="cuda") + 0.5
    stats[:, 2] -= 1.0
    if values == "the same":
        y, dh, stats = (t[:1].expand(t.shape).contiguous() for t in (y, dh, stats))
    weight = torch.ones(cols, device="cuda").bfloat16()
    got = zt.zt_residual_norm_backward(None, dh, y, None, stats, kind=zt.ZT_LAYER, pre_weight=weight, pre_bias=weight)
    unit = (y.double() - stats[:, 2:3].double()) * stats[:, 3:4].double()
    for name, terms in (("pre_weight", dh.double() * unit), ("pre_bias", dh.double())):
        off, magnitude = (got[name].double() - terms.sum(0)).abs(), terms.abs().sum(0)
        print(name, float((off / magnitude).max() / 2.0 ** -24), "roundings", flush=True)
        assert bool((off <= 195 * 2.0 ** -24 * magnitude).all()), name
