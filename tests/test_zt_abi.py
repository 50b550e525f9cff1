"""The training-step operators' C ABI (include/zt.h): every declared symbol is there, and whatever a call does not take is refused before
any launch.  No GPU: every call below returns before it reaches one."""
import ctypes
import os
import re

import pytest
import torch

from paper_2409_02423_amd import zc, zt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GOOD, ODD, ODD4 = 0x10000, 0x10001, 0x10004   # never dereferenced
BIG = (1 << 40) + 8


def _header():
    text = open(os.path.join(ROOT, "include", "zt.h")).read()
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def test_library_exports_every_declared_symbol():
    declared = set(re.findall(r"\b(zt_[a-z_0-9]+)\s*\(", _header()))
    assert declared == set(zt.EXPORTS)
    for name in declared:
        assert hasattr(zt.lib(), name), name


def test_binding_has_the_headers_numbers_and_structures(tmp_path):
    values = {k: eval(v) for k, v in re.findall(r"\b(ZT_[A-Z_]+) = ([0-9 <]+)", _header())}
    assert set(values) == {"ZT_RMS", "ZT_LAYER", "ZT_GATE_NONE", "ZT_GATE_CHANNEL", "ZT_GATE_FULL", "ZT_MAX_COLS", "ZT_MAX_ROWS", "ZT_SLOTS"}
    for k, v in values.items():
        assert getattr(zt, k) == v, k
    # a C program prints the structures as a C compiler lays them out
    source = ['#include <stdio.h>', '#include "%s"' % os.path.join(ROOT, "include", "zt.h"), "int main(void) {"]
    for name, cls in (("zt_residual", zt.Residual), ("zt_adamw_form", zt.AdamwForm)):
        source.append('printf("%%zu\\n", sizeof(struct %s));' % name)
        source += ['printf("%%zu\\n", offsetof(struct %s, %s));' % (name, f[0]) for f in cls._fields_]
    (tmp_path / "layout.c").write_text("\n".join(source + ["return 0; }"]))
    import subprocess
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", str(tmp_path / "layout.c"), "-o", str(tmp_path / "layout")])
    said = [int(v) for v in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for cls in (zt.Residual, zt.AdamwForm):
        want += [ctypes.sizeof(cls)] + [getattr(cls, f[0]).offset for f in cls._fields_]
    assert said == want


def test_error_code_has_a_description():
    assert zc.zc_strerror(zt.ZC_ERR_ARG) not in ("unknown error code", zc.zc_strerror(zc.ZC_ERR_NULL))


def _form(**change):
    f = zt.Residual(rows=4, cols=64, dtype=zc.ZC_BF16, kind=zt.ZT_LAYER, post=1, gate=zt.ZT_GATE_FULL, residual_scale=1.0, eps=1e-5)
    for k, v in change.items():
        setattr(f, k, v)
    return f


FORWARD = dict(x=GOOD, b=GOOD, gate=GOOD, pre_w=GOOD, pre_c=GOOD, post_w=GOOD, post_c=GOOD, y=GOOD, h=GOOD, stats=GOOD)
BACKWARD = dict(dy=GOOD, dh=GOOD, y=GOOD, b=GOOD, gate=GOOD, pre_w=GOOD, post_w=GOOD, post_c=GOOD, stats=GOOD, dx=GOOD, db=GOOD, dgate=GOOD,
                dpre_w=GOOD, dpre_c=GOOD, dpost_w=GOOD, dpost_c=GOOD, work=GOOD)
BAD_FORMS = [(dict(dtype=3), zc.ZC_ERR_DTYPE), (dict(dtype=-1), zc.ZC_ERR_DTYPE), (dict(kind=2), zt.ZC_ERR_ARG), (dict(post=2), zt.ZC_ERR_ARG),
             (dict(gate=3), zt.ZC_ERR_ARG), (dict(gate=-1), zt.ZC_ERR_ARG), (dict(residual_scale=float("inf")), zt.ZC_ERR_ARG),
             (dict(residual_scale=float("nan")), zt.ZC_ERR_ARG), (dict(eps=-1e-6), zt.ZC_ERR_ARG), (dict(eps=float("nan")), zt.ZC_ERR_ARG),
             (dict(cols=zt.ZT_MAX_COLS + 1), zc.ZC_ERR_SIZE), (dict(rows=zt.ZT_MAX_ROWS + 1), zc.ZC_ERR_SIZE)]


@pytest.mark.parametrize("change, code", BAD_FORMS + [
    (dict(stride_x=BIG), zt.ZC_ERR_ARG), (dict(stride_b=BIG), zt.ZC_ERR_ARG), (dict(stride_gate=BIG), zt.ZC_ERR_ARG),
    (dict(stride_y=63), zt.ZC_ERR_ARG), (dict(stride_h=1), zt.ZC_ERR_ARG), (dict(stride_h=BIG), zt.ZC_ERR_ARG)])
def test_forward_refuses_forms(change, code):
    assert zt.lib().zt_residual_norm(_form(**change), *FORWARD.values(), None) == code


@pytest.mark.parametrize("change, code", [(dict(x=None), zc.ZC_ERR_NULL), (dict(b=None), zc.ZC_ERR_NULL), (dict(gate=None), zc.ZC_ERR_NULL),
                                          (dict(h=None), zc.ZC_ERR_NULL), (dict(stats=ODD4), zc.ZC_ERR_ALIGN)] +
                         [({k: ODD}, zc.ZC_ERR_ALIGN) for k in FORWARD])
def test_forward_refuses_pointers(change, code):
    assert zt.lib().zt_residual_norm(_form(), *dict(FORWARD, **change).values(), None) == code


def test_forward_of_nothing_and_biases_of_rms():
    L = zt.lib()
    assert L.zt_residual_norm(None, *FORWARD.values(), None) == zc.ZC_ERR_NULL
    for empty in (dict(rows=0), dict(cols=0)):
        assert L.zt_residual_norm(_form(**empty), *dict(FORWARD, x=None, h=None).values(), None) == zc.ZC_OK
    rms = _form(kind=zt.ZT_RMS)
    assert L.zt_residual_norm(rms, *dict(FORWARD, post_c=None).values(), None) == zt.ZC_ERR_ARG
    assert L.zt_residual_norm(rms, *dict(FORWARD, pre_c=None).values(), None) == zt.ZC_ERR_ARG
    # two bytes past an fp32's place
    assert L.zt_residual_norm(_form(dtype=zc.ZC_F32), *dict(FORWARD, x=0x10002).values(), None) == zc.ZC_ERR_ALIGN


@pytest.mark.parametrize("change, code", BAD_FORMS + [
    (dict(stride_dy=BIG), zt.ZC_ERR_ARG), (dict(stride_dh=BIG), zt.ZC_ERR_ARG), (dict(stride_dx=63), zt.ZC_ERR_ARG),
    (dict(stride_db=63), zt.ZC_ERR_ARG), (dict(stride_dgate=63), zt.ZC_ERR_ARG), (dict(post=0), zt.ZC_ERR_ARG), (dict(gate=zt.ZT_GATE_NONE), zt.ZC_ERR_ARG)])
def test_backward_refuses_forms(change, code):
    assert zt.lib().zt_residual_norm_backward(_form(**change), *BACKWARD.values(), 1 << 40, None) == code


@pytest.mark.parametrize("change, code", [({k: None}, zc.ZC_ERR_NULL) for k in ("dh", "y", "b", "gate", "stats", "work")] +
                         [({k: ODD}, zc.ZC_ERR_ALIGN) for k in BACKWARD] +
                         [({k: 0x10002}, zc.ZC_ERR_ALIGN) for k in ("dpre_w", "dpre_c", "dpost_w", "dpost_c")] +
                         [(dict(stats=ODD4), zc.ZC_ERR_ALIGN), (dict(work=ODD4), zc.ZC_ERR_ALIGN)])
def test_backward_refuses_pointers(change, code):
    assert zt.lib().zt_residual_norm_backward(_form(), *dict(BACKWARD, **change).values(), 1 << 40, None) == code


def test_backward_workspace():
    L = zt.lib()
    assert L.zt_residual_work_bytes(_form(rows=0)) == 0 and L.zt_residual_work_bytes(_form(dtype=9)) == 0 and L.zt_residual_work_bytes(None) == 0
    for rows in (1, 3, 255, 100000):
        for cols in (1, 63, 513, 4099, 30001):
            for dtype in (zc.ZC_F32, zc.ZC_F16):
                f = _form(rows=rows, cols=cols, dtype=dtype)
                need = L.zt_residual_work_bytes(f)
                assert need >= 4 * 4 * cols and need % 16 == 0       # four sums over rows at least once each
                assert L.zt_residual_norm_backward(f, *BACKWARD.values(), need - 1, None) == zc.ZC_ERR_CAPACITY
    f = _form(kind=zt.ZT_RMS)
    assert L.zt_residual_norm_backward(f, *dict(BACKWARD, post_c=None, dpre_c=None).values(), 1 << 40, None) == zt.ZC_ERR_ARG
    assert L.zt_residual_norm_backward(_form(cols=0), *BACKWARD.values(), 0, None) == zc.ZC_OK


def _list(pointers, lengths, types):
    n = len(pointers)
    return (ctypes.c_void_p * n)(*pointers), (ctypes.c_size_t * n)(*lengths), (ctypes.c_int * n)(*types), n


def test_sum_of_squares_refusals():
    L = zt.lib()
    assert L.zt_sum_squares(*_list([GOOD], [4], [0])[:3], -1, 0, GOOD, None) == zc.ZC_ERR_K
    assert L.zt_sum_squares(None, None, None, 1, 0, GOOD, None) == zc.ZC_ERR_NULL
    assert L.zt_sum_squares(*_list([None], [4], [0]), 0, GOOD, None) == zc.ZC_ERR_NULL
    assert L.zt_sum_squares(*_list([GOOD], [4], [0]), 0, None, None) == zc.ZC_ERR_NULL
    assert L.zt_sum_squares(*_list([GOOD], [4], [5]), 0, GOOD, None) == zc.ZC_ERR_DTYPE
    assert L.zt_sum_squares(*_list([GOOD], [BIG], [0]), 0, GOOD, None) == zc.ZC_ERR_SIZE
    assert L.zt_sum_squares(*_list([GOOD, 0x10002], [4, 4], [0, 0]), 0, GOOD, None) == zc.ZC_ERR_ALIGN
    assert L.zt_sum_squares(*_list([GOOD, ODD], [4, 4], [0, 1]), 0, GOOD, None) == zc.ZC_ERR_ALIGN
    assert L.zt_sum_squares(*_list([GOOD], [4], [0]), 0, 0x10008, None) == zc.ZC_ERR_ALIGN
    assert L.zt_norm(None, 1.0, GOOD, None) == zc.ZC_ERR_NULL
    assert L.zt_norm(GOOD, 1.0, None, None) == zc.ZC_ERR_NULL
    assert L.zt_norm(0x10008, 1.0, GOOD, None) == zc.ZC_ERR_ALIGN
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert L.zt_norm(GOOD, scale, GOOD, None) == zt.ZC_ERR_ARG


def test_clip_refusals():
    L = zt.lib()

    def clip(pointers=(GOOD,), lengths=(4,), types=(0,), outs=(GOOD,), out_types=(0,), slots=GOOD, scale=1.0, max_norm=1.0, norm=GOOD, count=None):
        p, n, t, k = _list(pointers, lengths, types)
        o, _, ot, _ = _list(outs, lengths, out_types)
        return L.zt_clip(p, n, t, o, ot, k if count is None else count, slots, scale, max_norm, norm, None)

    assert clip(count=-1) == zc.ZC_ERR_K
    assert clip(pointers=(None,)) == clip(outs=(None,)) == clip(slots=None) == zc.ZC_ERR_NULL
    assert clip(types=(7,)) == clip(out_types=(-2,)) == zc.ZC_ERR_DTYPE
    assert clip(out_types=(1,)) == zt.ZC_ERR_ARG                       # in place, but of another type
    assert clip(outs=(0x20002,)) == clip(slots=0x10008) == clip(norm=0x10002) == zc.ZC_ERR_ALIGN
    assert clip(lengths=(BIG,)) == zc.ZC_ERR_SIZE
    for bad in (0.0, -2.0, float("nan")):
        assert clip(scale=bad) == clip(max_norm=bad) == zt.ZC_ERR_ARG
    assert clip(scale=float("inf")) == zt.ZC_ERR_ARG
    assert clip(pointers=(None,), outs=(None,), lengths=(0,), norm=None) == zc.ZC_OK   # nothing to do


def test_adamw_refusals():
    L = zt.lib()

    def adamw(grad=GOOD, slots=GOOD, param=GOOD, m=GOOD, v=GOOD, half=GOOD, norm=GOOD, **change):
        f = zt.AdamwForm(n=8, grad_dtype=zc.ZC_F32, half_dtype=zc.ZC_BF16, step=1, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, scale=1.0,
                         max_norm=1.0)
        for k, value in change.items():
            setattr(f, k, value)
        return L.zt_adamw(f, grad, slots, param, m, v, half, norm, None)

    nan, inf = float("nan"), float("inf")
    assert L.zt_adamw(None, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, None) == zc.ZC_ERR_NULL
    assert adamw(grad_dtype=4) == adamw(half_dtype=0) == zc.ZC_ERR_DTYPE
    for change in (dict(step=0), dict(step=-1), dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(eps=-1.0), dict(weight_decay=nan), dict(beta1=1.0),
                   dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan), dict(scale=0.0), dict(scale=nan), dict(max_norm=0.0), dict(max_norm=nan)):
        assert adamw(**change) == zt.ZC_ERR_ARG, change
    assert adamw(n=BIG) == zc.ZC_ERR_SIZE
    assert adamw(grad=None) == adamw(param=None) == adamw(m=None) == adamw(v=None) == adamw(slots=None) == zc.ZC_ERR_NULL
    for change in (dict(grad=0x10002), dict(slots=0x10008), dict(param=0x10002), dict(m=ODD), dict(v=0x10002), dict(half=ODD), dict(norm=0x10002)):
        assert adamw(**change) == zc.ZC_ERR_ALIGN, change
    assert adamw(n=0, grad=None, param=None, m=None, v=None, half=None, norm=None, slots=None) == zc.ZC_OK


def test_binding_rejects_host_tensors_and_wrong_combinations():
    t = torch.zeros(4, 8)
    for call in (lambda: zt.zt_residual_norm(t, t), lambda: zt.zt_residual_norm_backward(t, t, t, t, t), lambda: zt.zt_sum_squares([t]),
                 lambda: zt.zt_norm(t), lambda: zt.zt_clip([t], 1.0), lambda: zt.zt_adamw(t, t, t, t, 1e-3, 0.9, 0.95, 1e-8, 0.0, 1)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        zt.zt_sum_squares([], accumulate=True)


def test_adamw_takes_no_limit_without_the_sum_of_squares():
    """A limit that nothing is held against would leave the gradients as they are, and the step unguarded."""
    t = torch.zeros(4)
    for limit in (1.0, 1e30, float("nan")):
        with pytest.raises(ValueError):
            zt.zt_adamw(t, t, t, t, 1e-3, 0.9, 0.95, 1e-8, 0.0, 1, max_norm=limit)


def test_adamw_with_its_state_on_the_gpu_takes_no_numbers_in_its_place():
    L = zt.lib()
    good = dict(n=8, grad_dtype=zc.ZC_F32, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, scale=1.0, max_norm=1.0)
    for change, code in ((dict(d_state=0x10008), zc.ZC_ERR_ALIGN), (dict(d_state=GOOD, beta1=1.0), zt.ZC_ERR_ARG), (dict(d_state=GOOD, eps=-1.0), zt.ZC_ERR_ARG),
                         (dict(d_state=None, step=0), zt.ZC_ERR_ARG), (dict(d_state=None, step=1, lr=-1.0), zt.ZC_ERR_ARG)):
        assert L.zt_adamw(zt.AdamwForm(**dict(good, **change)), GOOD, GOOD, GOOD, GOOD, GOOD, None, None, None) == code, change
    t = torch.zeros(4)
    for lr, step, state in ((1e-3, 1, t), (None, 1, t), (1e-3, None, t), (None, None, None), (None, 1, None), (1e-3, None, None)):
        with pytest.raises(ValueError):
            zt.zt_adamw(t, t, t, t, lr, 0.9, 0.95, 1e-8, 0.0, step, d_state=state)
