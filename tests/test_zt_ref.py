"""The 64-bit reference of the training-step operators against differences of its own forward formulas and against torch's
automatic differentiation in 64 bits; no GPU."""
import numpy as np
import pytest
import torch

from oracle import zt_ref


def _case(seed, rows, cols, layer, post, gate):
    r = np.random.default_rng(seed)
    a = {"x": r.standard_normal((rows, cols)) * 2, "b": r.standard_normal((rows, cols)) + 0.3, "pre_w": 1 + 0.1 * r.standard_normal(cols)}
    a["pre_c"] = 0.1 * r.standard_normal(cols) if layer else None
    a["post_w"] = 1 + 0.1 * r.standard_normal(cols) if post else None
    a["post_c"] = 0.1 * r.standard_normal(cols) if post and layer else None
    a["gate"] = None if gate == "none" else 0.5 + 0.2 * r.standard_normal(cols if gate == "channel" else (rows, cols))
    return a, r.standard_normal((rows, cols)), r.standard_normal((rows, cols))


FORMS = [(layer, post, gate) for layer in (False, True) for post in (False, True) for gate in ("none", "channel", "full")]
NAMES = {"x": "x", "b": "b", "pre_w": "pre_weight", "pre_c": "pre_bias", "post_w": "post_weight", "post_c": "post_bias"}


@pytest.mark.parametrize("layer, post, gate", FORMS)
def test_gradients_against_differences(layer, post, gate):
    a, cy, ch = _case(5, 3, 7, layer, post, gate)

    def loss(a):
        (y, h, _), _ = zt_ref.residual_norm(a["x"], a["b"], layer, post, a["pre_w"], a["pre_c"], a["post_w"], a["post_c"], a["gate"], scale=0.7, eps=1e-3)
        return (y * cy).sum() + (h * ch).sum()

    (y, _, _), _ = zt_ref.residual_norm(a["x"], a["b"], layer, post, a["pre_w"], a["pre_c"], a["post_w"], a["post_c"], a["gate"], scale=0.7, eps=1e-3)
    got, _ = zt_ref.residual_norm_backward(cy, ch, y, a["b"], layer, post, a["pre_w"], a["post_w"], a["post_c"], a["gate"], scale=0.7, eps=1e-3)
    names = dict(NAMES, gate="gate_sum" if gate == "channel" else "gate")
    step = 1e-5     # differences are off by step^2 times third derivatives of about one, and by 1e-15 / step times the loss
    for k, v in a.items():
        if v is None:
            continue
        g = got[names[k]]
        for at in np.ndindex(v.shape):
            up, down = dict(a, **{k: v.copy()}), dict(a, **{k: v.copy()})
            up[k][at] += step
            down[k][at] -= step
            assert abs((loss(up) - loss(down)) / (2 * step) - g[at]) < 2e-8, (k, at)


@pytest.mark.parametrize("layer, post, gate", FORMS)
def test_forward_and_gradients_against_automatic_differentiation(layer, post, gate):
    a, cy, ch = _case(6, 4, 33, layer, post, gate)
    t = {k: None if v is None else torch.tensor(v, requires_grad=True) for k, v in a.items()}

    def normed(v, w, c):
        if layer:
            return torch.nn.functional.layer_norm(v, v.shape[-1:], w, c, 1e-5)
        return v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-5) * w

    z = normed(t["b"], t["post_w"], t["post_c"]) if post else t["b"]
    y = 0.7 * t["x"] + (z if t["gate"] is None else t["gate"] * z)
    h = normed(y, t["pre_w"], t["pre_c"])
    ((y * torch.tensor(cy)).sum() + (h * torch.tensor(ch)).sum()).backward()
    (y_ref, h_ref, _), _ = zt_ref.residual_norm(a["x"], a["b"], layer, post, a["pre_w"], a["pre_c"], a["post_w"], a["post_c"], a["gate"], scale=0.7)
    assert np.allclose(y_ref, y.detach().numpy(), rtol=1e-12, atol=1e-12) and np.allclose(h_ref, h.detach().numpy(), rtol=1e-12, atol=1e-12)
    got, _ = zt_ref.residual_norm_backward(cy, ch, y_ref, a["b"], layer, post, a["pre_w"], a["post_w"], a["post_c"], a["gate"], scale=0.7)
    names = dict(NAMES, gate="gate_sum" if gate == "channel" else "gate")
    for k, v in t.items():
        if v is not None:
            assert np.allclose(got[names[k]], v.grad.numpy(), rtol=1e-10, atol=1e-10), k


def test_adamw_against_torch():
    r = np.random.default_rng(7)
    n = 200
    param, grads = r.standard_normal(n), r.standard_normal((4, n))
    p = torch.tensor(param, requires_grad=True)
    optimizer = torch.optim.AdamW([p], lr=1e-2, betas=(0.9, 0.95), eps=1e-6, weight_decay=0.1, foreach=False)
    m = v = np.zeros(n)
    for step in range(1, 5):
        p.grad = torch.tensor(0.5 * grads[step - 1])
        optimizer.step()
        (param, m, v, _), _ = zt_ref.adamw(grads[step - 1], param, m, v, 0.5, 1e-2, 0.9, 0.95, 1e-6, 0.1, step)
        assert np.allclose(param, p.detach().numpy(), rtol=1e-10, atol=1e-12)
