"""The training-step operators of include/zt.h from their formulas, in 64 bits (numpy), with bounds on what fp32 arithmetic in any order
may differ by.  Shares no code with the HIP library.

A bound is `ROUNDINGS` unit roundoffs of fp32 times the sum of the magnitudes of all terms that a value is made of, and one rounding
to the stored type.  A row or column is added up by lanes that take at most a few dozen terms one after the other, then in a tree: a
sum's error is far below ROUNDINGS times that of one rounding of its terms' magnitudes.
"""
import numpy as np

U32 = 2.0 ** -24
ROUNDINGS = 128
# unit roundoff and half the smallest step of each type
STORED = {"f32": (2.0 ** -24, 2.0 ** -150), "bf16": (2.0 ** -8, 2.0 ** -134), "f16": (2.0 ** -11, 2.0 ** -25)}


def _units(v, layer, eps):
    mean = v.mean(1, keepdims=True) if layer else np.zeros((v.shape[0], 1))
    r = 1.0 / np.sqrt(((v - mean) ** 2).mean(1, keepdims=True) + eps)
    return (v - mean) * r, mean, r


def _bound(exact, magnitude, dtype):
    unit, step = STORED[dtype]
    return unit * np.abs(exact) + step + ROUNDINGS * U32 * magnitude


def residual_norm(x, b, layer, post, pre_w=None, pre_c=None, post_w=None, post_c=None, gate=None, scale=1.0, eps=1e-5, dtype="f32"):
    """(y, h, stats) and bounds for them; float64 arrays [rows, cols]; weights, biases and a channel gate [cols]."""
    rows, cols = x.shape
    z = np.zeros_like(x) if b is None else b
    z_mag = np.abs(z)
    stats = np.zeros((rows, 4))
    stats_bound = np.zeros((rows, 4))
    w1, c1 = (1.0 if post_w is None else post_w), (0.0 if post_c is None else post_c)
    if post:
        u, mean, r = _units(b, layer, eps)
        z = u * w1 + c1
        z_mag = (np.abs(b) + np.abs(b).mean(1, keepdims=True)) * r * np.abs(w1) + np.abs(c1)
        stats[:, 0:1], stats[:, 1:2] = mean, r
        stats_bound[:, 0:1] = ROUNDINGS * U32 * np.abs(b).mean(1, keepdims=True)
        # the squares' sum is of values that are off by the mean's error and one rounding each
        stats_bound[:, 1:2] = ROUNDINGS * U32 * r * (1 + np.abs(b).mean(1, keepdims=True) * r)
    g = 1.0 if gate is None else gate
    y = scale * x + g * z
    y_mag = np.abs(scale * x) + np.abs(g) * z_mag
    w, c = (1.0 if pre_w is None else pre_w), (0.0 if pre_c is None else pre_c)
    u, mean, r = _units(y, layer, eps)
    h = u * w + c
    wide = y_mag.mean(1, keepdims=True)
    h_mag = (y_mag + np.abs(y) + wide + np.abs(u) * wide) * r * np.abs(w) + np.abs(u * w) + np.abs(c)
    stats[:, 2:3], stats[:, 3:4] = mean, r
    stats_bound[:, 2:3] = ROUNDINGS * U32 * wide
    stats_bound[:, 3:4] = ROUNDINGS * U32 * r * (1 + wide * r)
    if not layer:
        stats_bound[:, 0] = stats_bound[:, 2] = 0.0
    return (y, h, stats), (_bound(y, y_mag, dtype), _bound(h, h_mag, dtype), stats_bound)


def residual_norm_backward(dy, dh, y, b, layer, post, pre_w=None, post_w=None, post_c=None, gate=None, scale=1.0, eps=1e-5, dtype="f32"):
    """The gradients as a dict (a gate's for each element and, "gate_sum", for each channel) and bounds for them."""
    rows, cols = dh.shape
    out, mag = {}, {}

    def through(g, g_mag, v, weight):
        """Gradient of the normed values from that of weight * unit + bias; and of weight and bias."""
        u, mean, r = _units(v, layer, eps)
        u_mag = (np.abs(v) + np.abs(mean)) * r
        t, t_mag = g * weight, g_mag * np.abs(weight)
        d = t - u * (t * u).mean(1, keepdims=True)
        d_mag = t_mag + u_mag * (t_mag * u_mag).mean(1, keepdims=True)
        if layer:
            d = d - t.mean(1, keepdims=True)
            d_mag = d_mag + t_mag.mean(1, keepdims=True)
        return r * d, r * d_mag, (g * u).sum(0), (g_mag * u_mag).sum(0), g.sum(0), g_mag.sum(0), u, u_mag

    d, d_mag, out["pre_weight"], mag["pre_weight"], out["pre_bias"], mag["pre_bias"], _, _ = through(dh, np.abs(dh), y, 1.0 if pre_w is None else pre_w)
    if dy is not None:
        d, d_mag = d + dy, d_mag + np.abs(dy)
    out["x"], mag["x"] = scale * d, np.abs(scale) * d_mag
    if b is not None:
        z, z_mag = b, np.abs(b)
        w1, c1 = (1.0 if post_w is None else post_w), (0.0 if post_c is None else post_c)
        if post:
            u, mean, r = _units(b, layer, eps)
            z, z_mag = u * w1 + c1, (np.abs(b) + np.abs(mean)) * r * np.abs(w1) + np.abs(c1)
        if gate is not None:
            out["gate"], mag["gate"] = d * z, d_mag * z_mag
            out["gate_sum"], mag["gate_sum"] = (d * z).sum(0), (d_mag * z_mag).sum(0)
            d, d_mag = d * gate, d_mag * np.abs(gate)
        if post:
            d, d_mag, out["post_weight"], mag["post_weight"], out["post_bias"], mag["post_bias"], _, _ = through(d, d_mag, b, w1)
        out["b"], mag["b"] = d, d_mag
    stored = {k: dtype if k in ("x", "b", "gate") else "f32" for k in out}
    return out, {k: _bound(out[k], mag[k], stored[k]) for k in out}


def clip_factor(norm, scale, max_norm):
    return scale if norm <= max_norm else scale * (max_norm / norm)


def adamw(grad, param, m, v, factor, lr, beta1, beta2, eps, weight_decay, step, half="f32"):
    """(param, m, v, half_param) after one step and bounds for them."""
    g = factor * grad
    m1, v1 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    m_off = 8 * U32 * (np.abs(beta1 * m) + np.abs((1 - beta1) * g)) + 2.0 ** -149
    v_off = 16 * U32 * v1 + 2.0 ** -148
    c1, c2 = 1.0 / (1 - beta1 ** step), 1.0 / (1 - beta2 ** step)
    root = np.sqrt(v1 * c2) + eps
    update = m1 * c1 / root + weight_decay * param
    p1 = param - lr * update
    # a second moment that is off by v_off moves its root by at most v_off c2 / root, or by the root of it where it is all there is
    root_off = np.minimum(v_off * c2 / root, np.sqrt(v_off * c2)) + 8 * U32 * root
    p_off = lr * (m_off * c1 / root + np.abs(m1) * c1 * root_off / root ** 2 + 16 * U32 * (np.abs(m1 * c1 / root) + np.abs(weight_decay * param)))
    p_off = p_off + U32 * 2 * np.abs(p1) + 4 * U32 * np.abs(lr * update) + 2.0 ** -149
    unit, tiny = STORED[half]
    return (p1, m1, v1, p1), (p_off, m_off, v_off, p_off + (np.abs(p1) + p_off) * unit + tiny)
