"""The vocabulary's operators of include/ze.h from their formulas, in 64 bits (torch, on any device), with bounds on what fp32 arithmetic in
any order may differ by.  Shares no code with the HIP library.

Bounds count roundings.  An fp32 operation is off by at most U32 = 2^-24 of its result, a matrix instruction's sum by 2 U32 (its inner
sums may be cut instead of rounded), v_exp_f32 by 2 U32, a value stored in a type by half its step.  A product over k is a chain of k / 32 matrix
instructions in half precision and k / 4 in fp32, of 32 and 4 products each, which a few more (pieces, splits) are joined to: each of its
roundings is of at most the sum of the terms' magnitudes.
"""
import torch

U32 = 2.0 ** -24
# half a step relative to the value, and half the smallest step, of each type
STORED = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float16: (2.0 ** -11, 2.0 ** -25)}


def stored(value, off, dtype):
    """The bound of a value that is off by `off` and rounded to a type."""
    unit, step = STORED[dtype]
    return off + unit * (value.abs() + off) + step


def _chain(k, dtype):
    return (k / 4 + 4 if dtype == torch.float32 else k / 32 + 32) + 80


def _local(ids, first, rows):
    at = ids.long() - first
    return at, (at >= 0) & (at < rows)


def embedding(ids, table, first=0, scale=1.0):
    """(out, bound) of the lookup."""
    at, here = _local(ids.reshape(-1), first, table.shape[0])
    out = torch.zeros((ids.numel(), table.shape[1]), dtype=torch.float64, device=table.device)
    out[here] = scale * table[at[here]].double()
    return out, stored(out, U32 * out.abs(), table.dtype)


def embedding_backward(ids, dout, rows, first=0, scale=1.0, old=None, dtype=torch.float32):
    """(dtable, bound): sums of c terms take at most c roundings of the magnitudes' sum, the scale one, what is added to one."""
    at, here = _local(ids.reshape(-1), first, rows)
    shape = (rows, dout.shape[-1])
    d = dout.reshape(-1, shape[1]).double()
    out, size = torch.zeros(shape, dtype=torch.float64, device=d.device), torch.zeros(shape, dtype=torch.float64, device=d.device)
    count = torch.zeros(rows, dtype=torch.float64, device=d.device)
    out.index_add_(0, at[here], d[here])
    size.index_add_(0, at[here], d[here].abs())
    count.index_add_(0, at[here], torch.ones_like(at[here], dtype=torch.float64))
    off = U32 * (count[:, None] + 1) * size * abs(scale)
    out = out * scale
    if old is not None:
        out = out + old.double()
        off = off + U32 * (out.abs() + off)
    bound = stored(out, off, dtype)
    if old is not None:
        bound[count == 0] = 0.0
    return out, bound


def _logits(hidden, table, scale):
    """Logits and what each may be off by."""
    h, w = hidden.reshape(-1, hidden.shape[-1]).double(), table.double()
    l = scale * (h @ w.t())
    size = abs(scale) * (h.abs() @ w.abs().t())
    return l, 2 * U32 * _chain(h.shape[1], hidden.dtype) * size + U32 * l.abs()


def vocab_loss(hidden, table, labels, first=0, scale=1.0):
    """(m, lse, target) of this rank's rows and bounds for them; m + log(s) is what m and s say together."""
    labels = labels.reshape(-1)
    n, rows = labels.numel(), table.shape[0]
    absent = labels < 0
    inf = float("inf")
    if rows == 0:
        m = torch.full((n,), -inf, dtype=torch.float64, device=hidden.device)
        return (m, m.clone(), torch.where(absent, 0.0, m)), (torch.zeros_like(m),) * 3
    hidden = torch.where(absent[:, None], torch.zeros_like(hidden.reshape(n, -1)), hidden.reshape(n, -1))
    l, off = _logits(hidden, table, scale)
    m = l.max(1).values
    lse = torch.logsumexp(l, 1)
    p = torch.exp(l - lse[:, None])
    at, here = _local(labels, first, rows)
    target = torch.full_like(m, -inf)
    target_off = torch.zeros_like(m)
    target[here] = l[here, at[here]]
    target_off[here] = off[here, at[here]]
    # each exponential's argument is off by its logit's error, the greatest logit's (taken out again where the two are joined) and two roundings
    lse_off = (p * (off + 4 * U32 * (l - m[:, None]).abs())).sum(1) + (96 + rows / 4096) * U32 + 4 * U32 * (m.abs() + (lse - m).abs())
    m_off = off.max(1).values
    m, lse, target = (torch.where(absent, v, t) for v, t in ((torch.full_like(m, -inf), m), (torch.full_like(m, -inf), lse), (torch.zeros_like(m), target)))
    return (m, lse, target), tuple(torch.where(absent, torch.zeros_like(v), v) for v in (m_off, lse_off, target_off))


def join_loss(stats, labels):
    """(loss, lse) and bounds for them from stats [ranks, 3, tokens]."""
    s = stats.double()
    labels = labels.reshape(-1)
    m = s[:, 0].max(0).values
    parts = torch.where(s[:, 1] > 0, s[:, 0] + torch.log(s[:, 1]), torch.full_like(m, -float("inf")))
    lse = torch.logsumexp(parts, 0)
    target = s[:, 2].max(0).values
    # the largest term counts with one rounding or none, each other with its argument's two and the exponential's
    gap = torch.where(s[:, 1] > 0, (s[:, 0] - m).abs() * torch.exp(parts - lse), torch.zeros_like(m)).sum(0)
    off = U32 * (4 * gap + 8 + s.shape[0] + 4 * (lse - m).abs() + 2 * lse.abs())
    loss = lse - target
    loss_off = off + U32 * torch.where(loss.isfinite(), loss.abs(), torch.zeros_like(loss))
    zero = torch.zeros_like(lse)
    absent = labels < 0
    return tuple(torch.where(absent, zero, v) for v in (loss, lse)), tuple(torch.where(absent, zero, v) for v in (loss_off, off))


def vocab_loss_backward(hidden, table, labels, lse, dloss, first=0, scale=1.0):
    """(dhidden, dtable) and bounds for them: g is off by its probability's error and rounded to the inputs' type before the products."""
    dtype = hidden.dtype
    labels = labels.reshape(-1)
    n, rows = labels.numel(), table.shape[0]
    present = labels >= 0
    h = torch.where(present[:, None], hidden.reshape(n, -1), torch.zeros_like(hidden.reshape(n, -1)))
    lse = torch.where(present, lse.reshape(-1).double(), torch.zeros(n, dtype=torch.float64, device=h.device))
    dloss = torch.where(present, dloss.reshape(-1).double(), torch.zeros(n, dtype=torch.float64, device=h.device))
    l, off = _logits(h, table, scale)
    p = torch.exp(l - lse[:, None])
    p_off = p * torch.expm1(off + 4 * U32 * (l.abs() + lse.abs()[:, None]) + 4 * U32)
    at, here = _local(labels, first, rows)
    hit = torch.zeros_like(p)
    hit[here, at[here]] = 1.0
    g, d = dloss[:, None] * (p - hit), dloss.abs()[:, None]
    most = dloss.abs().max() if n else torch.zeros((), dtype=torch.float64)
    g_off = d * (p_off + 4 * U32 * (p + p_off + hit))
    unit, step = STORED[dtype]
    lift = 2.0 ** 15 if dtype == torch.float16 else 1.0
    g_off = g_off + unit * (g.abs() + g_off) + step * most / lift
    g_off[~present] = 0.0
    g[~present] = 0.0
    w, hd = table.double(), h.double()

    def product(a, a_off, b, k):
        value = scale * (a @ b)
        size = abs(scale) * ((a.abs() + a_off) @ b.abs())
        return value, stored(value, abs(scale) * (a_off @ b.abs()) + 2 * U32 * _chain(k, dtype) * size + 4 * U32 * value.abs(), dtype)

    dhidden, dhidden_off = product(g, g_off, w, rows)
    dtable, dtable_off = product(g.t().contiguous(), g_off.t().contiguous(), hd, n)
    dhidden_off[~present] = 0.0
    return (dhidden, dtable), (dhidden_off, dtable_off)


def vocab_loss_backward_as_stored(hidden, table, labels, lse, dloss, first=0, exact_logits=False):
    """vocab_loss_backward at scale 1 with g / max |dloss| (fp16: times 2^15) rounded to the inputs' type, as the header says that it lies in the workspace, so that
    the bounds hold what is left: roundings of the products, and of g only where it lies so near to the middle between two values of its type that
    its own error decides.  Rounding keeps order, so g as stored lies between its formula less its error, rounded, and plus its error, rounded.  exact_logits: the
    caller has chosen inputs whose products and sums fp32 holds exactly, in any order."""
    dtype = hidden.dtype
    labels = labels.reshape(-1)
    n, rows = labels.numel(), table.shape[0]
    present = labels >= 0
    h = torch.where(present[:, None], hidden.reshape(n, -1), torch.zeros_like(hidden.reshape(n, -1)))
    zero = torch.zeros(n, dtype=torch.float64, device=h.device)
    lse, dloss = (torch.where(present, v.reshape(-1).double(), zero) for v in (lse, dloss))
    l, off = _logits(h, table, 1.0)
    if exact_logits:
        off = torch.zeros_like(off)
    p = torch.exp(l - lse[:, None])
    off = p * torch.expm1(off + 4 * U32 * (l.abs() + lse.abs()[:, None]) + 4 * U32)
    at, here = _local(labels, first, rows)
    most, lift = dloss.abs().max(), 2.0 ** 15 if dtype == torch.float16 else 1.0
    unit = (dloss / most * lift)[:, None]
    off = unit.abs() * (off + 4 * U32 * (p + off))
    g = unit * p
    g[here, at[here]] -= unit[here, 0]
    off[here, at[here]] += 4 * U32 * unit[here, 0].abs()
    low, high = (g - off).to(dtype).double(), (g + off).to(dtype).double()
    g, off = (low + high) / 2, (high - low) / 2
    g[~present], off[~present] = 0.0, 0.0
    factor = most / lift

    def product(a, a_off, b, k):
        value = factor * (a @ b)
        size = factor * ((a.abs() + a_off) @ b.abs())
        return value, stored(value, factor * (a_off @ b.abs()) + 2 * U32 * _chain(k, dtype) * size + 4 * U32 * value.abs(), dtype)

    dhidden, dhidden_off = product(g, off, table.double(), rows)
    dtable, dtable_off = product(g.t().contiguous(), off.t().contiguous(), h.double(), n)
    return (dhidden, dtable), (dhidden_off, dtable_off)
