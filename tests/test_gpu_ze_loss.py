"""The softmax cross entropy over a part of the vocabulary (include/ze.h) and its gradients on the GPU against their formulas in 64 bits, within
bounds that oracle/ze_ref.py derives."""
import pytest
import torch

from oracle import ze_ref
from paper_2409_02423_amd import ze

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF = float("inf")


def _close(got, want, bound):
    got = got.double().reshape(want.shape)
    same = got == want               # infinities
    over = torch.where(same, torch.zeros_like(want), (got - want).abs() - bound)
    assert not got.isnan().any()
    assert not over.numel() or over.max() <= 0, "off by %g more than its bound" % over.max()


def _inputs(tokens, rows, cols, dtype, seed, first=0, ranks=1, absent=0.2, ids=torch.int64, logits=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    hidden = torch.randn((tokens, cols), generator=g, device="cuda").to(dtype)
    table = (torch.randn((rows, cols), generator=g, device="cuda") * logits / cols ** 0.5).to(dtype)
    labels = torch.randint(0, max(1, rows * ranks), (tokens,), generator=g, device="cuda")
    labels[torch.rand(tokens, generator=g, device="cuda") < absent] = -100
    dloss = (0.2 + torch.rand(tokens, generator=g, device="cuda")) / tokens
    return hidden, table, labels.to(ids), dloss


def _check_stats(stats, hidden, table, labels, first, scale):
    (m, lse, target), (m_off, lse_off, target_off) = ze_ref.vocab_loss(hidden, table, labels, first, scale)
    got = stats.double()
    _close(got[0], m, m_off)
    _close(torch.where(got[1] > 0, got[0] + torch.log(got[1]), torch.full_like(m, -INF)), lse, lse_off)
    _close(got[2], target, target_off)


SHAPES = [(1, 1, 1), (1, 5, 7), (2, 300, 64), (64, 64, 64), (65, 257, 100), (300, 513, 200), (129, 1000, 333), (17, 2000, 1024), (256, 256, 512), (257, 255, 65)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("tokens, rows, cols", SHAPES)
def test_loss_and_gradients(dtype, tokens, rows, cols):
    for first, ranks, scale, ids in ((0, 1, 1.0, torch.int64), (rows, 3, 0.4, torch.int32)):
        hidden, table, labels, dloss = _inputs(tokens, rows, cols, TYPES[dtype], tokens + rows + cols, first, ranks, ids=ids)
        stats = ze.ze_vocab_loss(hidden, table, labels, first=first, scale=scale)
        _check_stats(stats, hidden, table, labels, first, scale)
        loss, lse = ze.ze_join_loss(stats, labels)
        (want_loss, want_lse), (loss_off, lse_off) = ze_ref.join_loss(stats[None], labels)
        _close(loss, want_loss, loss_off)
        _close(lse, want_lse, lse_off)
        got = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, first=first, scale=scale)
        for a, b, c in zip(got, *ze_ref.vocab_loss_backward(hidden, table, labels, lse, dloss, first, scale)):
            _close(a, b, c)


# sizes that the large and the medium tiles take, with edges in all three directions
LARGE = [(2048, 6200, 6208, "bf16"), (2047, 6201, 4106, "f16"), (1600, 2100, 1030, "f32"), (1700, 2049, 1030, "bf16")]


@pytest.mark.parametrize("tokens, rows, cols, dtype", LARGE)
def test_large_tiles(tokens, rows, cols, dtype):
    hidden, table, labels, dloss = _inputs(tokens, rows, cols, TYPES[dtype], 5)
    stats = ze.ze_vocab_loss(hidden, table, labels)
    _check_stats(stats, hidden, table, labels, 0, 1.0)
    lse = ze.ze_join_loss(stats, labels)[1]
    got = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss)
    for a, b, c in zip(got, *ze_ref.vocab_loss_backward(hidden, table, labels, lse, dloss)):
        _close(a, b, c)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens, rows, cols", [(4096, 4200, 40), (4100, 4096, 64), (2300, 9000, 130), (4096, 4500, 192), (2048, 5000, 254)])
def test_large_tiles_of_short_rows(tokens, rows, cols, dtype):
    """No whole step, one, two with an end, three, and three with one."""
    hidden, table, labels, dloss = _inputs(tokens, rows, cols, TYPES[dtype], 6, absent=0.4)
    stats = ze.ze_vocab_loss(hidden, table, labels)
    _check_stats(stats, hidden, table, labels, 0, 1.0)
    lse = ze.ze_join_loss(stats, labels)[1]
    got = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss)
    for a, b, c in zip(got, *ze_ref.vocab_loss_backward(hidden, table, labels, lse, dloss)):
        _close(a, b, c)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("tokens, rows, cols, piece", [(70, 1000, 136, 256), (70, 1000, 136, 1), (70, 1000, 136, 999), (70, 1000, 136, 1 << 40), (5, 2600, 64, 512),
                                                      (300, 700, 4096, 256)])
def test_gradients_in_pieces(dtype, tokens, rows, cols, piece):
    """However the vocabulary is cut, within the same bounds; and the same each time."""
    hidden, table, labels, dloss = _inputs(tokens, rows, cols, TYPES[dtype], 8)
    lse = ze.ze_join_loss(ze.ze_vocab_loss(hidden, table, labels), labels)[1]
    want, bound = ze_ref.vocab_loss_backward(hidden, table, labels, lse, dloss)
    got = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, piece=piece)
    for a, b, c in zip(got, want, bound):
        _close(a, b, c)
    for a, b in zip(got, ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, piece=piece)):
        assert torch.equal(a, b)


def test_shards_of_a_vocabulary_together():
    """Three ranks' statistics give the whole vocabulary's loss, and their gradients its gradients."""
    hidden, table, labels, dloss = _inputs(90, 900, 256, torch.float32, 21)
    whole = ze.ze_join_loss(ze.ze_vocab_loss(hidden, table, labels, scale=0.7), labels)
    cuts = ((0, 1), (1, 500), (500, 900))
    stats = torch.empty((3, 3, 90), device="cuda")
    for r, (a, b) in enumerate(cuts):
        ze.ze_vocab_loss(hidden, table[a:b], labels, first=a, scale=0.7, d_stats=stats[r])
    loss, lse = ze.ze_join_loss(stats, labels)
    for got, want, off in zip((loss, lse), *ze_ref.join_loss(stats, labels)):
        _close(got, want, off)
    # each of the two is within its bound of the formula
    (_, exact, _), (_, off, _) = ze_ref.vocab_loss(hidden, table, labels, 0, 0.7)
    present = labels >= 0
    for got in (lse, whole[1]):
        _close(got[present], exact[present], off[present] * 2 + 2.0 ** -20)
    want, bound = ze_ref.vocab_loss_backward(hidden, table, labels, lse, dloss, 0, 0.7)
    dhidden, off = 0.0, 0.0
    for a, b in cuts:
        dh, dw = ze.ze_vocab_loss_backward(hidden, table[a:b], labels, lse, dloss, first=a, scale=0.7)
        dhidden = dhidden + dh.double()
        off = off + ze_ref.vocab_loss_backward(hidden, table[a:b], labels, lse, dloss, a, 0.7)[1][0]
        _close(dw, want[1][a:b], bound[1][a:b])
    _close(dhidden, want[0], off)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_tokens_without_a_label_are_not_read(dtype):
    """Hidden states, lse and dloss of padding may hold anything; its results are zeros, whatever lay there."""
    t = TYPES[dtype]
    for tokens, absent in ((70, 0.5), (70, 1.1), (300, 0.9)):
        hidden, table, labels, dloss = _inputs(tokens, 333, 192, t, 31, absent=absent)
        gone = labels < 0
        clean = hidden.clone()
        hidden[gone] = float("nan")
        stats = ze.ze_vocab_loss(hidden, table, labels)
        _check_stats(stats, clean, table, labels, 0, 1.0)
        loss, lse = ze.ze_join_loss(stats, labels)
        assert (loss[gone] == 0).all() and (lse[gone] == 0).all()
        lse[gone], dloss[gone] = float("nan"), float("inf")
        out = (torch.full_like(hidden, float("nan")), torch.full_like(table, float("nan")))
        got = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, d_dhidden=out[0], d_dtable=out[1])
        assert (got[0][gone] == 0).all()
        for a, b, c in zip(got, *ze_ref.vocab_loss_backward(clean, table, labels, lse, dloss)):
            _close(a, b, c)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_slices_at_odd_places(dtype):
    """Operands and outputs that start anywhere and are apart by a stride; what lies between the outputs' rows stays as it was."""
    t = TYPES[dtype]
    for tokens, rows, cols in ((40, 90, 64), (33, 70, 65), (20, 300, 129)):
        h, w, labels, dloss = _inputs(tokens, rows, cols, t, 41)
        for pad, start in ((0, 1), (8, 0), (3, 2)):
            def spread(v):
                flat = torch.full((start + v.shape[0] * (cols + pad),), 7.0, dtype=t, device="cuda")
                view = flat[start:].view(v.shape[0], cols + pad)[:, :cols]
                view.copy_(v)
                return flat, view
            (_, hidden), (_, table), (all_dh, dh), (all_dw, dw) = spread(h), spread(w), spread(h), spread(w)
            stats = ze.ze_vocab_loss(hidden, table, labels)
            assert torch.equal(stats, ze.ze_vocab_loss(h, w, labels))
            lse = ze.ze_join_loss(stats, labels)[1]
            ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, d_dhidden=dh, d_dtable=dw)
            for a, b, c in zip((dh, dw), *ze_ref.vocab_loss_backward(h, w, labels, lse, dloss)):
                _close(a, b, c)
            dh.fill_(7.0)
            dw.fill_(7.0)
            assert (all_dh == 7.0).all() and (all_dw == 7.0).all()


def test_one_output_alone():
    hidden, table, labels, dloss = _inputs(60, 200, 128, torch.bfloat16, 51)
    lse = ze.ze_join_loss(ze.ze_vocab_loss(hidden, table, labels), labels)[1]
    both = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss)
    first = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, want_table=False)
    second = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, want_hidden=False)
    assert first[1] is None and second[0] is None and torch.equal(first[0], both[0]) and torch.equal(second[1], both[1])


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_losses_with_weights_that_lie_far_apart(dtype):
    """Gradients of losses between 2^-20 and 2^3, and of exactly nothing: each row within its bound."""
    hidden, table, labels, _ = _inputs(50, 120, 96, TYPES[dtype], 61, absent=0.0)
    lse = ze.ze_join_loss(ze.ze_vocab_loss(hidden, table, labels), labels)[1]
    for dloss in (2.0 ** (torch.arange(50, device="cuda") % 24 - 20).float(), -torch.ones(50, device="cuda"), torch.zeros(50, device="cuda"),
                  torch.where(torch.arange(50, device="cuda") == 7, 1e-3, 0.0)):
        got = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss)
        for a, b, c in zip(got, *ze_ref.vocab_loss_backward(hidden, table, labels, lse, dloss)):
            _close(a, b, c)


def test_logits_far_apart_and_infinite():
    """Exponentials never overflow; -inf logits count as nothing, NaN and +inf make their token's loss not a number and no other's."""
    hidden = torch.zeros((6, 64), device="cuda")
    table = torch.zeros((200, 64), device="cuda")
    table[:, 0] = torch.arange(200, device="cuda")
    hidden[0, 0], hidden[1, 0] = 1e6, -1e30
    table[:, 1] = -1.0
    table[5, 1] = 1.0
    hidden[2, 1] = INF                 # logits -inf, but +inf at 5
    hidden[3, 2] = float("nan")
    table[:, 3] = 1.0
    hidden[4, 3] = -INF                # all logits -inf (0 * -inf is NaN: its other factors are not zero)
    labels = torch.tensor([199, 0, 1, 2, 3, 4], device="cuda")
    loss, lse = ze.ze_join_loss(ze.ze_vocab_loss(hidden, table, labels), labels)
    assert float(loss[0]) == 0.0 and float(loss[1]) == 0.0
    assert loss[2].isnan() and loss[3].isnan() and not loss[4] < 1e30
    assert abs(float(loss[5]) - 5.298317) < 1e-5
    d = torch.ones(6, device="cuda")
    dh, _ = ze.ze_vocab_loss_backward(hidden, table, labels, lse, d)
    assert dh[3].isnan().any() and dh[0].isfinite().all() and dh[5].isfinite().all()


def test_only_minus_infinity_somewhere():
    """A shard whose logits are all -inf adds nothing to the sum over the ranks."""
    hidden = torch.full((3, 1), INF, device="cuda")
    table = torch.full((70, 1), -1.0, device="cuda")
    labels = torch.tensor([0, 100, 2], device="cuda")
    stats = ze.ze_vocab_loss(hidden, table, labels)
    assert (stats[0] == -INF).all() and (stats[1] == 0).all() and stats[2].tolist() == [-INF] * 3
    other = torch.tensor([[1.0] * 3, [2.0] * 3, [-INF, 0.5, -INF]], device="cuda")
    loss, lse = ze.ze_join_loss(torch.stack([stats, other]), labels)
    assert (lse - (1.0 + 0.6931472)).abs().max() < 1e-6
    assert loss[0] == INF and abs(float(loss[1]) - 1.1931472) < 1e-6 and loss[2] == INF


def test_a_label_that_no_rank_has():
    hidden, table, _, dloss = _inputs(4, 50, 64, torch.bfloat16, 71, absent=0.0)
    labels = torch.tensor([3, 50, 1 << 40, 49], device="cuda")
    loss, lse = ze.ze_join_loss(ze.ze_vocab_loss(hidden, table, labels), labels)
    assert loss[1] == INF and loss[2] == INF and loss[0] < 20 and loss[3] < 20
    got = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss)
    for a, b, c in zip(got, *ze_ref.vocab_loss_backward(hidden, table, labels, lse, dloss)):
        _close(a, b, c)


def test_gradients_against_differences():
    """The mean loss in fp32, moved along the gradient's own direction: what it changes by is the gradient's square to first order."""
    hidden, table, labels, _ = _inputs(12, 40, 24, torch.float32, 81)
    present = labels >= 0
    dloss = torch.where(present, 1.0 / present.sum(), torch.zeros(12, device="cuda"))

    def value(h, w):
        # the formula in 64 bits, at the places where the gradients are taken
        l = h.double() @ w.double().t()
        each = torch.logsumexp(l, 1) - l.gather(1, labels.clamp_min(0)[:, None])[:, 0]
        return float((each * dloss.double()).sum())

    lse = ze.ze_join_loss(ze.ze_vocab_loss(hidden, table, labels), labels)[1]
    dh, dw = (d.double() for d in ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss))
    for h, w, want in ((dh, torch.zeros_like(dw), dh.square().sum()), (torch.zeros_like(dh), dw, dw.square().sum())):
        eps = 1e-4
        got = (value(hidden.double() + eps * h, table.double() + eps * w) - value(hidden.double() - eps * h, table.double() - eps * w)) / (2 * eps)
        # third derivatives of the loss are below 1 in a direction of length |logits' change| < 10: 10^3 eps^2 / 6; the gradients are off by 1e-5 of them
        assert abs(got - float(want)) < 1e-5 + 1e-4 * float(want)


def _form(hidden, table, labels):
    types = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    return ze.Form(labels.numel(), table.shape[0], table.shape[1], 0, types[hidden.dtype], types[hidden.dtype], ze.ZE_I64, 1.0)


@pytest.mark.parametrize("tokens, rows, cols, dtype, absent", [
    (1700, 2049, 1030, "bf16", 0.2), (1700, 2049, 1030, "bf16", 0.9), (300, 9000, 520, "f16", 0.5), (2047, 3001, 2050, "f16", 0.5), (130, 5000, 260, "bf16", 0.0),
    (70, 3000, 64, "bf16", 0.3), (65, 4000, 200, "f32", 0.0), (513, 1200, 1025, "f32", 0.5), (1, 3000, 77, "bf16", 0.0), (2100, 2600, 4104, "bf16", 0.1)])
def test_a_workspace_as_large_as_it_has_to_be(tokens, rows, cols, dtype, absent):
    """What lies behind a workspace of just the bytes that a call asks for stays as it was."""
    hidden, table, labels, dloss = _inputs(tokens, rows, cols, TYPES[dtype], 13, absent=absent)
    L, f, behind = ze.lib(), _form(hidden, table, labels), 96 << 20
    stats, lse = torch.empty((3, tokens), device="cuda"), None
    dh, dw = torch.empty_like(hidden), torch.empty_like(table)
    at = (hidden.data_ptr(), table.data_ptr(), labels.data_ptr())
    for piece in (None, 0, 512):
        size = L.ze_loss_work_bytes(f, *at[:2]) if piece is None else L.ze_loss_backward_work_bytes(f, *at[:2], piece)
        work = torch.full((size + behind,), 0x5A, dtype=torch.uint8, device="cuda")
        if piece is None:
            assert L.ze_vocab_loss(f, *at, stats.data_ptr(), work.data_ptr(), size, torch.cuda.current_stream().cuda_stream) == 0
            lse = ze.ze_join_loss(stats, labels)[1]
        else:
            assert L.ze_vocab_loss_backward(f, *at, lse.data_ptr(), dloss.data_ptr(), dh.data_ptr(), dw.data_ptr(), piece, work.data_ptr(), size,
                                            torch.cuda.current_stream().cuda_stream) == 0
            for a, b, c in zip((dh, dw), *ze_ref.vocab_loss_backward(hidden, table, labels, lse, dloss)):
                _close(a, b, c)
        assert (work[size:] == 0x5A).all()


def test_nothing_to_do():
    hidden, table, labels, dloss = _inputs(3, 20, 32, torch.bfloat16, 91, absent=0.0)
    none = labels[:0]
    assert ze.ze_vocab_loss(hidden[:0], table, none).shape == (3, 0)
    assert ze.ze_join_loss(torch.empty((2, 3, 0), device="cuda"), none)[0].shape == (0,)
    dh, dw = ze.ze_vocab_loss_backward(hidden[:0], table, none, dloss[:0], dloss[:0], d_dtable=torch.full_like(table, 7.0))
    assert dh.shape == (0, 32) and (dw == 0).all()
    stats = ze.ze_vocab_loss(hidden, table[:0], labels)
    assert (stats[0] == -INF).all() and (stats[1] == 0).all() and (stats[2] == -INF).all()
    dh, dw = ze.ze_vocab_loss_backward(hidden, table[:0], labels, dloss, dloss, d_dhidden=torch.full_like(hidden, 7.0))
    assert (dh == 0).all() and dw.shape == (0, 32)
    gone = torch.full_like(labels, -1)
    dh, dw = ze.ze_vocab_loss_backward(hidden, table, gone, dloss, dloss)
    assert (dh == 0).all() and (dw == 0).all()
    stats = ze.ze_vocab_loss(hidden.view(3, 1, 32), table, labels.view(3, 1))
    assert ze.ze_join_loss(stats, labels.view(3, 1))[0].shape == (3, 1)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_rows_of_the_matrix_that_overlap(dtype):
    """An input's rows may overlap.  -inf where the last row alone has it, and the rows behind it would, were there any: the columns in which they would
    stay finite."""
    t, cols, stride = TYPES[dtype], 128, 64
    for rows in (65, 301):
        hidden, _, labels, dloss = _inputs(70, rows, cols, t, 71)
        flat = (torch.randn((rows - 1) * stride + cols, generator=torch.Generator(device="cuda").manual_seed(72), device="cuda") / 8).to(t)
        flat[-1] = -INF
        hidden[:, -1] = 1.0          # the last row's logits are -inf, and no token's label
        labels[labels == rows - 1] = 0
        table = flat.as_strided((rows, cols), (stride, 1))
        clean = table.clone()
        stats = ze.ze_vocab_loss(hidden, table, labels)
        assert torch.equal(stats, ze.ze_vocab_loss(hidden, clean, labels))
        lse = ze.ze_join_loss(stats, labels)[1]
        got, want = (ze.ze_vocab_loss_backward(hidden, m, labels, lse, dloss) for m in (table, clean))
        assert torch.equal(got[1], want[1]) and got[0][:, :-1].isfinite().all()
        assert torch.equal(got[0][:, :-1], want[0][:, :-1])


def test_pieces_of_more_rows_than_an_argument_holds():
    """As many as there are: 2^64 + 256 is not 256, nor 2^64 the library's choice."""
    hidden, table, labels, dloss = _inputs(70, 5000, 64, torch.float32, 8)
    lse = ze.ze_join_loss(ze.ze_vocab_loss(hidden, table, labels), labels)[1]
    whole = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, piece=5000)
    assert not torch.equal(ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, piece=256)[0], whole[0])   # (another order of sums)
    for piece in (ze.ZE_MAX_ROWS, 1 << 64, (1 << 64) + 256):
        for got, want in zip(ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, piece=piece), whole):
            assert torch.equal(got, want)


def _whole_inputs(tokens, rows, cols, dtype, seed, absent=0.2):
    """Hidden states of -1 and 1 and a matrix of 0 and two values that are a power of two from 0: logits of a spread of about 1, which fp32 holds exactly."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    sign = lambda *shape: torch.randint(0, 2, shape, generator=g, device="cuda") * 2 - 1
    hidden = sign(tokens, cols).to(dtype)
    step = 2.0 ** -((cols - 1).bit_length() // 2)
    table = (sign(rows, cols) * torch.randint(0, 3, (rows, cols), generator=g, device="cuda").clamp_max(1) * step).to(dtype)
    labels = torch.randint(0, rows, (tokens,), generator=g, device="cuda")
    labels[torch.rand(tokens, generator=g, device="cuda") < absent] = -100
    labels[-1] = rows - 1                                     # the last row of all is one of those that count
    return hidden, table, labels, (0.2 + torch.rand(tokens, generator=g, device="cuda")) / tokens


def _check_whole(hidden, table, labels, dloss, piece=0, **out):
    stats = ze.ze_vocab_loss(hidden, table, labels)
    _check_stats(stats, hidden, table, labels, 0, 1.0)
    lse = ze.ze_join_loss(stats, labels)[1]
    got = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, piece=piece, **out)
    for a, b, c in zip(got, *ze_ref.vocab_loss_backward_as_stored(hidden, table, labels, lse, dloss, exact_logits=True)):
        _close(a, b, c)
    for a, b in zip(got, ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, piece=piece)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens, rows, cols", [(90, 700, 128), (600, 3001, 520), (1030, 5000, 1024), (2048, 8192, 2048), (2047, 6201, 4106), (1024, 32003, 2048), (4100, 4096, 64)])
def test_gradients_are_off_by_the_rounding_of_g_alone(dtype, tokens, rows, cols):
    """All shapes of tiles in half precision: with g rounded as it is stored, what is left are roundings of fp32 sums and of the result, so that one step of a product
    too few would show."""
    _check_whole(*_whole_inputs(tokens, rows, cols, TYPES[dtype], 3))


# A matrix that has to be copied comes in pieces of 64 MiB, forward and backward: of odd width, at an odd place, of rows that overlap
@pytest.mark.parametrize("tokens, rows, cols, dtype, start", [(130, 50003, 2049, "bf16", 0), (600, 50003, 2049, "f16", 0), (200, 33000, 1026, "f16", 1), (5, 70001, 1023, "bf16", 0)])
def test_a_copied_matrix_in_pieces(tokens, rows, cols, dtype, start):
    hidden, close, labels, dloss = _whole_inputs(tokens, rows, cols, TYPES[dtype], 17)
    table = torch.empty(rows * cols + start, dtype=TYPES[dtype], device="cuda")[start:].view(rows, cols)
    table.copy_(close)
    labels[:4] = torch.tensor([0, rows // 2, rows - 2, rows // 3], device="cuda")
    _check_whole(hidden, table, labels, dloss)


def test_a_copied_matrix_of_rows_that_overlap_in_pieces():
    hidden, _, labels, dloss = _whole_inputs(70, 20001, 1000, torch.float32, 19)
    flat = torch.randint(-1, 2, (20000 * 500 + 1000,), generator=torch.Generator(device="cuda").manual_seed(20), device="cuda") / 32.0
    _check_whole(hidden, flat.as_strided((20001, 1000), (500, 1)), labels, dloss)


@pytest.mark.parametrize("absent", (0.1, 0.9))
@pytest.mark.parametrize("tokens, rows, cols, dtype, piece", [
    (2048, 16500, 4096, "bf16", 8192), (1021, 33000, 4098, "f16", 16384),     # large tiles of the hidden states' gradient: the last piece has two steps, and four
    (2048, 8300, 2048, "bf16", 4096), (2047, 8200, 2050, "f16", 4096),        # half ones, three steps under way
    (3000, 8300, 1024, "bf16", 4096), (1000, 3000, 4096, "f16", 1024),
    (300, 4200, 2048, "bf16", 2048), (300, 9000, 512, "f16", 1024), (300, 1100, 2048, "f32", 512)])
def test_pieces_whose_steps_are_shared_out(tokens, rows, cols, dtype, piece, absent):
    """Sums that several workgroups keep from piece to piece, the last piece with fewer steps than there are workgroups for them."""
    _check_whole(*_whole_inputs(tokens, rows, cols, TYPES[dtype], 23, absent), piece=piece)


def test_a_large_vocabulary_in_the_librarys_pieces():
    """Two pieces, five shares of each."""
    _check_whole(*_whole_inputs(4096, 50257, 768, torch.bfloat16, 29))


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("tokens, rows, cols, piece", [(70, 300, 65, 0), (500, 2000, 256, 512), (2100, 4200, 1024, 0), (40, 0, 64, 0)])
def test_gradients_in_the_hidden_states_place(dtype, tokens, rows, cols, piece):
    """Where many tokens have no label: their rows become zeros while the others' are read, which lie between them."""
    hidden, table, labels, dloss = _inputs(tokens, rows, cols, TYPES[dtype], 43, absent=0.5)
    hidden[labels < 0] = float("nan")
    lse = ze.ze_join_loss(ze.ze_vocab_loss(hidden, table, labels), labels)[1]
    want = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss, piece=piece)
    wide = torch.full((tokens, cols + 7), 7.0, dtype=TYPES[dtype], device="cuda")
    for place in (hidden.clone(), wide[:, 3:3 + cols].copy_(hidden)):
        got = ze.ze_vocab_loss_backward(place, table, labels, lse, dloss, d_dhidden=place, piece=piece)
        assert got[0] is place and torch.equal(place, want[0]) and torch.equal(got[1], want[1])
        assert (place[labels < 0] == 0).all()
    wide[:, 3:3 + cols] = 7.0
    assert (wide == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens, rows, cols", [(9, 700, 130), (500, 3000, 1026), (1700, 2049, 1030), (2047, 6201, 4106)])
def test_a_matrix_of_one_piece_gives_the_same_wherever_it_lies(dtype, tokens, rows, cols):
    """Read where it lies, or copied from an odd place: up to 64 MiB the same bits, of the statistics and of both gradients."""
    hidden, table, labels, dloss = _inputs(tokens, rows, cols, TYPES[dtype], 47)
    apart = []
    for t in (hidden, table):
        apart.append(torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape).copy_(t))
    stats = ze.ze_vocab_loss(hidden, table, labels)
    lse = ze.ze_join_loss(stats, labels)[1]
    want = ze.ze_vocab_loss_backward(hidden, table, labels, lse, dloss)
    for h, w in ((hidden, apart[1]), (apart[0], table), tuple(apart)):
        assert torch.equal(ze.ze_vocab_loss(h, w, labels), stats)
        for a, b in zip(ze.ze_vocab_loss_backward(h, w, labels, lse, dloss), want):
            assert torch.equal(a, b)
