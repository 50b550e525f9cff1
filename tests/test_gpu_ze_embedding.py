"""The embedding and its gradient (include/ze.h) on the GPU against their formulas in 64 bits, within bounds that oracle/ze_ref.py derives."""
import pytest
import torch

from oracle import ze_ref
from paper_2409_02423_amd import ze

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ids(n, low, high, g, dtype=torch.int64):
    return torch.randint(low, high, (n,), generator=g, device="cuda").to(dtype)


def _close(got, want, bound):
    got = got.double().reshape(want.shape)
    assert got.isfinite().all()
    over = (got - want).abs() - bound
    assert not over.numel() or over.max() <= 0, "off by %g more than its bound" % over.max()


SHAPES = [(1, 1, 1), (1, 5, 7), (4, 300, 64), (5, 3, 8), (65, 257, 100), (300, 513, 1025), (7, 50, 4099), (1000, 40, 72), (33, 9, 8192), (2, 4, 65536)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("tokens, rows, cols", SHAPES)
def test_lookup(dtype, tokens, rows, cols):
    t, g = TYPES[dtype], _generator(tokens + rows + cols)
    table = torch.randn((rows, cols), generator=g, device="cuda").to(t)
    for first, scale, ids in ((0, 1.0, torch.int64), (11, 0.3, torch.int32)):
        at = _ids(tokens, first - 2, first + rows + 2, g, ids)       # some of them of other ranks, or negative
        _close(ze.ze_embedding(at, table, first=first, scale=scale), *ze_ref.embedding(at, table, first, scale))


def test_lookup_without_a_scale_is_a_copy_with_every_value():
    table = torch.arange(1 << 16, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(256, 256)
    table = torch.where(table.isnan(), torch.zeros_like(table), table)
    got = ze.ze_embedding(torch.arange(256, device="cuda").flip(0), table)
    assert torch.equal(got, table.flip(0))


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_lookup_of_slices_at_odd_places(dtype):
    """Rows that start anywhere, apart by a stride; what lies between them stays as it was."""
    t, g = TYPES[dtype], _generator(3)
    for cols in (1, 6, 63, 130, 520):
        flat = torch.randn(1 + 20 * (cols + 5), generator=g, device="cuda").to(t)
        table = flat[1:].view(20, cols + 5)[:, 2:2 + cols]
        out = torch.full((3 + 9 * (cols + 3),), 7.0, dtype=t, device="cuda")
        rows = out[3:].view(9, cols + 3)[:, 1:1 + cols]
        at = _ids(9, -1, 22, g)
        assert ze.ze_embedding(at, table, scale=0.5, d_out=rows) is rows
        _close(rows, *ze_ref.embedding(at, table, 0, 0.5))
        rows.fill_(7.0)
        assert (out == 7.0).all()


def test_lookup_of_infinities_and_nan_and_of_ids_past_32_bits():
    table = torch.tensor([[1.0, float("inf"), float("nan"), -float("inf")]] * 3, device="cuda")
    first = (1 << 40) + 5
    ids = torch.tensor([first, first + 2, first + 3, 5, 0, -(1 << 62), (1 << 62)], device="cuda")
    got = ze.ze_embedding(ids, table, first=first, scale=-2.0)
    assert (got[:2, 1] == -float("inf")).all() and got[:2, 2].isnan().all() and (got[:2, 0] == -2.0).all()
    assert (got[2:] == 0).all()


BACKWARD = SHAPES + [(8192, 300, 16), (8193, 300, 16), (20000, 70000, 24), (100001, 5, 40), (1 << 16, 257, 8)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("tokens, rows, cols", BACKWARD)
def test_gradient(dtype, tokens, rows, cols):
    t, g = TYPES[dtype], _generator(tokens * 3 + rows + cols)
    dout = torch.randn((tokens, cols), generator=g, device="cuda").to(t)
    for first, scale, ids, out, accumulate in ((0, 1.0, torch.int64, torch.float32, False), (11, 0.3, torch.int32, t, True), (5, -2.0, torch.int64, t, False)):
        at = _ids(tokens, first - 2, first + rows + 2, g, ids)
        old = torch.randn((rows, cols), generator=g, device="cuda").to(out)
        got = ze.ze_embedding_backward(at, dout, rows, first=first, scale=scale, d_dtable=old.clone(), accumulate=accumulate)
        _close(got, *ze_ref.embedding_backward(at, dout, rows, first, scale, old if accumulate else None, out))


@pytest.mark.parametrize("tokens", (15, 16, 17, 160, 5000, 20000, 70000))
def test_gradient_of_tokens_that_come_often(tokens):
    """Runs of one row that fill pieces of the sorted list, begin and end inside them and at their borders."""
    g = _generator(tokens)
    dout = torch.randn((tokens, 72), generator=g, device="cuda").bfloat16()
    half = torch.zeros(tokens, dtype=torch.int64, device="cuda")
    half[tokens // 2:] = 3
    for at in (torch.zeros_like(half), half, half.flip(0), torch.where(torch.arange(tokens, device="cuda") % 3 == 0, half, half - 7),
               torch.arange(tokens, device="cuda") // 16, torch.arange(tokens, device="cuda") // 17, torch.full_like(half, -100)):
        rows = max(4, int(at.max()) + 2)
        _close(ze.ze_embedding_backward(at, dout, rows), *ze_ref.embedding_backward(at, dout, rows))


def test_gradient_is_the_same_each_time_and_for_any_place():
    g = _generator(9)
    for tokens in (3000, 30000):
        at = (torch.rand(tokens, generator=g, device="cuda") ** 4 * 50).long()
        dout = torch.randn((tokens, 129), generator=g, device="cuda").bfloat16()
        wide = torch.zeros((tokens, 140), dtype=torch.bfloat16, device="cuda")
        wide[:, 3:132] = dout
        first = ze.ze_embedding_backward(at, dout, 60)
        for _ in range(3):
            assert torch.equal(first, ze.ze_embedding_backward(at, dout, 60))
        assert torch.equal(first, ze.ze_embedding_backward(at, wide[:, 3:132], 60))


def test_gradient_leaves_alone_what_is_not_its_own():
    """Padding between the rows; with accumulate the rows of no token, NaN among them."""
    g = _generator(4)
    for t in TYPES.values():
        out = torch.full((2 + 30 * 70,), 7.0, dtype=t, device="cuda")
        rows = out[2:].view(30, 70)[:, 1:66]
        dout = torch.randn((50, 65), generator=g, device="cuda").to(t)
        at = _ids(50, 0, 20, g)
        ze.ze_embedding_backward(at, dout, 30, d_dtable=rows)
        _close(rows, *ze_ref.embedding_backward(at, dout, 30, dtype=t))
        rows[20:] = float("nan")
        before = rows.clone()
        ze.ze_embedding_backward(at, dout, 30, d_dtable=rows, accumulate=True)
        assert rows[20:].isnan().all()
        want, bound = ze_ref.embedding_backward(at, dout, 20, old=before[:20], dtype=t)
        _close(rows[:20], want, bound)
        rows.fill_(7.0)
        assert (out == 7.0).all()


def test_gradient_of_infinities_stays_in_its_row():
    dout = torch.ones((4, 40), device="cuda")
    dout[1, 3] = float("inf")
    dout[2, 5] = float("nan")
    got = ze.ze_embedding_backward(torch.tensor([0, 1, -1, 2], device="cuda"), dout, 4)
    assert got[1, 3] == float("inf") and got.isnan().sum() == 0 and got.isinf().sum() == 1 and (got[3] == 0).all()


def test_gradient_against_differences():
    """The sum of the lookup's output times a weight, and what it changes by with the table: linear, so that differences say it exactly."""
    g = _generator(12)
    table = torch.randn((6, 5), generator=g, device="cuda")
    at = torch.tensor([0, 3, 3, 5, -1, 9, 3], device="cuda")
    weight = torch.randn((7, 5), generator=g, device="cuda")
    got = ze.ze_embedding_backward(at, weight, 6, scale=2.0)

    def value(t):
        return (ze.ze_embedding(at, t, scale=2.0).double() * weight.double()).sum()

    for v, x in ((0, 0), (3, 4), (5, 2), (1, 1)):
        more = table.clone()
        more[v, x] += 1.0
        assert abs(float(value(more) - value(table)) - float(got[v, x])) < 1e-4


@pytest.mark.parametrize("tokens, rows, cols", [(1, 5, 3), (15, 40, 100), (512, 1000, 256), (4097, 3, 64), (8192, 500, 72), (8193, 500, 72), (30000, 70001, 9)])
def test_a_workspace_as_large_as_it_has_to_be(tokens, rows, cols):
    """What lies behind a workspace of just the bytes that a call asks for stays as it was."""
    g = _generator(tokens)
    at = _ids(tokens, -1, min(rows, 30), g)
    dout = torch.randn((tokens, cols), generator=g, device="cuda").bfloat16()
    out = torch.empty((rows, cols), device="cuda")
    L, f = ze.lib(), ze.Form(tokens, rows, cols, 0, 1, 0, ze.ZE_I64, 1.0)
    size = L.ze_embedding_work_bytes(f)
    work = torch.full((size + (16 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
    assert L.ze_embedding_backward(f, at.data_ptr(), dout.data_ptr(), out.data_ptr(), 0, work.data_ptr(), size, torch.cuda.current_stream().cuda_stream) == 0
    _close(out, *ze_ref.embedding_backward(at, dout, rows))
    assert (work[size:] == 0x5A).all()


def test_nothing_to_do():
    empty = torch.empty(0, dtype=torch.int64, device="cuda")
    table = torch.ones((3, 4), device="cuda")
    assert ze.ze_embedding(empty, table).shape == (0, 4)
    assert (ze.ze_embedding(torch.tensor([0, 1], device="cuda"), table[:0]) == 0).all()
    d = torch.full((3, 4), 7.0, device="cuda")
    assert (ze.ze_embedding_backward(empty, table[:0], 3, d_dtable=d.clone()) == 0).all()
    assert (ze.ze_embedding_backward(empty, table[:0], 3, d_dtable=d.clone(), accumulate=True) == 7.0).all()
    assert ze.ze_embedding_backward(torch.tensor([0], device="cuda"), table[:1], 0).shape == (0, 4)
    assert ze.ze_embedding(torch.zeros((2, 3), dtype=torch.int64, device="cuda"), table).shape == (2, 3, 4)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("cols", (24, 1100))
def test_gradient_of_runs_around_the_length_that_is_shared_out(dtype, cols):
    """Rows whose tokens fill 31 to 34, 63 to 66 and several hundred pieces of the sorted list, one behind the other, from any place in a piece on; the
    columns in one and in several parts.  (Pieces are 8 to 64 tokens long.)"""
    t, g = TYPES[dtype], _generator(cols)
    for lengths in ([8 * 32 + k for k in range(-9, 10, 3)] * 3, [16 * 33 - 1, 1, 16 * 33, 2, 16 * 33 + 1, 16 * 34, 16 * 31 + 5], [5, 8 * 64, 8 * 65, 8 * 63, 8 * 66 + 1, 3, 8 * 64 - 1],
                    [4000, 1, 4095], [1, 9000, 30, 7000], [70000]):
        at = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), torch.tensor(lengths, device="cuda"))
        at = at[torch.randperm(at.numel(), generator=g, device="cuda")] * 3
        rows = 3 * len(lengths) + 1
        dout = torch.randn((at.numel(), cols), generator=g, device="cuda").to(t)
        got = ze.ze_embedding_backward(at, dout, rows, scale=0.5)
        _close(got, *ze_ref.embedding_backward(at, dout, rows, 0, 0.5))
        assert torch.equal(got, ze.ze_embedding_backward(at, dout, rows, scale=0.5))
        old = torch.randn((rows, cols), generator=g, device="cuda").to(t)
        got = ze.ze_embedding_backward(at, dout, rows, d_dtable=old.clone(), accumulate=True)
        _close(got, *ze_ref.embedding_backward(at, dout, rows, 0, 1.0, old, t))


def test_gradient_of_a_token_that_the_whole_batch_has_takes_no_multiple_of_the_time():
    """A pad token that is an ordinary row.  (Added up by one wavefront its parts took 4.4 times the time of as many tokens of many rows; shared out, 1.6.)"""
    g = _generator(2)
    dout = torch.randn((16384, 256), generator=g, device="cuda").bfloat16()
    many = _ids(16384, 0, 12608, g)
    out = torch.empty((12608, 256), device="cuda")

    def time_of(at):
        times = []
        for _ in range(12):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            for _ in range(10):
                ze.ze_embedding_backward(at, dout, 12608, d_dtable=out)
            end.record()
            end.synchronize()
            times.append(begin.elapsed_time(end))
        return min(times)

    assert time_of(torch.zeros_like(many)) < 2.5 * time_of(many)
