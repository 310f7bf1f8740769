"""Counts that are below a table's own entries (include/cdsl_tree.h): latched by every page call whatever threads come first, and no
page that a sequence keeps is dealt to another."""
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from test_gpu_pages import batch_of, holders, plain_compact, plain_resize, pool, raw, tensor, workspace  # noqa: E402
from test_gpu_tree import cdsl, ints, status  # noqa: E402,F401
from tree_reference import BF, F8  # noqa: E402

U8 = torch.uint8


def resize(cdsl, c, refs, slots, in_place=False):
    """Status, table and counts."""
    st, ws = status(), workspace(cdsl, c)
    if in_place:
        c, r = c.at(c.page_table.clone()), ints(*refs)
        cdsl.cdsl_kv_resize(c, r, ints(*slots), c.page_table, r, ws, status=st)
        return int(st), c.page_table.tolist(), r.tolist()
    out = [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in (c.page_table.shape, (len(refs),))]
    cdsl.cdsl_kv_resize(c, ints(*refs), ints(*slots), *out, ws, status=st)
    return int(st), out[0].tolist(), out[1].tolist()


def held_once(table, n):
    """The counts of n pages, of which no entry is twice."""
    refs = holders(table, n)
    assert max(refs) == 1
    return refs


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("cols", [2, 64, 1500])
@pytest.mark.parametrize("giver", [0, 1])
def test_resize_keeps_a_page_that_another_entry_gives_up(cdsl, in_place, cols, giver):
    """A page with a count of 1 that two sequences hold: one gives it up, a third one grows."""
    P, at, n = 16, cols - 1, 3 * cols + 2
    table = [list(range(cols)), list(range(cols, 2 * cols)), [-1] * cols]
    table[1][at] = table[0][at]
    c = pool(cdsl, U8, 1, n, 1, P, 64, tensor(table))
    refs = [min(r, 1) for r in holders(table, n)]
    slots = [0 if b == giver else P * cols for b in range(2)] + [P * cols]
    for _ in range(5):
        st, now, counts = resize(cdsl, c, refs, slots, in_place)
        assert st == cdsl.CDSL_EINVAL
        assert now[giver] == [-1] * cols and now[1 - giver] == table[1 - giver]
        assert counts == held_once(now, n)
        kept = set(now[1 - giver])
        assert now[2] == [p for p in range(n) if p not in kept][:cols]   # the lowest that nobody keeps


@pytest.mark.parametrize("in_place", [False, True])
def test_resize_of_a_page_that_two_entries_keep(cdsl, in_place):
    """Latched, and the counts are the entries' afterwards; a holder beyond the table counts, a count below 0 does not."""
    table = [[0, 1], [2, 1], [-1, -1]]
    c = pool(cdsl, BF, 1, 8, 1, 16, 64, tensor(table))
    run = lambda *refs: resize(cdsl, c, refs, [32, 32, 16], in_place)  # noqa: E731
    want = [[0, 1], [2, 1], [3, -1]]
    assert run(1, 2, 1, 0, 0, 0, 0, 0) == (cdsl.CDSL_OK, want, [1, 2, 1, 1, 0, 0, 0, 0])
    assert run(1, 3, 1, 0, 0, 0, 0, 0) == (cdsl.CDSL_OK, want, [1, 3, 1, 1, 0, 0, 0, 0])
    assert run(1, 1, 1, 0, 0, 0, 0, 0) == (cdsl.CDSL_EINVAL, want, [1, 2, 1, 1, 0, 0, 0, 0])
    assert run(1, 2, 1, 0, 0, 0, 0, -1) == (cdsl.CDSL_EINVAL, want, [1, 2, 1, 1, 0, 0, 0, 0])


def test_fork_copies_from_a_page_that_two_entries_hold(cdsl):
    """A partly filled page with two entries and a count of 1 or 0 stays neither with one successor nor with the free pages before
    its rows have been copied."""
    P, table, lens, src = 16, [[0, 1], [2, 1], [3, -1]], [20, 20, 10], [0, 2, 2]
    c = pool(cdsl, F8, 2, 6, 2, P, 64, tensor(table))
    before = raw(c)
    for low in (1, 0):
        for x, y in zip((c.pool, c.scale), before):
            x.view(U8).copy_(y.view(x.view(U8).shape))
        st, out = status(), [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((3, 2), (3,), (6,))]
        cdsl.cdsl_kv_fork(c, ints(1, low, 1, 1, 0, 0), ints(*src), ints(*lens), *out, workspace(cdsl, c, 3), status=st)
        assert int(st) == cdsl.CDSL_EINVAL
        assert [x.tolist() for x in out] == [[[0, 2], [3, -1], [4, -1]], [20, 10, 10], [1, 0, 1, 1, 1, 0]]
        for old, now in zip(before, raw(c)):
            assert torch.equal(now[:, 2, :, :, :4], old[:, 1, :, :, :4]) and torch.equal(now[:, 4, :, :, :10], old[:, 3, :, :, :10])
            assert all(torch.equal(now[:, p], old[:, p]) for p in (0, 1, 3, 5))


def test_fork_shares_a_whole_page_whose_count_is_too_low(cdsl):
    """It is not dealt out for a copy."""
    P, table = 16, [[1, 0], [1, 2]]
    c = pool(cdsl, U8, 1, 6, 1, P, 64, tensor(table))
    st, out = status(), [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((3, 2), (3,), (6,))]
    cdsl.cdsl_kv_fork(c, ints(1, 1, 1, 0, 0, 0), ints(0, 0, 1), ints(20, 16), *out, workspace(cdsl, c, 3), status=st)
    assert int(st) == cdsl.CDSL_EINVAL
    assert [x.tolist() for x in out] == [[[1, 0], [1, 2], [1, -1]], [20, 20, 16], [1, 3, 1, 0, 0, 0]]


def test_compact_of_a_page_that_two_entries_hold(cdsl):
    table = [[4, 1], [5, 1]]
    c = pool(cdsl, U8, 1, 6, 1, 16, 64, tensor(table))
    for count, want in ((1, cdsl.CDSL_EINVAL), (2, cdsl.CDSL_OK), (3, cdsl.CDSL_OK)):
        refs = [0, count, 0, 0, 1, 1]
        st, out = status(), [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((2, 2), (6,), (6,), (1,))]
        cdsl.cdsl_kv_compact(c, ints(*refs), *out, workspace(cdsl, c), status=st)
        assert int(st) == want
        assert [x.tolist() for x in out] == [[[0, 1], [2, 1]], [1, count, 1, 0, 0, 0], [-1, 1, -1, -1, 0, 2], [3]]


@pytest.mark.parametrize("B,cols", [(12, 30), (40, 60), (8, 1500)])
def test_one_count_too_low_among_many(cdsl, B, cols):
    """More pages and entries than a block has threads; every call latches, and the counts as they are do not."""
    rng, P = random.Random(cols), 16
    lens, table, n = batch_of(rng, B, cols, P, 40 if cols < 1000 else 2000)
    lens = [min(a, P * sum(p >= 0 for p in row)) for a, row in zip(lens, table)]
    for b in range(1, B):                      # every whole page that both can have is shared
        m = min(lens[b - 1:b + 1]) // P
        table[b][:m] = table[b - 1][:m]
    c = pool(cdsl, U8, 1, n, 1, P, 64, tensor(table))
    right = holders(table, n)
    twice = [p for p in range(n) if right[p] > 1]
    slots = [rng.randint(0, P * cols) for _ in range(B)]
    assert twice
    for p in [None] + rng.sample(twice, min(4, len(twice))):
        refs = list(right)
        if p is not None:
            refs[p] -= 1
        want = cdsl.CDSL_OK if p is None else cdsl.CDSL_EINVAL
        st, now, counts = resize(cdsl, c, refs, slots)
        # (a count that is too low counts as the entries': the result is that of the right ones)
        table_after, refs_after = plain_resize(table, right, slots, P)
        full = any(-1 in row[:-(-s // P)] for row, s in zip(table_after, slots))
        assert st == (cdsl.CDSL_ENOMEM if p is None and full else want)
        assert now == table_after and counts == refs_after == holders(now, n)
        st, out = status(), [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((B, cols), (B,), (n,))]
        cdsl.cdsl_kv_fork(c, ints(*refs), ints(*range(B)), ints(*lens), *out, workspace(cdsl, c, B), status=st)
        assert int(st) == want and out[2].tolist() == holders(out[0].tolist(), n)
        st, out = status(), [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((B, cols), (n,), (n,), (1,))]
        cdsl.cdsl_kv_compact(c, ints(*refs), *out, workspace(cdsl, c), status=st)
        assert int(st) == want and out[0].tolist() == plain_compact(table, refs)[0]


def test_fork_latches_the_entries_that_a_successor_was_to_have(cdsl):
    """Pages that are not, whole or partly filled, inside the length; none behind it or of a sequence without successors."""
    P, n = 16, 8
    refs = [1, 1, 1, 1, 0, 0, 0, 0]

    def fork(table, src, lens):
        c = pool(cdsl, U8, 1, n, 1, P, 64, tensor(table))
        st, out = status(), [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((len(src), 3), (len(src),), (n,))]
        cdsl.cdsl_kv_fork(c, ints(*refs), ints(*src), ints(*lens), *out, workspace(cdsl, c, len(src)), status=st)
        return [int(st)] + [x.tolist() for x in out]

    keeps = [cdsl.CDSL_OK, [[0, 1, -1]], [20], [1, 1, 0, 0, 0, 0, 0, 0]]
    assert fork([[0, 1, 99], [2, 3, -1]], [0], [20, 0]) == keeps          # behind the length
    assert fork([[0, 1, -1], [2, 3, -7]], [0], [20, 48]) == keeps         # without successors
    for bad in (-1, 8, -(1 << 31)):
        assert fork([[0, bad, 1], [2, 3, -1]], [0], [40, 0]) == [cdsl.CDSL_ERANGE, [[0, -1, 1]], [40], [1, 1, 0, 0, 0, 0, 0, 0]]
        assert fork([[0, 1, bad], [2, 3, -1]], [0], [40, 0]) == [cdsl.CDSL_ERANGE, [[0, 1, -1]], [32], [1, 1, 0, 0, 0, 0, 0, 0]]


@pytest.mark.parametrize("dtype", [U8, F8, BF])
def test_going_back_into_a_shared_page_by_a_fork(cdsl, dtype):
    """Two beams share a prompt's two whole pages; one goes back to 20 of its 32 tokens and writes others: the second beam's
    rows stay."""
    P, cols, n = 16, 3, 8
    cache = pool(cdsl, dtype, 2, n, 2, P, 64, tensor([[0, 1, -1], [0, 1, -1]]))
    refs = ints(2, 2, 0, 0, 0, 0, 0, 0)
    before, st = raw(cache), status()
    out = [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((2, cols), (2,), (n,))]
    cdsl.cdsl_kv_fork(cache, refs, ints(0, 1), ints(20, 32), *out, workspace(cdsl, cache, 2), status=st)
    assert [x.tolist() for x in out] == [[[0, 2, -1], [0, 1, -1]], [20, 32], [2, 1, 1, 0, 0, 0, 0, 0]]
    forked = cache.at(out[0])
    k = torch.ones((2, 8, 2, 64), dtype=BF, device="cuda")
    for layer in range(2):
        cdsl.cdsl_kv_write(forked, layer, k, k, out[1], ints(8, 0), status=st)
    now = raw(cache)
    for x, y in zip(before, now):
        assert torch.equal(y[:, :2], x[:, :2])                            # the prompt's pages
        assert torch.equal(y[:, 2, :, :, :4], x[:, 1, :, :, :4])          # the copied rows
        assert not torch.equal(y[:, 2, :, :, 4:12], x[:, 1, :, :, 4:12])  # and the new ones
    assert int(st) == cdsl.CDSL_OK
