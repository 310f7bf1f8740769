"""Which sequence has which pages (cdsl_kv_fork, cdsl_kv_resize, cdsl_kv_compact in include/cdsl_tree.h) against plain
lists, for every type of cache; and a served batch's life with all of them together."""
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import i4_reference as i4  # noqa: E402
import tree_reference as ref  # noqa: E402
from test_gpu_tree import cdsl, ints, randn, status  # noqa: E402,F401
from tree_reference import BF, F8  # noqa: E402

U8 = torch.uint8
CACHES = pytest.mark.parametrize("dtype,kvh,hd,page", [(U8, 2, 128, 64), (F8, 3, 64, 16), (BF, 1, 128, 32), (U8, 5, 64, 16),
                                                       (F8, 2, 128, 256)])


def pool(cdsl, dtype, layers, n, kvh, page, hd, table, seed=0):
    """A cache of random bytes, and a view of its codes and scales as bytes [layers, n, 2, kvh, page, ..]."""
    g = torch.Generator().manual_seed(seed)
    c = cdsl.KvCache.empty(layers, n, kvh, page, hd, table, dtype)
    for x in (c.pool, c.scale):
        x.view(U8).copy_(torch.randint(0, 256, x.view(U8).shape, generator=g, dtype=U8))
    return c


def raw(c):
    return [c.pool.view(U8).view(*c.pool.shape[:5], -1).clone(), c.scale.view(U8).view(*c.pool.shape[:5], -1).clone()]


def holders(table, n, more=()):
    refs = [0] * n
    for row in table:
        for p in row:
            if 0 <= p < n:
                refs[p] += 1
    for p in more:
        refs[p] += 1
    return refs


def workspace(cdsl, c, new=None):
    return torch.full((cdsl.cdsl_kv_pages_workspace(c, new),), 255, dtype=U8, device="cuda")


def plain_fork(table, refs, src, lens, P, cols):
    """New table, lengths, counts and the copies (from, to, rows)."""
    refs = list(refs)
    alone = [r == 1 for r in refs]
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] -= 1
    first, new, copies, want = {}, [], [], []
    for i, b in enumerate(src):
        first.setdefault(b, i)
        full, rest = divmod(lens[b], P)
        row = list(table[b][:full])
        for p in row:
            refs[p] += 1
        if rest:
            p = table[b][full]
            if first[b] == i and alone[p]:
                refs[p] += 1
                row.append(p)
            else:
                want.append((i, p, rest))
                row.append(None)
        new.append(row + [-1] * (cols - len(row)))
    busy = {p for _, p, _ in want}
    free = [p for p in range(len(refs)) if refs[p] == 0 and p not in busy]
    new_lens = [lens[b] for b in src]
    for i, p, rest in want:
        at = new[i].index(None)
        if free:
            to = free.pop(0)
            refs[to] += 1
            copies.append((p, to, rest))
            new[i][at] = to
        else:
            new[i][at] = -1
            new_lens[i] -= rest
    return new, new_lens, refs, copies


def plain_resize(table, refs, slots, P):
    refs, out = list(refs), [list(r) for r in table]
    for b, row in enumerate(out):
        for c in range(-(-slots[b] // P), len(row)):
            if row[c] >= 0:
                refs[row[c]] -= 1
            row[c] = -1
    free = [p for p in range(len(refs)) if refs[p] == 0]
    for b, row in enumerate(out):
        for c in range(-(-slots[b] // P)):
            if row[c] < 0 and free:
                row[c] = free.pop(0)
                refs[row[c]] = 1
    return out, refs


def plain_compact(table, refs):
    n = sum(r > 0 for r in refs)
    move = dict(zip([p for p in range(n, len(refs)) if refs[p] > 0], [p for p in range(n) if refs[p] <= 0]))
    page_map = [move.get(p, p) if refs[p] > 0 else -1 for p in range(len(refs))]
    new = [0] * len(refs)
    for p, r in enumerate(refs):
        if r > 0:
            new[page_map[p]] = r
    return [[page_map[p] if p >= 0 else -1 for p in row] for row in table], new, page_map, n, move


def batch_of(rng, B, cols, P, spare, shared=True):
    """Ragged sequences with pages past their length, some of which share their first pages; pages in random order."""
    lens = [rng.choice([0, 1, P, P * cols, rng.randint(0, P * cols), rng.randint(0, P * cols)]) for _ in range(B)]
    table, n = [], 0
    for b in range(B):
        held = min(cols, -(-lens[b] // P) + rng.randint(0, 2))
        row = []
        for c in range(cols):
            if shared and b % 3 and c < min(lens[b], lens[b - 1]) // P // 2:
                row.append(table[b - 1][c])
            elif c < held:
                row.append(n)
                n += 1
            else:
                row.append(-1)
        table.append(row)
    order = list(range(n + spare))
    rng.shuffle(order)
    return lens, [[order[p] if p >= 0 else -1 for p in row] for row in table], n + spare


def tensor(rows):
    return torch.tensor(rows, dtype=torch.int32, device="cuda")


@CACHES
@pytest.mark.parametrize("B,new,cols", [(1, 4, 3), (6, 6, 5), (17, 40, 2), (5, 1, 7)])
def test_fork(cdsl, dtype, kvh, hd, page, B, new, cols):
    rng = random.Random(B * new)
    lens, table, n = batch_of(rng, B, cols, page, new)
    src = [rng.randrange(B) for _ in range(new)]
    c = pool(cdsl, dtype, 3, n, kvh, page, hd, tensor(table), seed=B)
    refs = holders(table, n)
    before = raw(c)
    st, out = status(), [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((new, cols), (new,), (n,))]
    cdsl.cdsl_kv_fork(c, ints(*refs), ints(*src), ints(*lens), *out, workspace(cdsl, c, new), status=st)
    want = plain_fork(table, refs, src, lens, page, cols)
    assert [x.tolist() for x in out] == list(want[:3]) and int(st) == cdsl.CDSL_OK
    assert want[2] == holders(want[0], n)
    copied = {to: (p, rest) for p, to, rest in want[3]}
    for old, now in zip(before, raw(c)):
        for p in range(n):
            if p in copied:
                q, rest = copied[p]
                assert torch.equal(now[:, p, :, :, :rest], old[:, q, :, :, :rest])
            else:
                assert torch.equal(now[:, p], old[:, p])


def test_fork_keeps_what_others_hold(cdsl):
    """A partly filled page with two holders is copied even for a first successor, and not dealt out before it has been read;
    pages that a count holds beyond the table stay."""
    P = 16
    table = [[0, 2], [0, 2], [3, 4]]
    refs = holders(table, 8, more=[3])
    lens = [20, 20, 30]
    c = pool(cdsl, U8, 2, 8, 2, P, 64, tensor(table))
    before = raw(c)
    src = [0, 1, 1]
    out = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((3, 2), (3,), (8,))]
    cdsl.cdsl_kv_fork(c, ints(*refs), ints(*src), ints(*lens), *out, workspace(cdsl, c, 3))
    want = plain_fork(table, refs, src, lens, P, 2)
    assert [x.tolist() for x in out] == list(want[:3])
    assert out[0].tolist() == [[0, 1], [0, 4], [0, 5]] and out[2].tolist() == [3, 1, 0, 1, 1, 1, 0, 0]
    for old, now in zip(before, raw(c)):
        for to in (1, 4, 5):
            assert torch.equal(now[:, to, :, :, :4], old[:, 2, :, :, :4])


def test_fork_of_what_is_out_of_range(cdsl):
    """Sequences that are not there, lengths out of range, pages that are not, no free page, counts that are not the
    table's: latched, and every output has a value."""
    P, table = 16, [[0, 1], [2, -1], [3, 99]]
    c = pool(cdsl, F8, 1, 5, 1, P, 64, tensor(table))
    ws = workspace(cdsl, c, 2)

    def fork(src, lens, refs=(1, 1, 1, 1, 0)):
        st, out = status(), [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((2, 2), (2,), (5,))]
        cdsl.cdsl_kv_fork(c, ints(*refs), ints(*src), ints(*lens), *out, ws, status=st)
        return [int(st)] + [x.tolist() for x in out]

    assert fork([0, 3], [20, 3, 3]) == [cdsl.CDSL_ERANGE, [[0, 1], [-1, -1]], [20, 0], [1, 1, 0, 0, 0]]
    assert fork([-1, 1], [20, 3, 3]) == [cdsl.CDSL_ERANGE, [[-1, -1], [2, -1]], [0, 3], [0, 0, 1, 0, 0]]
    assert fork([0, 1], [33, -3, 3]) == [cdsl.CDSL_ERANGE, [[0, 1], [-1, -1]], [32, 0], [1, 1, 0, 0, 0]]
    assert fork([1, 2], [0, 20, 16]) == [cdsl.CDSL_ERANGE, [[2, -1], [3, -1]], [16, 16], [0, 0, 1, 1, 0]]
    assert fork([2, 2], [0, 0, 30]) == [cdsl.CDSL_ERANGE, [[3, -1], [3, -1]], [16, 16], [0, 0, 0, 2, 0]]
    assert fork([0, 0], [20, 0, 0], (1, 1, 2, 2, 1)) == [cdsl.CDSL_ENOMEM, [[0, 1], [0, -1]], [20, 16], [2, 1, 1, 1, 1]]
    assert fork([1, 0], [0, 0, 0], (0, 1, 1, 1, 0))[0] == cdsl.CDSL_EINVAL


@pytest.mark.parametrize("B,cols,page", [(1, 1, 16), (7, 9, 64), (40, 50, 16), (3, 1500, 256)])
def test_resize(cdsl, B, cols, page):
    """To nothing, to everything, and to some; in place too; more entries and pages than the block has threads."""
    rng = random.Random(cols)
    lens, table, n = batch_of(rng, B, cols, page, B * cols // 2 + 3)
    c = pool(cdsl, U8, 1, n, 1, page, 64, tensor(table)) if n < 3000 else \
        cdsl.KvCache.empty(1, n, 1, page, 64, tensor(table), U8)
    refs = holders(table, n)
    ws = workspace(cdsl, c)
    for slots in ([0] * B, [page * cols] * B, [rng.randint(0, page * cols) for _ in range(B)]):
        want = plain_resize(table, refs, slots, page)
        full = any(-1 in row[:-(-s // page)] for row, s in zip(want[0], slots))
        st, out = status(), [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((B, cols), (n,))]
        cdsl.cdsl_kv_resize(c, ints(*refs), ints(*slots), *out, ws, status=st)
        assert out[0].tolist() == want[0] and out[1].tolist() == want[1]
        assert int(st) == (cdsl.CDSL_ENOMEM if full else cdsl.CDSL_OK)
        own, r = c.at(tensor(table)), ints(*refs)
        cdsl.cdsl_kv_resize(own, r, ints(*slots), own.page_table, r, ws)
        assert own.page_table.tolist() == want[0] and r.tolist() == want[1]
    st, own, r = status(), c.at(tensor(table)), ints(*refs)
    cdsl.cdsl_kv_resize(own, r, ints(*[page * cols + 1] + [-1] * (B - 1)), own.page_table, r, ws, status=st)
    assert int(st) == cdsl.CDSL_ERANGE
    assert own.page_table.tolist() == plain_resize(table, refs, [page * cols] + [0] * (B - 1), page)[0]


@CACHES
@pytest.mark.parametrize("B,cols,gone", [(1, 1, 0.0), (9, 6, 0.5), (30, 60, 0.4), (4, 3, 1.0)])
def test_compact(cdsl, dtype, kvh, hd, page, B, cols, gone):
    if page == 256 and cols == 60:
        cols = 20
    rng = random.Random(B)
    lens, table, n = batch_of(rng, B, cols, page, 5)
    for row in table:
        if rng.random() < gone:
            row[:] = [-1] * cols
    refs = holders(table, n, more=[n - 1])        # (one that no table has)
    c = pool(cdsl, dtype, 2, n, kvh, page, hd, tensor(table), seed=B)
    before = raw(c)
    want = plain_compact(table, refs)
    outs = [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((B, cols), (n,), (n,), (1,))]
    st = status()
    cdsl.cdsl_kv_compact(c, ints(*refs), *outs, workspace(cdsl, c), status=st)
    assert [x.tolist() for x in outs] == [want[0], want[1], want[2], [want[3]]] and int(st) == cdsl.CDSL_OK
    for old, now in zip(before, raw(c)):
        idx = list(range(n))
        for p, q in want[4].items():
            idx[q] = p
        assert torch.equal(now, old[:, idx])
    own, r = c.at(tensor(table)), ints(*refs)
    cdsl.cdsl_kv_compact(own, r, own.page_table, r, outs[2], outs[3], workspace(cdsl, c))
    assert [own.page_table.tolist(), r.tolist()] == [want[0], want[1]]


def test_counts_below_the_tables_are_latched(cdsl):
    """An entry of a page that the counts call free: by every call, and nothing outside the outputs is written."""
    c = pool(cdsl, U8, 1, 6, 1, 16, 64, tensor([[0, 1], [2, -1]]))
    before = raw(c)
    ws = workspace(cdsl, c)
    outs = [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((2, 2), (6,), (6,), (1,))]
    for refs in ([1, 0, 1, 0, 0, 0], [1, -1, 1, 0, 0, 0]):
        st = status()
        cdsl.cdsl_kv_resize(c, ints(*refs), ints(32, 16), *outs[:2], ws, status=st)
        assert int(st) == cdsl.CDSL_EINVAL and outs[0].tolist() == [[0, 1], [2, -1]]
        st.zero_()
        cdsl.cdsl_kv_resize(c, ints(*refs), ints(0, 0), *outs[:2], ws, status=st)
        assert int(st) == cdsl.CDSL_EINVAL
        st.zero_()
        cdsl.cdsl_kv_compact(c, ints(*refs), *outs, ws, status=st)
        assert int(st) == cdsl.CDSL_EINVAL and int(outs[3]) == 2 and outs[0].tolist() == [[0, -1], [1, -1]]
        c = pool(cdsl, U8, 1, 6, 1, 16, 64, tensor([[0, 1], [2, -1]]))
        assert all(torch.equal(x, y) for x, y in zip(before, raw(c)))


def test_page_calls_in_graphs_and_on_other_streams(cdsl):
    """Captured once and replayed with other lengths and successors, on a side stream too."""
    rng, P = random.Random(5), 16
    lens, table, n = batch_of(rng, 4, 6, P, 12)
    c = pool(cdsl, U8, 2, n, 2, P, 64, tensor(table))
    refs, src, dl, ws = ints(*holders(table, n)), ints(0, 1, 2, 3), ints(*lens), workspace(cdsl, c, 4)
    out = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((4, 6), (4,), (n,))]
    nxt = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((4, 6), (n,))]
    forked, slots = c.at(out[0]), ints(1, 1, 1, 1)

    def step(stream=None):
        cdsl.cdsl_kv_fork(c, refs, src, dl, *out, ws, stream=stream)
        cdsl.cdsl_kv_resize(forked, out[2], slots, *nxt, ws, stream=stream)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    step(side.cuda_stream)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for s, l in (([1, 1, 0, 3], lens), ([2, 2, 2, 2], [5, 17, 40, 96])):
        src.copy_(ints(*s))
        l = [min(a, P * sum(p >= 0 for p in row)) for a, row in zip(l, table)]
        dl.copy_(ints(*l))
        slots.copy_(ints(*[l[b] + 1 for b in s]) - (ints(*[l[b] for b in s]) == 6 * P).int())
        g.replay()
        want = plain_fork(table, refs.tolist(), s, l, P, 6)
        assert [x.tolist() for x in out] == list(want[:3])
        wt, wr = plain_resize(want[0], want[2], slots.tolist(), P)
        assert nxt[0].tolist() == wt and nxt[1].tolist() == wr


@pytest.mark.parametrize("dtype", [U8, F8])
def test_a_served_batch(cdsl, dtype):
    """A prompt's cache, its beams, their tokens, an ended beam, a compacted pool: with rotated keys written, and the attention
    of every step what a cache of its own, in order, gives for the same tokens."""
    L, kvh, H, hd, P, cols, n = 2, 2, 8, 64, 16, 6, 24
    g = torch.Generator().manual_seed(1)
    rope = cdsl.Rope(hd)
    table, refs = tensor([[-1] * cols]), torch.zeros(n, dtype=torch.int32, device="cuda")
    cache = cdsl.KvCache.empty(L, n, kvh, P, hd, table, dtype)
    st = status()
    lens, history = [0], [[]]                     # a sequence's tokens so far: (k, v, node) of each
    mask1 = torch.tensor([[[1]]], dtype=torch.int32)

    def work(nbytes):
        return torch.full((nbytes,), 255, dtype=U8, device="cuda")

    def append(cache, refs, T):
        """T tokens more for every sequence; the attention of the last of them."""
        B = cache.batch
        ws = work(cdsl.cdsl_kv_pages_workspace(cache))
        cdsl.cdsl_kv_resize(cache, refs, ints(*[l + T for l in lens]), cache.page_table, refs, ws, status=st)
        dl = ints(*lens)
        q, k, v = (randn((L, B, T, h, hd), g, BF) for h in (H, kvh, kvh))
        for l in range(L):
            cdsl.cdsl_rope(rope, q[l], q[l], dl, k=k[l], k_out=k[l])
            cdsl.cdsl_kv_write(cache, l, k[l], v[l], dl, status=st)
        for b in range(B):
            history[b] = history[b] + [(k[:, b, t], v[:, b, t]) for t in range(T)]
            lens[b] += T
        last = ints(*[x - 1 for x in lens])
        mask = mask1.expand(B, 1, 1).contiguous().cuda()
        out = torch.empty((B, 1, H, hd), dtype=BF, device="cuda")
        ws = work(cdsl.cdsl_tree_attention_workspace(cache, 1, H))
        for l in range(L):
            cdsl.cdsl_tree_attention(cache, l, q[l, :, -1:], last, mask, out, ws, scale=0.125, max_len=cols * P - 1, status=st)
            for b in range(B):
                m = lens[b]
                own = cdsl.KvCache.empty(1, cols, kvh, P, hd, torch.arange(cols, dtype=torch.int32, device="cuda")[None], dtype)
                kk, vv = (torch.stack([h[i][l] for h in history[b]])[None] for i in (0, 1))
                cdsl.cdsl_kv_write(own, 0, kk, vv, ints(0))
                want = torch.empty((1, 1, H, hd), dtype=BF, device="cuda")
                cdsl.cdsl_tree_attention(own, 0, q[l, b:b + 1, -1:], ints(m - 1), mask[:1], want, ws, scale=0.125, max_len=m - 1)
                # (other runs: other roundings, of sums of values up to vv's largest)
                e = float(vv.abs().max()) * 2.0 ** -7
                assert (out[b].float() - want[0].float()).abs().max() <= e

    append(cache, refs, 21)
    assert sum(refs.tolist()) == 2
    for src in ([0, 0, 0], [1, 1, 2], [2, 0]):
        out = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((len(src), cols), (len(src),), (n,))]
        cdsl.cdsl_kv_fork(cache, refs, ints(*src), ints(*lens), *out, work(cdsl.cdsl_kv_pages_workspace(cache, len(src))), status=st)
        cache, refs = cache.at(out[0]), out[2]
        lens, history = [lens[b] for b in src], [history[b] for b in src]
        assert out[1].tolist() == lens
        append(cache, refs, 1)
        append(cache, refs, 13)
    maps = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((n,), (1,))]
    cdsl.cdsl_kv_compact(cache, refs, cache.page_table, refs, *maps, work(cdsl.cdsl_kv_pages_workspace(cache)), status=st)
    live = int(maps[1])
    assert int(cache.page_table.max()) == live - 1 and all(r > 0 for r in refs.tolist()[:live]) and not any(refs.tolist()[live:])
    append(cache, refs, 5)
    assert holders(cache.page_table.tolist(), n) == refs.tolist() and int(st) == cdsl.CDSL_OK
