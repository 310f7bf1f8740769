"""Tree speculation over a quantised paged cache (include/cdsl_tree.h) against plain 64-bit implementations: the
cache's write, read and commit, the tree attention, the validation. Pools start full of garbage (NaN codes
and scales among it), pages are in random order."""
import copy
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import tree_reference as ref  # noqa: E402
from tree_reference import BF, F32, F8  # noqa: E402


@pytest.fixture(scope="module")
def cdsl():
    from paper_2412_10418_gb300 import build
    build.build()
    import paper_2412_10418_gb300 as pkg
    return pkg


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def randn(shape, g, dtype=F32, rows=True):
    x = torch.randn(shape, generator=g)
    if rows:
        x = x * torch.randn(shape[:-1], generator=g).exp()[..., None]
    return x.to(dtype).cuda()


# ------------------------------------------------------------------------------ cache

CACHES = [(8, 128, 64, F8), (12, 64, 16, F8), (1, 128, 256, F8), (3, 64, 32, BF), (8, 128, 64, BF)]


@pytest.mark.parametrize("kvh,hd,page,dtype", CACHES)
@pytest.mark.parametrize("T,value", [(1, BF), (17, F32), (67, BF)])
def test_write_and_read(cdsl, kvh, hd, page, dtype, T, value):
    """Rows come back as their definition says, to the bit, at odd starts, ragged counts (0 too) and with rows
    of zeros, huge, tiny and non-finite values; no other row of the pool changes."""
    g = torch.Generator().manual_seed(hd + T)
    B, start = 4, [0, 5, page - 1, 131]
    c = ref.Cache(B, max(start) + T, kvh, hd, page, dtype, layers=2, seed=T)
    k, v = (randn((B, T, kvh, hd), g, value) for _ in range(2))
    k[0, 0, 0] = 0
    v[0, 0, 0] *= 2.0 ** 110
    k[1, 0, 0] *= 2.0 ** -110
    v[1, 0, 0] = 2.0 ** -130                      # a subnormal row
    k[2, 0, 0, :4] = torch.tensor([448.0, 17.0, -19.0, 1.0])   # ties of the rounding
    k[2, 0, 0, 4:] = 0.5
    k[3, 0, 0, 3] = float("nan")
    v[3, 0, 0, hd - 1] = float("-inf")
    count = [T, (T + 1) // 2, T, max(1, T - 3)]
    before, before_scale = c.c.pool.clone(), c.c.scale.clone()
    st = status()
    cdsl.cdsl_kv_write(c.c, 1, k, v, ints(*start), ints(*count), status=st)
    touched = torch.zeros(c.c.scale.shape, dtype=torch.bool, device="cuda")
    outs = []
    for dt in (F32, BF):
        kk, vv = (torch.full((1, B, T, kvh, hd), 7.0, dtype=dt, device="cuda") for _ in range(2))
        cdsl.cdsl_kv_read(c.c, 1, ints(*start), kk, vv, ints(*count), status=st)
        outs.append((kk[0], vv[0]))
    for b in range(B):
        n = count[b]
        for i in range(n):
            s = start[b] + i
            touched[1, int(c.table[b, s // page]), :, :, s % page] = True
        stored = c.values(1, b, start[b], n)
        for j, x in enumerate((k, v)):
            want = ref.quantised(x[b, :n].float())[0] if dtype is F8 else x[b, :n].float().to(BF).double()
            bad = ~torch.isfinite(x[b, :n].float()).all(-1)
            want[bad] = float("nan")
            assert torch.equal(torch.nan_to_num(stored[j], 1e9), torch.nan_to_num(want, 1e9))
            assert torch.equal(torch.nan_to_num(outs[0][j][b, :n].double(), 1e9), torch.nan_to_num(want.float().double(), 1e9))
            assert torch.equal(torch.nan_to_num(outs[1][j][b, :n], 1e9), torch.nan_to_num(want.to(BF), 1e9))
            assert (outs[0][j][b, n:] == 0).all() and (outs[1][j][b, n:] == 0).all()
    raw = (lambda t: t.view(torch.uint8)) if dtype is F8 else (lambda t: t.view(torch.int16))
    assert torch.equal(raw(c.c.pool)[~touched], raw(before)[~touched])
    assert torch.equal(c.c.scale[~touched], before_scale[~touched])
    assert int(st) == cdsl.CDSL_OK


@pytest.mark.parametrize("value", [BF, F32])
def test_write_takes_strided_and_unaligned_rows(cdsl, value):
    """K and V as slices of a fused projection, tokens and heads in other orders, off 16 bytes."""
    g = torch.Generator().manual_seed(1)
    B, T, kvh, hd = 2, 9, 4, 64
    for offset in (0, 8, 1):
        fused = randn((B, T, 3 * kvh * hd + offset), g, value, rows=False)
        k = fused[..., offset:offset + kvh * hd].view(B, T, kvh, hd)
        v = randn((kvh, T, B, hd), g, value).permute(2, 1, 0, 3)
        c = ref.Cache(B, T, kvh, hd, 16, F8, seed=offset)
        cdsl.cdsl_kv_write(c.c, 0, k, v, ints(0, 0))
        for b in range(B):
            for got, x in zip(c.values(0, b, 0, T), (k, v)):
                assert torch.equal(got, ref.quantised(x[b].float())[0])


def test_write_and_read_past_the_pages_latch_erange(cdsl):
    c = ref.Cache(2, 32, 2, 64, 16, F8)
    k = torch.ones((2, 20, 2, 64), dtype=BF, device="cuda")
    st = status()
    before = c.c.scale.clone()
    cdsl.cdsl_kv_write(c.c, 0, k, k, ints(-20, 32), status=st)      # slots below 0 and past the table
    assert int(st) == cdsl.CDSL_ERANGE and torch.equal(c.c.scale, before)
    out = torch.full((1, 2, 20, 2, 64), 3.0, dtype=BF, device="cuda")
    st.zero_()
    cdsl.cdsl_kv_read(c.c, 0, ints(-20, 32), out, out.clone(), status=st)
    assert int(st) == cdsl.CDSL_ERANGE and (out == 0).all()
    bad = c.c.at(torch.tensor([[-1, 1 << 20], [0, 1]], dtype=torch.int32, device="cuda"))
    st.zero_()
    cdsl.cdsl_kv_write(bad, 0, k[:, :1], k[:, :1], ints(17, 1), status=st)   # a page id past the pool
    assert int(st) == cdsl.CDSL_ERANGE
    cdsl.cdsl_kv_write(bad, 0, k[:, :1], k[:, :1], ints(17, 1))              # the same without a status word
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [F8, BF])
@pytest.mark.parametrize("T", [1, 7, 40, 128])
def test_commit_moves_the_path(cdsl, dtype, T):
    """Every layer, paths of any depth (the root alone, all nodes, none), bad paths refused on the device."""
    rng = random.Random(T)
    B, kvh, hd, page, layers = 6, 3, 64, 16, 3
    c = ref.Cache(B, 50 + T, kvh, hd, page, dtype, layers=layers, seed=T)
    g = torch.Generator().manual_seed(T)
    lens = [0, 1, 15, 16, 33, 50]
    for l in range(layers):
        cdsl.cdsl_kv_write(c.c, l, randn((B, T, kvh, hd), g, BF), randn((B, T, kvh, hd), g, BF), ints(*lens))
    paths = [[0], list(range(T)), [0] + sorted(rng.sample(range(1, T), (T - 1) // 2)), [],
             [0] + sorted(rng.sample(range(1, T), min(T - 1, 3))), [0, T - 1] if T > 1 else [0]]
    path = torch.full((B, T), -1, dtype=torch.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    n = ints(*[len(p) for p in paths])
    want = [[c.values(l, b, lens[b], T) for b in range(B)] for l in range(layers)]
    new, st = ints(*[-5] * B), status()
    cdsl.cdsl_kv_commit(c.c, ints(*lens), path.cuda(), n, new, status=st)
    assert new.tolist() == [a + len(p) for a, p in zip(lens, paths)] and int(st) == cdsl.CDSL_OK
    for l in range(layers):
        for b, p in enumerate(paths):
            for got, x in zip(c.values(l, b, lens[b], max(1, len(p))), want[l][b]):
                assert torch.equal(got[:len(p)], x[p])
    if T > 2:   # not increasing, not from 0, too long: nothing of that sequence moves
        for p, m in (([0, 2, 2], 3), ([1, 2], 2), ([0], T + 1), ([0, T], 2)):
            path[0, :len(p)] = torch.tensor(p, dtype=torch.int32)
            n[0] = m
            old = c.values(0, 0, lens[0], T)
            st.zero_()
            cdsl.cdsl_kv_commit(c.c, ints(*lens), path.cuda(), n, new, status=st)
            assert int(st) == cdsl.CDSL_EINVAL and int(new[0]) == lens[0]
            assert all(torch.equal(a, b) for a, b in zip(old, c.values(0, 0, lens[0], T)))


# ------------------------------------------------------------------------------ attention

def problem(cdsl, B, T, H, kvh, hd, page, lens, cache, dtype, kind="random", nodes=None, seed=0, layers=2):
    rng = random.Random(seed)
    g = torch.Generator().manual_seed(seed)
    nodes = nodes or [T] * B
    c = ref.Cache(B, max(lens) + T, kvh, hd, page, cache, layers=layers, seed=seed)
    n = max(lens) + T
    cdsl.cdsl_kv_write(c.c, layers - 1, randn((B, n, kvh, hd), g, BF), randn((B, n, kvh, hd), g, BF), ints(*[0] * B),
                       ints(*[a + b for a, b in zip(lens, nodes)]))
    mask = torch.stack([cdsl.cdsl_tree_mask(ref.tree(kind, T, rng))[0] for _ in range(B)])
    q = randn((B, T, H, hd), g, dtype, rows=False)
    return c, q, mask, nodes


def attend(cdsl, c, layer, q, lens, mask, nodes, scale, max_len=None, out=None, **kw):
    B, T, H, hd = q.shape
    out = torch.full((B, T, H, hd), 9.0, dtype=q.dtype, device="cuda") if out is None else out
    lse = torch.full((B, T, H), 9.0, device="cuda")
    ws = torch.full((cdsl.cdsl_tree_attention_workspace(c.c, T, H),), 255, dtype=torch.uint8, device="cuda")
    st = status()
    cdsl.cdsl_tree_attention(c.c, layer, q, ints(*lens), mask.cuda(), out, ws, scale=scale,
                             max_len=max(lens) if max_len is None else max_len, nodes=ints(*nodes), lse=lse,
                             status=st, **kw)
    torch.cuda.synchronize()
    assert int(st) == cdsl.CDSL_OK
    return out, lse


def check(c, layer, q, lens, mask, nodes, scale, got):
    out, lse, s_abs, v_abs = ref.attention(c, layer, q, lens, mask, nodes, scale)
    e, el = ref.bounds(out, s_abs, v_abs, q.shape[3], max(lens) + q.shape[1], q.dtype)
    nan = torch.isnan(out)
    assert torch.equal(torch.isnan(got[0]), nan)
    d = torch.where(nan, 0.0, got[0].double() - out).abs()
    assert (d <= torch.where(nan, 1.0, e)).all(), float((d - torch.where(nan, 1.0, e)).max())
    live = torch.isfinite(lse)
    assert torch.equal(torch.isneginf(got[1]), torch.isneginf(lse))
    d = (got[1].double() - lse).abs()[live]
    assert (d <= (el + 2.0 ** -22 * lse.abs())[live] + 1e-6).all()


SHAPES = [  # B, T, H, kvh, hd, page, lens
    (1, 1, 32, 8, 128, 64, [0]),
    (1, 1, 4, 1, 128, 16, [1]),
    (2, 1, 8, 8, 64, 32, [127, 128]),
    (3, 5, 8, 2, 128, 64, [0, 129, 300]),
    (2, 17, 12, 12, 64, 16, [200, 63]),
    (1, 33, 5, 1, 128, 128, [511]),
    (2, 64, 4, 2, 64, 256, [100, 257]),
    (1, 128, 8, 1, 128, 64, [130]),
    (5, 3, 16, 1, 128, 64, [1000, 0, 7, 640, 127]),
    (1, 7, 64, 1, 64, 64, [2050]),
]


@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
@pytest.mark.parametrize("cache", [F8, BF], ids=["f8", "bf16"])
@pytest.mark.parametrize("dtype", [F32, BF], ids=["q32", "q16"])
def test_attention_matches_64_bits(cdsl, shape, cache, dtype):
    B, T, H, kvh, hd, page, lens = shape
    c, q, mask, nodes = problem(cdsl, B, T, H, kvh, hd, page, lens, cache, dtype, seed=T + hd)
    scale = hd ** -0.5
    got = attend(cdsl, c, 1, q, lens, mask, nodes, scale)
    check(c, 1, q, lens, mask, nodes, scale, got)
    again = attend(cdsl, c, 1, q, lens, mask, nodes, scale)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])       # sums in a fixed order
    wide = attend(cdsl, c, 1, q, lens, mask, nodes, scale, max_len=c.table.shape[1] * page - T)
    check(c, 1, q, lens, mask, nodes, scale, wide)


@pytest.mark.parametrize("cache", [F8, BF], ids=["f8", "bf16"])
@pytest.mark.parametrize("dtype,B,T", [(BF, 40, 2), (BF, 24, 40), (F32, 20, 128)])
def test_attention_of_more_items_than_runs(cdsl, cache, dtype, B, T):
    """Many short sequences: most items are whole, the others are joined from the bounds between runs."""
    rng = random.Random(B)
    lens = [rng.choice([0, 1, 120, 127, 200, 300]) for _ in range(B)]
    nodes = [rng.choice([0, 1, T // 2, T, T]) for _ in range(B)]
    c, q, mask, _ = problem(cdsl, B, T, 8, 8, 64, 32, lens, cache, dtype, nodes=nodes, seed=B)
    got = attend(cdsl, c, 1, q, lens, mask, nodes, 0.125)
    pick = rng.sample(range(B), 5)
    some = copy.copy(c)
    some.table = c.table[pick]
    check(some, 1, q[pick], [lens[b] for b in pick], mask[pick], [nodes[b] for b in pick], 0.125,
          (got[0][pick], got[1][pick]))
    each = [attend(cdsl, part, 1, q[b:b + 1], lens[b:b + 1], mask[b:b + 1], nodes[b:b + 1], 0.125)[0]
            for b, part in ((b, alone(c, b)) for b in range(B))]
    far = (got[0].float() - torch.cat(each).float()).abs().max()      # other runs: other roundings
    assert far <= (2.0 ** -6 if dtype is BF else 2.0 ** -14) * got[0].float().abs().max()


def alone(c, b):
    part = copy.copy(c)
    part.table = c.table[b:b + 1].contiguous()
    part.c = c.c.at(part.table)
    return part


@pytest.mark.parametrize("cache", [F8, BF], ids=["f8", "bf16"])
@pytest.mark.parametrize("dtype", [F32, BF], ids=["q32", "q16"])
def test_attention_of_ragged_trees_and_empty_rows(cdsl, cache, dtype):
    """Fewer nodes than T (none too), masks without a bit, masks that see later nodes, no cached tokens."""
    lens, nodes = [0, 0, 140, 3, 128], [9, 0, 4, 21, 1]
    c, q, mask, _ = problem(cdsl, 5, 21, 8, 2, 128, 16, lens, cache, dtype, nodes=nodes, seed=3)
    mask[0, 2] = 0                                   # sees nothing at all
    mask[0, 3] = 0x1ff                               # sees every node
    mask[2, 1] = 0                                   # sees the cached tokens alone
    mask[3, 5] = (1 << 20) | 1                       # some node after it
    got = attend(cdsl, c, 1, q, lens, mask, nodes, 0.1)
    check(c, 1, q, lens, mask, nodes, 0.1, got)
    assert (got[0][0, 2] == 0).all() and (got[0][1] == 0).all() and (got[0][2, 4:] == 0).all()


@pytest.mark.parametrize("cache", [F8, BF], ids=["f8", "bf16"])
@pytest.mark.parametrize("dtype", [F32, BF], ids=["q32", "q16"])
def test_attention_keeps_what_is_not_finite_apart(cdsl, cache, dtype):
    """A node whose K or V is not finite gives NaN to the nodes that see it and to no other; so does a query."""
    lens = [130, 40]
    c, q, mask, nodes = problem(cdsl, 2, 6, 4, 2, 64, 32, lens, cache, dtype, kind="star", seed=4)
    k = torch.randn((2, 6, 2, 64), device="cuda")
    v = torch.randn((2, 6, 2, 64), device="cuda")
    k[0, 2, 0, 5], v[0, 3, 1, 6], v[1, 4, 0, 7] = float("nan"), float("inf"), float("nan")
    cdsl.cdsl_kv_write(c.c, 1, k, v, ints(*lens))
    q[1, 1, 3, 2] = float("nan")
    got = attend(cdsl, c, 1, q, lens, mask, nodes, 0.125)
    check(c, 1, q, lens, mask, nodes, 0.125, got)
    bad = torch.isnan(got[0]).all(-1)
    want = torch.zeros((2, 6, 4), dtype=torch.bool, device="cuda")
    want[0, 2, :2] = want[0, 3, 2:] = want[1, 4, :2] = want[1, 1, 3] = True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("cache", [F8, BF], ids=["f8", "bf16"])
@pytest.mark.parametrize("dtype", [F32, BF], ids=["q32", "q16"])
def test_attention_with_peaked_scores_and_uneven_values(cdsl, cache, dtype):
    """Scores of standard deviation 25 that rise along the sequence, so that the running maximum moves in every
    chunk, with values whose sizes differ by factors of a thousand between tokens."""
    B, T, H, kvh, hd, lens = 1, 4, 4, 1, 128, [900]
    c, q, mask, nodes = problem(cdsl, B, T, H, kvh, hd, 64, lens, cache, dtype, seed=5)
    g = torch.Generator().manual_seed(6)
    n = lens[0] + T
    ramp = torch.linspace(0.0, 1.0, n)[None, :, None, None]
    k = (torch.randn((1, n, 1, hd), generator=g) + q[0, 0, 0].float().cpu() * ramp * 3).to(BF).cuda()
    v = (torch.randn((1, n, 1, hd), generator=g) * 10.0 ** (3 * torch.rand((1, n, 1, 1), generator=g))).to(BF).cuda()
    cdsl.cdsl_kv_write(c.c, 1, k, v, ints(0))
    got = attend(cdsl, c, 1, q, lens, mask, nodes, 0.25)
    check(c, 1, q, lens, mask, nodes, 0.25, got)


@pytest.mark.parametrize("dtype", [F32, BF], ids=["q32", "q16"])
def test_attention_takes_strides_and_streams(cdsl, dtype):
    """Queries as a slice of a fused projection, off 16 bytes too; output in another order; a stream that is
    not the tensors' own; a captured call replayed at other lengths."""
    lens, scale = [70, 200], 0.1
    c, q0, mask, nodes = problem(cdsl, 2, 5, 8, 4, 64, 32, lens, F8, dtype, seed=7)
    for offset in (0, 3):
        fused = torch.zeros((2, 5, 8 * 64 * 2 + offset), dtype=dtype, device="cuda")
        q = fused[..., offset:offset + 512].view(2, 5, 8, 64)
        q.copy_(q0)
        out = torch.zeros((8, 2, 5, 64 + offset), dtype=dtype, device="cuda")[..., offset:].permute(1, 2, 0, 3)
        got = attend(cdsl, c, 1, q, lens, mask, nodes, scale, out=out)
        check(c, 1, q, lens, mask, nodes, scale, got)
    out, ws = torch.empty_like(q0), torch.empty(cdsl.cdsl_tree_attention_workspace(c.c, 5, 8), dtype=torch.uint8,
                                                device="cuda")
    dl, dm = ints(*lens), mask.cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call = lambda s=None: cdsl.cdsl_tree_attention(c.c, 1, q0, dl, dm, out, ws, scale=scale, max_len=200, stream=s)  # noqa: E731
    call(side.cuda_stream)
    side.synchronize()
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    out.zero_()
    graph.replay()
    assert torch.equal(out, first)
    dl.copy_(ints(20, 199))
    cdsl.cdsl_kv_write(c.c, 1, torch.ones((2, 5, 4, 64), dtype=BF, device="cuda"),
                       torch.ones((2, 5, 4, 64), dtype=BF, device="cuda"), dl)
    graph.replay()
    want = ref.attention(c, 1, q0, [20, 199], mask, [5, 5], scale)
    e, _ = ref.bounds(want[0], want[2], want[3], 64, 205, dtype)
    assert ((out.double() - want[0]).abs() <= e).all()


@pytest.mark.parametrize("dtype", [F32, BF], ids=["q32", "q16"])
def test_attention_past_32_bits(cdsl, dtype):
    """A layer of 2^31 codes and more, pages at its end, in the second layer of the pool."""
    n_pages, kvh, page, hd = 4200, 8, 256, 128            # 2.2 GB a layer
    table = torch.tensor([[4199, 0, 4198]], dtype=torch.int32, device="cuda")
    cache = cdsl.KvCache.empty(2, n_pages, kvh, page, hd, table)
    c = object.__new__(ref.Cache)
    c.c, c.table, c.page, c.layers = cache, table, page, 2
    g = torch.Generator().manual_seed(8)
    n, T, lens = 600, 3, [597]
    cdsl.cdsl_kv_write(cache, 1, randn((1, n, kvh, hd), g, BF), randn((1, n, kvh, hd), g, BF), ints(0))
    q = randn((1, T, 16, hd), g, dtype, rows=False)
    mask = cdsl.cdsl_tree_mask([0, 0, 1])[0][None]
    got = attend(cdsl, c, 1, q, lens, mask, [T], hd ** -0.5)
    check(c, 1, q, lens, mask, [T], hd ** -0.5, got)


@pytest.mark.parametrize("dtype", [F32, BF], ids=["q32", "q16"])
def test_attention_latches_lengths_and_pages_out_of_range(cdsl, dtype):
    c, q, mask, nodes = problem(cdsl, 2, 3, 4, 2, 64, 16, [100, 50], F8, dtype, seed=9)
    out, st = torch.empty_like(q), status()
    ws = torch.empty(cdsl.cdsl_tree_attention_workspace(c.c, 3, 4), dtype=torch.uint8, device="cuda")
    for lens in ([101, 50], [-1, 50]):
        st.zero_()
        cdsl.cdsl_tree_attention(c.c, 1, q, ints(*lens), mask.cuda(), out, ws, scale=0.1, max_len=100, status=st)
        assert int(st) == cdsl.CDSL_ERANGE
        want = ref.attention(c, 1, q, [min(100, max(0, x)) for x in lens], mask, [3, 3], 0.1)[0]
        if lens[0] > 0:
            assert ((out.double() - want).abs() < 0.05).all()
    table = c.table.clone()
    table[0, 2], table[1, 0] = -1, 1 << 22              # slots 32..47 of the first, 0..15 of the second
    st.zero_()
    cdsl.cdsl_tree_attention(c.c.at(table), 1, q, ints(100, 50), mask.cuda(), out, ws, scale=0.1, max_len=100, status=st)
    assert int(st) == cdsl.CDSL_ERANGE and torch.isfinite(out).all()
    for b, (first, n, total) in enumerate(((32, 16, 103), (0, 16, 53))):   # the same without those slots
        k, v = c.values(1, b, 0, total)
        keep = torch.ones(total, dtype=torch.bool, device="cuda")
        keep[first:first + n] = False
        for t in range(3):
            see = keep.clone()
            see[total - 3:] &= torch.tensor(ref.bits_of(mask, b, t, 3), dtype=torch.bool, device="cuda")
            for h in range(4):
                s = k[see][:, h // 2] @ q[b, t, h].double() * 0.1
                assert ((out[b, t, h].double() - torch.softmax(s, 0) @ v[see][:, h // 2]).abs() < 0.1).all()


# ------------------------------------------------------------------------------ validation

def verify_inputs(B, T, V, dtype, drafts, temperature, seed, nodes=None, spread=2.0):
    rng = random.Random(seed)
    g = torch.Generator().manual_seed(seed)
    logits = (torch.randn((B, T, V), generator=g) * spread).to(dtype)
    near = (logits.float() + 0.7 * torch.randn((B, T, V), generator=g)).to(dtype)
    parents = [ref.tree(rng.choice(["random", "chain", "star"]), T, rng) for _ in range(B)]
    tokens = torch.zeros((B, T), dtype=torch.int32)
    for b in range(B):
        for i in range(1, T):
            row = near[b, parents[b][i]].float()
            if drafts:
                tokens[b, i] = int(torch.multinomial(torch.softmax(row / (temperature or 1.0), 0), 1, generator=g))
            else:
                tokens[b, i] = int(row.topk(min(V, 4)).indices[rng.randrange(min(V, 4))])
    u, u_last = torch.rand((B, T), generator=g), torch.rand(B, generator=g)
    return logits, near if drafts else None, tokens, parents, u, u_last


def run_verify(cdsl, logits, draft, tokens, parents, u, u_last, temperature, nodes=None):
    B, T, V = logits.shape
    path, emitted = (torch.full((B, T), 5, dtype=torch.int32, device="cuda") for _ in range(2))
    n, st = torch.full((B,), 5, dtype=torch.int32, device="cuda"), status()
    cdsl.cdsl_tree_verify(logits.cuda(), tokens.cuda(), torch.tensor(parents, dtype=torch.int32, device="cuda"), u.cuda(),
                          u_last.cuda(), path, n, emitted, draft_logits=None if draft is None else draft.cuda(),
                          temperature=temperature, nodes=None if nodes is None else ints(*nodes), status=st)
    return path.cpu(), n.cpu().tolist(), emitted.cpu(), int(st)


# Decisions nearer than this to their bound may go either way: the weights' error, a few roundings of 2^-24
# and a 2^-31 for each token of the vocabulary, is below 1e-5 for the vocabularies here.
NEAR = 3e-5


@pytest.mark.parametrize("B,T,V", [(3, 1, 1), (4, 5, 7), (6, 17, 512), (2, 33, 31999), (3, 49, 4097), (2, 128, 1000)])
@pytest.mark.parametrize("dtype", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("drafts,temperature", [(False, 1.0), (False, 0.5), (True, 1.0), (True, 0.8), (False, 0.0)])
def test_verify_matches_64_bits(cdsl, B, T, V, dtype, drafts, temperature):
    logits, draft, tokens, parents, u, u_last = verify_inputs(B, T, V, dtype, drafts, temperature, seed=T + V)
    nodes = [T - (b * 5) % T for b in range(B)]
    if T > 1:
        nodes[-1] = 0
    path, n, emitted, st = run_verify(cdsl, logits, draft, tokens, parents, u, u_last, temperature, nodes)
    assert st == cdsl.CDSL_OK
    compared = 0
    for b in range(B):
        p, e, margin = ref.verify(logits[b], None if draft is None else draft[b], tokens[b].tolist(), parents[b],
                                  nodes[b], u[b].tolist(), float(u_last[b]), temperature)
        assert len(p) == n[b] or margin < NEAR
        if margin < NEAR:
            continue
        compared += 1
        assert path[b].tolist() == p + [-1] * (T - len(p))
        assert emitted[b].tolist() == e + [-1] * (T - len(e))
    assert compared >= B // 2
    again = run_verify(cdsl, logits, draft, tokens, parents, u, u_last, temperature, nodes)
    assert torch.equal(again[0], path) and torch.equal(again[2], emitted)


@pytest.mark.parametrize("B,T,V", [(1, 9, 32000), (2, 3, 163841), (40, 6, 4999), (100, 4, 20500), (160, 3, 700)])
@pytest.mark.parametrize("drafts", [False, True])
def test_verify_by_any_number_of_blocks(cdsl, B, T, V, drafts):
    """Batches and vocabularies that give a sequence eight blocks, two and one, and rows beyond the registers."""
    logits, draft, tokens, parents, u, u_last = verify_inputs(B, T, V, BF, drafts, 1.0, seed=B + V, spread=5.0)
    path, n, emitted, st = run_verify(cdsl, logits, draft, tokens, parents, u, u_last, 1.0)
    assert st == cdsl.CDSL_OK
    compared = 0
    for b in range(B):
        p, e, margin = ref.verify(logits[b], None if draft is None else draft[b], tokens[b].tolist(), parents[b], T,
                                  u[b].tolist(), float(u_last[b]), 1.0)
        if margin >= NEAR:
            compared += 1
            assert path[b].tolist() == p + [-1] * (T - len(p)) and emitted[b].tolist() == e + [-1] * (T - len(e))
    assert compared > 0


@pytest.mark.parametrize("drafts", [False, True])
def test_verify_draws_from_the_targets_distribution(cdsl, drafts):
    """The first emitted token over 40,960 walks of one small tree has the target's probabilities: a chi-square
    statistic of 7 degrees of freedom stays below 29.9 (probability 1e-4)."""
    V, T, B, rounds = 8, 5, 1024, 40
    g = torch.Generator().manual_seed(11)
    target, near = torch.randn(V, generator=g) * 1.5, torch.randn(V, generator=g) * 1.5
    p, q = torch.softmax(target.double(), 0), torch.softmax(near.double(), 0)
    parents = [[0, 0, 0, 0, 1]] * B
    counts = torch.zeros(V)
    for _ in range(rounds):
        if drafts:
            tokens = torch.multinomial(q, B * T, replacement=True, generator=g).view(B, T).int()
        else:
            tokens = torch.tensor([0, 3, 1, 6, 2], dtype=torch.int32).expand(B, T).contiguous()
        u, u_last = torch.rand((B, T), generator=g), torch.rand(B, generator=g)
        _, n, emitted, _ = run_verify(cdsl, target.expand(B, T, V).contiguous(),
                                      near.expand(B, T, V).contiguous() if drafts else None, tokens, parents, u, u_last, 1.0)
        counts += torch.bincount(emitted[:, 0].long(), minlength=V)
    want = p * B * rounds
    assert float(((counts - want) ** 2 / want).sum()) < 29.9


@pytest.mark.parametrize("dtype", [F32, BF], ids=["f32", "bf16"])
def test_verify_with_masked_logits_and_bad_rows(cdsl, dtype):
    """-inf logits are never drawn; rows with NaN, +inf or nothing finite end the walk without a token; tokens
    outside the vocabulary and parents out of order are not taken."""
    V, T = 300, 3
    logits = torch.full((8, T, V), float("-inf"), dtype=dtype)
    logits[:, :, 7] = -1e30                                   # the only token there is
    tokens = torch.tensor([[0, 7, 7]] * 8, dtype=torch.int32)
    parents = [[0, 0, 1]] * 8
    parents[6] = [0, -1, 1]                                   # node 1 has no parent, nor 2 a path to the root
    parents[7] = [0, 2, 0]                                    # node 1's parent comes after it
    logits[1, 1] = float("-inf")
    logits[2, 1, 3] = float("nan")
    logits[3, 2, 9] = float("inf")
    tokens[4, 1], tokens[5, 2] = V, -1
    u, u_last = torch.full((8, T), 0.999), torch.full((8,), 0.99999994)
    path, n, emitted, st = run_verify(cdsl, logits, None, tokens, parents, u, u_last, 1.0)
    assert st in (cdsl.CDSL_ENONFINITE, cdsl.CDSL_ERANGE)
    assert n == [3, 2, 2, 3, 1, 2, 1, 2]
    assert emitted.tolist() == [[7, 7, 7], [7, -1, -1], [7, -1, -1], [7, 7, -1], [7, -1, -1], [7, 7, -1], [7, -1, -1],
                                [7, 7, -1]]
    assert path[7].tolist() == [0, 2, -1]
    draft = torch.zeros_like(logits)
    draft[0, 0, 0] = float("nan")
    path, n, emitted, st = run_verify(cdsl, logits[:1], draft[:1], tokens[:1], parents[:1], u[:1], u_last[:1], 1.0)
    assert st == cdsl.CDSL_ENONFINITE and n == [1] and emitted.tolist() == [[-1, -1, -1]]


def test_verify_edges_of_the_random_numbers(cdsl):
    """u = 0 takes every child with a weight and no other; u_last = 0 draws the first token with one, u_last just
    below 1 the last."""
    logits = torch.zeros((2, 2, 10))
    logits[:, :, 0] = logits[:, :, 9] = float("-inf")
    tokens = torch.tensor([[0, 4], [0, 9]], dtype=torch.int32)
    top = torch.tensor([1.0]).nextafter(torch.tensor([0.0]))
    path, n, emitted, st = run_verify(cdsl, logits, None, tokens, [[0, 0]] * 2, torch.zeros((2, 2)),
                                      torch.stack([torch.zeros(1), top])[:, 0], 1.0)
    assert n == [2, 1] and emitted.tolist() == [[4, 1], [8, -1]] and st == cdsl.CDSL_OK
    # rejected drafts that were all the target has: nothing is left but what it was
    logits = torch.full((1, 2, 4), float("-inf"))
    logits[..., 2] = 0
    path, n, emitted, st = run_verify(cdsl, logits, logits.clone(), torch.tensor([[0, 1]], dtype=torch.int32), [[0, 0]],
                                      torch.full((1, 2), 0.5), torch.full((1,), 0.5), 1.0)
    assert n == [1] and emitted.tolist() == [[2, -1]]


def test_verify_takes_strided_logits(cdsl):
    logits, _, tokens, parents, u, u_last = verify_inputs(3, 6, 101, BF, False, 1.0, seed=12)
    want = run_verify(cdsl, logits, None, tokens, parents, u, u_last, 1.0)
    wide = torch.full((6, 3, 107), float("nan"), dtype=BF)
    wide[..., 3:104] = logits.transpose(0, 1)
    got = run_verify(cdsl, wide.cuda()[..., 3:104].transpose(0, 1), None, tokens, parents, u, u_last, 1.0)
    assert torch.equal(got[0], want[0]) and got[1] == want[1] and torch.equal(got[2], want[2])


@pytest.mark.parametrize("dtype", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [9, 1001, 20003])
def test_verify_by_any_alignment(cdsl, dtype, V):
    """Rows that start at 16 bytes are read 16 bytes at a time, to an end anywhere; others by single values."""
    logits, draft, tokens, parents, u, u_last = verify_inputs(4, 7, V, dtype, True, 1.0, seed=V, spread=4.0)
    up = -(-V // 8) * 8
    want = None
    for pitch, first in ((V, 0), (up, 0), (up + 16, 8), (up + 8, 1)):
        wide = [torch.full((4, 7, pitch), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
        for w, x in zip(wide, (logits, draft)):
            w[..., first:first + V] = x.cuda()
        path, n, emitted, st = run_verify(cdsl, wide[0][..., first:first + V], wide[1][..., first:first + V], tokens, parents,
                                          u, u_last, 1.0)
        got = path.tolist(), n, emitted.tolist(), st
        assert st == cdsl.CDSL_OK and got == (want or got)
        want = got
    assert max(want[1]) > 1 and all(0 <= e[m - 1] < V for e, m in zip(want[2], want[1]))
