"""The 4-bit cache (include/cdsl_tree.h) against plain 64-bit implementations: write, read, commit and the tree attention.
Pools start full of garbage (scales that are not finite among it), pages are in random order."""
import copy
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import i4_reference as i4  # noqa: E402
import tree_reference as ref  # noqa: E402
from i4_reference import check  # noqa: E402
from test_gpu_tree import alone, attend, cdsl, ints, randn, status  # noqa: E402,F401
from tree_reference import BF, F32  # noqa: E402


# ------------------------------------------------------------------------------ cache

@pytest.mark.parametrize("kvh,hd,page", [(8, 128, 64), (12, 64, 16), (1, 128, 256), (3, 64, 32)])
@pytest.mark.parametrize("T,value", [(1, BF), (17, F32), (67, BF)])
def test_write_and_read(cdsl, kvh, hd, page, T, value):
    """Rows come back as their definition says, to the bit, at odd starts, ragged counts and with rows of zeros, ties of the
    rounding, huge, tiny and non-finite values; no other row of the pool changes."""
    g = torch.Generator().manual_seed(hd + T)
    B, start = 4, [0, 5, page - 1, 131]
    c = i4.Cache(B, max(start) + T, kvh, hd, page, layers=2, seed=T)
    k, v = (randn((B, T, kvh, hd), g, value) for _ in range(2))
    k[0, 0, 0] = 0
    v[0, 0, 0] *= 2.0 ** 110
    k[1, 0, 0] *= 2.0 ** -118
    v[1, 0, 0] = 2.0 ** -130                      # a subnormal row
    k[2, 0, 0, :32] = torch.arange(32).float() / 2 - 8.5    # ties, of a scale of 1.25 (8.5 / 7 = 1.214)
    v[2, 0, 0, :32] = torch.arange(32).float() * 0.5625 - 7.875     # of a scale of 1.125
    v[2, 0, 0, 32:34] = torch.tensor([7 * 1.0625, 1.0])     # the scale itself in the middle: to even, 1
    k[3, 0, 0, 3] = float("nan")
    v[3, 0, 0, hd - 1] = float("-inf")
    if T > 1:
        k[3, 1, 0, 7], v[3, 1, 0, 7] = 2.0 ** 120, 2.0 ** 119
    count = [T, (T + 1) // 2, T, max(1, T - 3)]
    before, before_scale = c.c.pool.clone(), c.c.scale.clone()
    st = status()
    cdsl.cdsl_kv_write(c.c, 1, k, v, ints(*start), ints(*count), status=st)
    touched = torch.zeros(c.c.scale.shape[:5], dtype=torch.bool, device="cuda")
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
            want = i4.quantised(x[b, :n])
            assert torch.equal(torch.nan_to_num(stored[j], 1e9), torch.nan_to_num(want, 1e9))
            assert torch.equal(torch.nan_to_num(outs[0][j][b, :n].double(), 1e9), torch.nan_to_num(want, 1e9))
            assert torch.equal(torch.nan_to_num(outs[1][j][b, :n].double(), 1e9), torch.nan_to_num(want, 1e9))
            assert (outs[0][j][b, n:] == 0).all() and (outs[1][j][b, n:] == 0).all()
    assert torch.equal(c.c.pool[~touched], before[~touched])
    assert torch.equal(c.c.scale.view(torch.int16)[~touched], before_scale.view(torch.int16)[~touched])
    assert int(st) == cdsl.CDSL_OK


def test_every_code_of_many_scales(cdsl):
    """Values at and next to every tie between codes, in float32, for scales of all 8 fractions: to the bit."""
    rows = []
    for m in range(8, 16):
        for e in (-3.0, 0.0, 5.0):
            s = m / 8 * 2.0 ** e
            ties = torch.tensor([(2 * c + 1) / 2 * s for c in range(-7, 7)])
            for x in (ties, torch.nextafter(ties, torch.tensor(9e9)), torch.nextafter(ties, torch.tensor(-9e9))):
                r = torch.zeros(64)
                r[:14], r[14], r[32:46], r[46] = x, 7 * s, -x, -7 * s
                rows.append(r)
    k = torch.stack(rows)[None, :, None].cuda()
    c = i4.Cache(1, k.shape[1], 1, 64, 16)
    cdsl.cdsl_kv_write(c.c, 0, k, -k, ints(0))
    for got, x in zip(c.values(0, 0, 0, k.shape[1]), (k, -k)):
        assert torch.equal(got, i4.quantised(x[0]))


@pytest.mark.parametrize("value", [BF, F32])
def test_write_takes_strided_and_unaligned_rows(cdsl, value):
    g = torch.Generator().manual_seed(1)
    B, T, kvh, hd = 2, 9, 4, 64
    for offset in (0, 8, 1):
        fused = randn((B, T, 3 * kvh * hd + offset), g, value, rows=False)
        k = fused[..., offset:offset + kvh * hd].view(B, T, kvh, hd)
        v = randn((kvh, T, B, hd), g, value).permute(2, 1, 0, 3)
        c = i4.Cache(B, T, kvh, hd, 16, seed=offset)
        cdsl.cdsl_kv_write(c.c, 0, k, v, ints(0, 0))
        for b in range(B):
            for got, x in zip(c.values(0, b, 0, T), (k, v)):
                assert torch.equal(got, i4.quantised(x[b]))


def test_write_and_read_past_the_pages_latch_erange(cdsl):
    c = i4.Cache(2, 32, 2, 64, 16)
    k = torch.ones((2, 20, 2, 64), dtype=BF, device="cuda")
    st, before = status(), c.c.scale.view(torch.int16).clone()
    cdsl.cdsl_kv_write(c.c, 0, k, k, ints(-20, 32), status=st)      # slots below 0 and past the table
    assert int(st) == cdsl.CDSL_ERANGE and torch.equal(c.c.scale.view(torch.int16), before)
    out = torch.full((1, 2, 20, 2, 64), 3.0, dtype=BF, device="cuda")
    st.zero_()
    cdsl.cdsl_kv_read(c.c, 0, ints(-20, 32), out, out.clone(), status=st)
    assert int(st) == cdsl.CDSL_ERANGE and (out == 0).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("T", [1, 7, 128])
def test_commit_moves_the_path(cdsl, hd, T):
    rng = random.Random(T)
    B, kvh, page, layers = 4, 3, 16, 3
    c = i4.Cache(B, 50 + T, kvh, hd, page, layers=layers, seed=T)
    g = torch.Generator().manual_seed(T)
    lens = [0, 15, 33, 50]
    for l in range(layers):
        cdsl.cdsl_kv_write(c.c, l, randn((B, T, kvh, hd), g, BF), randn((B, T, kvh, hd), g, BF), ints(*lens))
    paths = [[0], list(range(T)), [0] + sorted(rng.sample(range(1, T), (T - 1) // 2)), []]
    path = torch.full((B, T), -1, dtype=torch.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    want = [[c.values(l, b, lens[b], T) for b in range(B)] for l in range(layers)]
    new, st = ints(*[-5] * B), status()
    cdsl.cdsl_kv_commit(c.c, ints(*lens), path.cuda(), ints(*[len(p) for p in paths]), new, status=st)
    assert new.tolist() == [a + len(p) for a, p in zip(lens, paths)] and int(st) == cdsl.CDSL_OK
    for l in range(layers):
        for b, p in enumerate(paths):
            for got, x in zip(c.values(l, b, lens[b], max(1, len(p))), want[l][b]):
                assert torch.equal(got[:len(p)], x[p])


# ------------------------------------------------------------------------------ attention

def problem(cdsl, B, T, H, kvh, hd, page, lens, dtype, kind="random", nodes=None, seed=0, layers=2):
    rng = random.Random(seed)
    g = torch.Generator().manual_seed(seed)
    nodes = nodes or [T] * B
    n = max(lens) + T
    c = i4.Cache(B, n, kvh, hd, page, layers=layers, seed=seed)
    cdsl.cdsl_kv_write(c.c, layers - 1, randn((B, n, kvh, hd), g, BF), randn((B, n, kvh, hd), g, BF), ints(*[0] * B),
                       ints(*[a + b for a, b in zip(lens, nodes)]))
    mask = torch.stack([cdsl.cdsl_tree_mask(ref.tree(kind, T, rng))[0] for _ in range(B)])
    q = randn((B, T, H, hd), g, dtype, rows=False)
    return c, q, mask, nodes


SHAPES = [  # B, T, H, kvh, hd, page, lens
    (1, 1, 32, 8, 128, 64, [0]),
    (1, 1, 4, 1, 128, 16, [1]),
    (2, 1, 8, 8, 64, 32, [127, 128]),
    (3, 5, 8, 2, 128, 64, [0, 129, 300]),
    (2, 2, 16, 2, 64, 64, [511, 63]),
    (1, 3, 10, 2, 128, 128, [700]),
    (2, 17, 12, 12, 64, 16, [200, 63]),
    (2, 6, 10, 2, 128, 32, [95, 513]),
    (1, 33, 5, 1, 128, 128, [511]),
    (2, 64, 4, 2, 64, 256, [100, 257]),
    (1, 128, 8, 1, 128, 64, [130]),
    (5, 3, 16, 1, 128, 64, [1000, 0, 7, 640, 127]),
    (1, 7, 64, 1, 64, 64, [2050]),
]
DTYPES = pytest.mark.parametrize("dtype", [F32, BF], ids=["q32", "q16"])


@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
@DTYPES
def test_attention_matches_64_bits(cdsl, shape, dtype):
    B, T, H, kvh, hd, page, lens = shape
    c, q, mask, nodes = problem(cdsl, B, T, H, kvh, hd, page, lens, dtype, seed=T + hd)
    scale = hd ** -0.5
    got = attend(cdsl, c, 1, q, lens, mask, nodes, scale)
    check(c, 1, q, lens, mask, nodes, scale, got)
    again = attend(cdsl, c, 1, q, lens, mask, nodes, scale)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])       # sums in a fixed order
    wide = attend(cdsl, c, 1, q, lens, mask, nodes, scale, max_len=c.table.shape[1] * page - T)
    check(c, 1, q, lens, mask, nodes, scale, wide)


@pytest.mark.parametrize("dtype,B,T", [(BF, 40, 2), (BF, 24, 40), (F32, 20, 128)])
def test_attention_of_more_items_than_runs(cdsl, dtype, B, T):
    """Many short sequences: most items are whole, the others are joined from the bounds between runs."""
    rng = random.Random(B)
    lens = [rng.choice([0, 1, 120, 127, 200, 300]) for _ in range(B)]
    nodes = [rng.choice([0, 1, T // 2, T, T]) for _ in range(B)]
    c, q, mask, _ = problem(cdsl, B, T, 8, 8, 64, 32, lens, dtype, nodes=nodes, seed=B)
    got = attend(cdsl, c, 1, q, lens, mask, nodes, 0.125)
    pick = rng.sample(range(B), 5)
    some = copy.copy(c)
    some.table = c.table[pick]
    check(some, 1, q[pick], [lens[b] for b in pick], mask[pick], [nodes[b] for b in pick], 0.125,
          (got[0][pick], got[1][pick]))


@DTYPES
@pytest.mark.parametrize("G", [1, 4])
def test_attention_of_ragged_trees_and_empty_rows(cdsl, dtype, G):
    """Fewer nodes than T (none too), masks without a bit, masks that see later nodes, no cached tokens."""
    lens, nodes = [0, 0, 140, 3, 128], [9, 0, 4, 21, 1]
    c, q, mask, _ = problem(cdsl, 5, 21, 2 * G, 2, 128, 16, lens, dtype, nodes=nodes, seed=3)
    mask[0, 2] = 0                                   # sees nothing at all
    mask[0, 3] = 0x1ff                               # sees every node
    mask[2, 1] = 0                                   # sees the cached tokens alone
    mask[3, 5] = (1 << 20) | 1                       # some node after it
    got = attend(cdsl, c, 1, q, lens, mask, nodes, 0.1)
    check(c, 1, q, lens, mask, nodes, 0.1, got)
    assert (got[0][0, 2] == 0).all() and (got[0][1] == 0).all() and (got[0][2, 4:] == 0).all()


@DTYPES
@pytest.mark.parametrize("G", [1, 2, 8])
def test_attention_keeps_what_is_not_finite_apart(cdsl, dtype, G):
    """A node whose K or V is not finite gives NaN to the nodes that see it and to no other; so does a query."""
    lens = [130, 40]
    H = 2 * G
    c, q, mask, nodes = problem(cdsl, 2, 6, H, 2, 64, 32, lens, dtype, kind="star", seed=4)
    k = torch.randn((2, 6, 2, 64), device="cuda")
    v = torch.randn((2, 6, 2, 64), device="cuda")
    k[0, 2, 0, 5], v[0, 3, 1, 6], v[1, 4, 0, 7] = float("nan"), float("inf"), float("nan")
    cdsl.cdsl_kv_write(c.c, 1, k, v, ints(*lens))
    q[1, 1, H - 1, 2] = float("nan")
    got = attend(cdsl, c, 1, q, lens, mask, nodes, 0.125)
    check(c, 1, q, lens, mask, nodes, 0.125, got)
    bad = torch.isnan(got[0]).all(-1)
    want = torch.zeros((2, 6, H), dtype=torch.bool, device="cuda")
    want[0, 2, :G] = want[0, 3, G:] = want[1, 4, :G] = want[1, 1, H - 1] = True
    assert torch.equal(bad, want)


@DTYPES
@pytest.mark.parametrize("T,G", [(1, 4), (4, 4), (16, 4)])
def test_attention_with_peaked_scores_and_uneven_values(cdsl, dtype, T, G):
    """Scores of standard deviation 25 that rise along the sequence, so that the running maximum moves in every
    chunk, with values whose sizes differ by factors of a thousand between tokens."""
    H, hd, lens = G, 128, [900]
    c, q, mask, nodes = problem(cdsl, 1, T, H, 1, hd, 64, lens, dtype, seed=5)
    g = torch.Generator().manual_seed(6)
    n = lens[0] + T
    ramp = torch.linspace(0.0, 1.0, n)[None, :, None, None]
    k = (torch.randn((1, n, 1, hd), generator=g) + q[0, 0, 0].float().cpu() * ramp * 3).to(BF).cuda()
    v = (torch.randn((1, n, 1, hd), generator=g) * 10.0 ** (3 * torch.rand((1, n, 1, 1), generator=g))).to(BF).cuda()
    cdsl.cdsl_kv_write(c.c, 1, k, v, ints(0))
    got = attend(cdsl, c, 1, q, lens, mask, nodes, 0.25)
    check(c, 1, q, lens, mask, nodes, 0.25, got)


@DTYPES
@pytest.mark.parametrize("T", [1, 3, 20])
def test_small_values_keep_their_weights_beside_huge_ones(cdsl, dtype, T):
    """Slots without weight have values 2^60 times the others', or 2^60 times smaller in one group than in the next."""
    H, hd, lens = 4, 64, [300]
    c, q, mask, nodes = problem(cdsl, 1, T, H, 1, hd, 64, lens, dtype, kind="chain", seed=8)
    n = lens[0] + T
    g = torch.Generator().manual_seed(9)
    q[:] = 1.0
    k = torch.full((1, n, 1, hd), 2.0)
    k[:, 7::11] = -100.0                             # no weight: the scores are 1600 below
    v = torch.randn((1, n, 1, hd), generator=g) * 2.0 ** -30
    v[:, 7::11] *= 2.0 ** 60
    v[..., 32:] *= 2.0 ** -60
    cdsl.cdsl_kv_write(c.c, 1, k.cuda(), v.cuda(), ints(0))
    got, lse = attend(cdsl, c, 1, q, lens, mask, nodes, 0.125)
    vv = c.values(1, 0, 0, n)[1][:, 0]
    for t in range(T):
        see = [i for i in range(lens[0] + t + 1) if i % 11 != 7]
        want = vv[see].mean(0)
        e = vv[see].abs().amax(0) * (2.0 ** -11 if dtype is BF else 400 * 2.0 ** -23) + want.abs() * 2.0 ** -8 * (dtype is BF)
        assert ((got[0, t].double() - want).abs() <= e).all()


@DTYPES
@pytest.mark.parametrize("B,kvh,G,hd,n", [(1, 1, 4, 128, 9000), (1, 2, 1, 64, 6001), (2, 1, 12, 64, 5000), (1, 1, 16, 128, 4097)])
def test_attention_of_few_long_sequences(cdsl, dtype, B, kvh, G, hd, n):
    """Items of many runs, which blocks of several warps join."""
    lens = [n] + [n // 3] * (B - 1)
    c, q, mask, nodes = problem(cdsl, B, 1, kvh * G, kvh, hd, 64, lens, dtype, seed=n)
    got = attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)
    check(c, 1, q, lens, mask, nodes, hd ** -0.5, got)
    again = attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@DTYPES
@pytest.mark.parametrize("T", [1, 3])
def test_attention_of_runs_of_thousands_of_slots(cdsl, dtype, T):
    """64 sequences over the same 16,384 slots: a run has more slots than one chain of sums takes; their sizes rise with the
    slots, so that what comes first does not vanish beside the rest, and scores rise and fall."""
    n, H, kvh, hd, B = 16384, 32, 8, 64, 64
    one, q, mask, _ = problem(cdsl, 1, T, H, kvh, hd, 64, [n], dtype, kind="chain", seed=1)
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((1, n + T, kvh, hd), generator=g) for _ in range(2))
    v *= torch.linspace(3, 1, n + T)[None, :, None, None]
    k *= torch.linspace(0.5, 1.5, n + T)[None, :, None, None]
    cdsl.cdsl_kv_write(one.c, 1, k.cuda(), v.cuda(), ints(0))
    many = copy.copy(one)
    many.table = one.table.expand(B, -1).contiguous()
    many.c = one.c.at(many.table)
    lens, nodes = [n - 7 * b for b in range(B)], [T] * B
    qs, masks = torch.cat([q * (1 + b / 64) for b in range(B)]), mask.expand(B, -1, -1)
    got = attend(cdsl, many, 1, qs, lens, masks, nodes, 0.125)
    for b in (0, 31, 63):
        check(one, 1, qs[b:b + 1], lens[b:b + 1], mask, [T], 0.125, (got[0][b:b + 1], got[1][b:b + 1]))


@DTYPES
def test_attention_takes_strides_streams_and_graphs(cdsl, dtype):
    """Queries as a slice of a fused projection, off 16 bytes too; output in another order; a stream that is not the
    tensors' own; a captured call replayed at other lengths, two graphs with one workspace one after the other."""
    lens, scale = [70, 200], 0.1
    c, q0, mask, nodes = problem(cdsl, 2, 5, 8, 4, 64, 32, lens, dtype, seed=7)
    for offset in (0, 3):
        fused = torch.zeros((2, 5, 8 * 64 * 2 + offset), dtype=dtype, device="cuda")
        q = fused[..., offset:offset + 512].view(2, 5, 8, 64)
        q.copy_(q0)
        out = torch.zeros((8, 2, 5, 64 + offset), dtype=dtype, device="cuda")[..., offset:].permute(1, 2, 0, 3)
        got = attend(cdsl, c, 1, q, lens, mask, nodes, scale, out=out)
        check(c, 1, q, lens, mask, nodes, scale, got)
    ws = torch.empty(cdsl.cdsl_tree_attention_workspace(c.c, 5, 8), dtype=torch.uint8, device="cuda")
    dl, dm = ints(*lens), mask.cuda()
    outs = [torch.empty_like(q0) for _ in range(2)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call = lambda o, s=None: cdsl.cdsl_tree_attention(c.c, 1, q0, dl, dm, o, ws, scale=scale, max_len=200, stream=s)  # noqa: E731
    call(outs[0], side.cuda_stream)
    side.synchronize()
    want = attend(cdsl, c, 1, q0, lens, mask, nodes, scale, max_len=200)[0]
    assert torch.equal(outs[0], want)
    graphs = []
    for o in outs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(o)
    for new in ([0, 1], [64, 190]):
        dl.copy_(ints(*new))
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        want = attend(cdsl, c, 1, q0, new, mask, nodes, scale, max_len=200)[0]
        assert all(torch.equal(o, want) for o in outs)


@DTYPES
@pytest.mark.parametrize("T", [1, 30])
def test_pages_out_of_range_are_not_seen(cdsl, dtype, T):
    c, q, mask, nodes = problem(cdsl, 2, T, 8, 2, 64, 32, [300, 300], dtype, seed=11)
    bad = copy.copy(c)
    bad.table = c.table.clone()
    bad.table[0, 3], bad.table[1, 0], bad.table[1, 5] = -1, 1 << 22, -7
    bad.c = c.c.at(bad.table)
    out, ws = torch.empty_like(q), torch.empty(cdsl.cdsl_tree_attention_workspace(c.c, T, 8), dtype=torch.uint8, device="cuda")
    st = status()
    cdsl.cdsl_tree_attention(bad.c, 1, q, ints(300, 300), mask.cuda(), out, ws, scale=0.125, max_len=300, status=st)
    assert int(st) == cdsl.CDSL_ERANGE
    gone = {0: [3], 1: [0, 5]}
    for b in range(2):
        slots = [i for i in range(300 + T) if i // 32 not in gone[b]]
        k, v = (x[slots] for x in c.values(1, b, 0, 300 + T))
        for t in range(T):
            see = torch.tensor([s < 300 or bool((int(mask[b][t][0]) >> (s - 300)) & 1) for s in slots], device="cuda")
            for h in range(8):
                s = (k[see][:, h // 4] @ q[b, t, h].double()) * 0.125
                want = torch.softmax(s, 0) @ v[see][:, h // 4]
                e = v.abs().max() * (2.0 ** -10 if dtype is BF else 2.0 ** -13) + want.abs() * 2.0 ** -8
                assert ((out[b, t, h].double() - want).abs() <= e).all()
