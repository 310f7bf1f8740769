"""Tree attention (include/cdsl_tree.h) where V's sizes differ by orders of magnitude between slots: what a query gives
no weight, or does not see, takes nothing from what it does see."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import tree_reference as ref  # noqa: E402
from test_gpu_tree import attend, cdsl, ints  # noqa: E402,F401
from tree_reference import BF, F32, F8  # noqa: E402


def attention(c, layer, q, lens, mask, nodes, scale):
    """out, sum of p |v|, the largest sum of |q_d k_d| * scale, and the largest weight, in 64 bits."""
    B, T, H, hd = q.shape
    G = H // c.c.n_kv_heads
    out, size = (torch.zeros((B, T, H, hd), dtype=torch.float64, device="cuda") for _ in range(2))
    s_abs, p_top = (torch.zeros((B, T, H, 1), dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(B):
        n, m = lens[b], nodes[b]
        k, v = (x.repeat_interleave(G, 1) for x in c.values(layer, b, 0, n + m))
        see = torch.tensor([[1] * n + ref.bits_of(mask, b, t, m) for t in range(m)], dtype=torch.bool, device="cuda")
        x = torch.einsum("thd,nhd->thn", q[b, :m].double(), k) * scale
        p = torch.softmax(x.masked_fill(~see[:, None], float("-inf")), -1)
        out[b, :m], size[b, :m] = (torch.einsum("thn,nhd->thd", p, y) for y in (v, v.abs()))
        s_abs[b, :m, :, 0] = (torch.einsum("thd,nhd->thn", q[b, :m].double().abs(), k.abs()) * scale).amax(-1)
        p_top[b, :m, :, 0] = p.amax(-1)
    return out, size, s_abs, p_top


def check(c, layer, q, lens, mask, nodes, scale, got):
    """Per element. The weights' relative error is that of tree_reference.bounds, scores and 32-bit sums, and 2^-8 of
    two planes of 4 bits at worst, each weight's on its own |v|. The result's rounding is 2^-9 of it; twice that,
    as there. Where V's scales in a chunk lie within 2^8 of one another a weight may be held to a step of 2^-21 of
    the largest product of weight and scale there: as independent roundings, six standard deviations of their sum (448:
    the largest code). `s_abs` is over all slots, `2^-13` for queries to 2^-17 of the row's largest value."""
    out, size, s_abs, p_top = attention(c, layer, q, lens, mask, nodes, scale)
    hd, keys = q.shape[3], max(lens) + q.shape[1]
    dw = 2 * (hd + 4) * 2.0 ** -24 * s_abs + (keys + 16) * 2.0 ** -24
    e = dw * size
    if q.dtype is BF:
        e = (dw + 2 * 2.0 ** -13 * s_abs + 2.0 ** -8) * size + 2.0 ** -8 * out.abs()
        if c.c.pool.dtype is F8:
            top = torch.stack([largest_scale(c, layer, b, lens[b] + nodes[b]) for b in range(len(lens))])
            e = e + 6 / 12 ** 0.5 * keys ** 0.5 * 2.0 ** -21 * p_top * 448 * top[:, None, None, None]
    d = (got.double() - out).abs()
    assert torch.isfinite(got).all()
    assert (d <= e).all(), float((d / e).max())


def largest_scale(c, layer, b, n):
    """The largest scale of V that can lie within 2^8 of the smallest one."""
    slot = torch.arange(n, device="cuda")
    x = c.c.scale[layer][c.table[b][slot // c.page].long(), 1, :, slot % c.page].double()
    return torch.exp2(torch.minimum(x.amax(), x.amin() + 8) - 127)


def problem(cdsl, T, H, kvh, hd, cache, dtype, size, seed, lens=(700, 260)):
    """Queries that share a large first component, keys without it, and values of about `size`; a star of T nodes."""
    g = torch.Generator().manual_seed(seed)
    lens, B, n = list(lens), len(lens), max(lens) + T
    c = ref.Cache(B, n, kvh, hd, 64, cache, layers=2, seed=seed)
    k, v = (torch.randn((B, n, kvh, hd), generator=g) for _ in range(2))
    k[..., 0] = 0
    q = torch.randn((B, T, H, hd), generator=g)
    q[..., 0] = 8
    mask = torch.stack([cdsl.cdsl_tree_mask(ref.tree("star", T, None))[0]] * B)
    return c, q.to(dtype).cuda(), k, v * size, lens, mask, [T] * B


# 1, 4, 32 and 16 vectors a K/V head (slots as the MMA's rows), 36 and 34 (vectors as rows)
HEADS = [(1, 2, 2, 128), (1, 8, 2, 64), (8, 8, 2, 128), (8, 4, 2, 64), (9, 8, 2, 128), (17, 4, 2, 64)]
CACHES = pytest.mark.parametrize("cache", [F8, BF], ids=["f8", "bf16"])
TYPES = pytest.mark.parametrize("dtype", [F32, BF], ids=["q32", "q16"])


@pytest.mark.parametrize("T,H,kvh,hd", HEADS, ids=[str(i) for i in range(len(HEADS))])
@CACHES
@TYPES
@pytest.mark.parametrize("up", [8, 9, 20, 60])
@pytest.mark.parametrize("at", [5, 259])
def test_a_large_value_without_weight(cdsl, T, H, kvh, hd, cache, dtype, up, at):
    """One cached token's V is 2^up times the others', its weight below 2^-60."""
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, cache, dtype, 1.0, up)
    v[:, at] *= 2.0 ** up
    k[:, at] = 0
    k[:, at, :, 0] = -7 * hd ** 0.5
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(0, 0))
    check(c, 1, q, lens, mask, nodes, hd ** -0.5, attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0])


@pytest.mark.parametrize("T,H,kvh,hd", HEADS[2:], ids=[str(i) for i in range(len(HEADS) - 2)])
@CACHES
@TYPES
@pytest.mark.parametrize("up", [9, 20, 40])
def test_a_large_value_that_is_not_seen(cdsl, T, H, kvh, hd, cache, dtype, up):
    """A node's V is 2^up times the others'; its siblings' results do not depend on it."""
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, cache, dtype, 1.0, up)
    for b, n in enumerate(lens):
        v[b, n + 2] *= 2.0 ** up
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(0, 0))
    check(c, 1, q, lens, mask, nodes, hd ** -0.5, attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0])


@pytest.mark.parametrize("T,H,kvh,hd", HEADS, ids=[str(i) for i in range(len(HEADS))])
@CACHES
@TYPES
@pytest.mark.parametrize("size", [0.1, 0.01, 1e-6])
def test_a_value_of_zeros(cdsl, T, H, kvh, hd, cache, dtype, size):
    """A row of zeros has scale 1, whatever the size of the others."""
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, cache, dtype, size, 1)
    v[:, 130] = 0
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(0, 0))
    check(c, 1, q, lens, mask, nodes, hd ** -0.5, attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0])


@pytest.mark.parametrize("T,H,kvh,hd", HEADS, ids=[str(i) for i in range(len(HEADS))])
@CACHES
@TYPES
@pytest.mark.parametrize("down", [6, 24])
def test_a_small_value_with_most_of_the_weight(cdsl, T, H, kvh, hd, cache, dtype, down):
    """The first token takes most of the weight and its V is 2^-down of the others'."""
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, cache, dtype, 1.0, down)
    v[:, 0] *= 2.0 ** -down
    k[:, 0] = 0
    k[:, 0, :, 0] = hd ** 0.5
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(0, 0))
    check(c, 1, q, lens, mask, nodes, hd ** -0.5, attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0])


@pytest.mark.parametrize("T,H,kvh,hd", HEADS, ids=[str(i) for i in range(len(HEADS))])
@TYPES
@pytest.mark.parametrize("low,high", [(127, 127), (124, 131), (60, 190)])
def test_scale_bytes_of_a_bf16_cache(cdsl, T, H, kvh, hd, dtype, low, high):
    """A caller's own bf16 rows: values are code * 2^(byte - 127) for every kernel, as for cdsl_kv_read. (K's bytes stay
    within 2^4, or one key takes all the weight.)"""
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, BF, dtype, 1.0, 2)
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(0, 0))
    g = torch.Generator().manual_seed(3)
    for kv, (a, b) in enumerate(((max(low, 123), min(high, 128)), (low, high))):
        c.c.scale[1, :, kv] = torch.randint(a, b + 1, c.c.scale[1, :, kv].shape, generator=g, dtype=torch.uint8).cuda()
    check(c, 1, q, lens, mask, nodes, hd ** -0.5, attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0])
    out = [torch.empty((1, 2, 200, kvh, hd), device="cuda") for _ in range(2)]
    cdsl.cdsl_kv_read(c.c, 1, ints(30, 60), *out)
    for b, first in enumerate((30, 60)):
        assert all(torch.equal(x[0, b].double(), y) for x, y in zip(out, c.values(1, b, first, 200)))


@CACHES
@pytest.mark.parametrize("T", [8, 40], ids=["slots", "rows"])
@TYPES
def test_values_that_the_cache_rounds_to_infinity(cdsl, cache, T, dtype):
    """fp32 values above bf16's largest by half a step and more: a bf16 row with one holds a value that is not finite, and what
    a node does not see of it does not reach the node. The largest that rounds down stays, and e4m3 holds all of them."""
    B, kvh, hd, lens = 1, 2, 64, [130]
    c, q, k, v, _, mask, nodes = problem(cdsl, T, 2, kvh, hd, cache, dtype, 1.0, 4, lens)
    big = torch.tensor([0x7F7F7FFF, 0x7F7F8000, 0x7F7FFFFF], dtype=torch.int32).view(F32)   # to bf16: its largest, inf, inf
    n = lens[0]
    v[0, n + 2, 0, 3], v[0, n + 3, 0, 4], v[0, n + 4, 0, 5] = big[0], -big[1], big[2]
    cdsl.cdsl_kv_write(c.c, 1, k.cuda(), v.cuda(), ints(0))
    rows = c.values(1, 0, n + 2, 3)[1]
    bad = torch.isnan(rows).all(-1)
    assert bad.tolist() == [[False, False]] + [[cache is BF, False]] * 2
    assert torch.isfinite(rows[~bad]).all()
    got = attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0]
    want = torch.ones(T, dtype=torch.bool, device="cuda")
    want[[2, 3, 4]] = False
    assert torch.isfinite(got[0, want]).all()
    if cache is BF:
        assert torch.isnan(got[0, 3:5, 0]).all() and torch.isfinite(got[0, 3:5, 1]).all()


MIXED = [  # B, T, H, kvh, hd, page: 1, 8, 24, 32, 40 and 128 vectors a K/V head, and 2 blocks of rows
    (6, 1, 4, 4, 128, 16), (5, 2, 8, 2, 64, 64), (6, 6, 8, 2, 128, 256), (5, 32, 3, 3, 64, 16), (5, 10, 8, 2, 128, 32),
    (4, 128, 1, 1, 64, 128), (4, 33, 8, 2, 128, 64)]


@pytest.mark.parametrize("shape", MIXED, ids=[str(i) for i in range(len(MIXED))])
@CACHES
@TYPES
@pytest.mark.parametrize("tail", [1.0, 4.0, 12.0])
def test_heavy_tails_with_all_that_is_rare(cdsl, shape, cache, dtype, tail):
    """Values whose sizes are spread by e^tail from row to row, so that chunks with scales far apart and others take turns
    in an item, together with ragged trees, rows that see nothing, a node whose V and one whose K is not finite, and a page
    that is out of range. Bits are the same in a second call."""
    import random
    B, T, H, kvh, hd, page = shape
    rng, g = random.Random(T), torch.Generator().manual_seed(T)
    lens = [rng.choice([0, 1, 127, 128, 129, 300, 700, 1000]) for _ in range(B - 1)] + [1000]
    nodes = [rng.randint((T + 1) // 2, T) for _ in range(B)]
    n = max(lens) + T
    c = ref.Cache(B, n, kvh, hd, page, cache, layers=2, seed=T)
    k, v = (torch.randn((B, n, kvh, hd), generator=g) for _ in range(2))
    v = v * torch.where(torch.rand((B, n, kvh, 1), generator=g) < 0.02, (torch.randn((B, n, kvh, 1), generator=g) * tail).exp(), 1.0)
    v[B - 1, :256] *= 2.0 ** -20               # (whole chunks of small values, then of large ones)
    bad_v, bad_k = lens[0] + nodes[0] - 1, lens[1] + nodes[1] - 1
    v[0, bad_v, 0, 3], k[1, bad_k, 0, 5] = float("inf"), float("nan")
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(*[0] * B), ints(*[a + b for a, b in zip(lens, nodes)]))
    mask = torch.stack([cdsl.cdsl_tree_mask(ref.tree("random", T, rng))[0] for _ in range(B)])
    if T > 2:
        mask[2, 1] = 0
    q = torch.randn((B, T, H, hd), generator=g).to(dtype).cuda()
    scale = hd ** -0.5
    got = attend(cdsl, c, 1, q, lens, mask, nodes, scale)[0]
    assert torch.equal(torch.nan_to_num(got, 7.0), torch.nan_to_num(attend(cdsl, c, 1, q, lens, mask, nodes, scale)[0], 7.0))
    G = H // kvh
    for b in range(B):
        sees = [ref.bits_of(mask, b, t, nodes[b]) for t in range(nodes[b])]
        blind = torch.tensor([lens[b] + sum(s) == 0 for s in sees], device="cuda")
        at = {0: bad_v, 1: bad_k}.get(b, -1) - lens[b]
        nan = torch.tensor([at >= 0 and s[at] == 1 for s in sees], device="cuda")
        assert (got[b, nodes[b]:] == 0).all() and (got[b, :nodes[b]][blind] == 0).all()
        assert torch.isnan(got[b, :nodes[b]][nan][:, :G]).all()
        rest = ~blind & ~nan
        if b < 2 and G < H:                    # (other heads' rows are finite)
            assert torch.isfinite(got[b, :nodes[b]][:, G:]).all()
        if rest.any():
            t = torch.nonzero(rest)[:, 0].cpu()
            part = c.values(1, b, 0, lens[b] + nodes[b])
            check_rows(c, b, part, q[b, t], [sees[i] for i in t.tolist()], lens[b], scale, got[b, t])
    lost = c.table.clone()
    lost[B - 1, 0] = 1 << 22
    out, ws = torch.empty_like(q), torch.empty(cdsl.cdsl_tree_attention_workspace(c.c, T, H), dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    cdsl.cdsl_tree_attention(c.c.at(lost), 1, q, ints(*lens), mask.cuda(), out, ws, scale=scale, max_len=max(lens),
                             nodes=ints(*nodes), status=st)
    assert int(st) == cdsl.CDSL_ERANGE
    b, t = B - 1, nodes[B - 1]
    part = [x[page:] for x in c.values(1, b, 0, lens[b] + t)]
    check_rows(c, b, part, q[b, :t], [ref.bits_of(mask, b, i, t) for i in range(t)], lens[b] - page, scale, out[b, :t])


def check_rows(c, b, kv, q, sees, n, scale, got):
    """Rows of one sequence that see its first n slots and some of the rest; as in check()."""
    G = q.shape[1] // kv[0].shape[1]
    finite = torch.isfinite(kv[0]).all(-1) & torch.isfinite(kv[1]).all(-1)
    k, v = (torch.where(finite[..., None], x, 0.0).repeat_interleave(G, 1) for x in kv)
    see = torch.tensor([[1] * n + s for s in sees], dtype=torch.bool, device="cuda")
    qd = q.double()
    x = torch.einsum("thd,nhd->thn", qd, k) * scale
    p = torch.softmax(x.masked_fill(~see[:, None], float("-inf")), -1)
    out, size = (torch.einsum("thn,nhd->thd", p, y) for y in (v, v.abs()))
    s_abs = (torch.einsum("thd,nhd->thn", qd.abs(), k.abs()) * scale).amax(-1, keepdim=True)
    keys = k.shape[0]
    dw = 2 * (q.shape[2] + 4) * 2.0 ** -24 * s_abs + (keys + 16) * 2.0 ** -24
    e = dw * size
    if q.dtype is BF:
        e = (dw + 2 * 2.0 ** -13 * s_abs + 2.0 ** -8) * size + 2.0 ** -8 * out.abs()
        if c.c.pool.dtype is F8:               # per chunk of 128 slots: scales within 2^8 of its smallest
            vmax = v.abs().amax(-1)            # [keys, heads]; a scale is at most vmax / 224
            for first in range(0, keys, 128):
                part = vmax[first:first + 128]
                small = torch.where(part > 0, part, float("inf")).amin(0)
                top = torch.minimum(part.amax(0), small * 2 ** 9) / 224
                step = p[..., first:first + 128].amax(-1) * 448 * top
                e = e + (6 / 12 ** 0.5 * part.shape[0] ** 0.5 * 2.0 ** -21 * step)[..., None]
    d = (got.double() - out).abs()
    assert torch.isfinite(got).all()
    assert (d <= e).all(), float((d / e).max())
