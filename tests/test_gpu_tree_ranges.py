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
