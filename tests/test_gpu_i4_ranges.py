"""The attention over a 4-bit cache where V's sizes differ by orders of magnitude between slots and between groups: what a query
gives no weight, or does not see, takes nothing from what it does see."""
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import i4_reference as i4  # noqa: E402
import tree_reference as ref  # noqa: E402
from test_gpu_tree import attend, cdsl, ints  # noqa: E402,F401
from tree_reference import BF, F32  # noqa: E402


def check_rows(hd, kv, q, sees, n, scale, got):
    """Rows of one sequence, q [t, H, hd], that see its first n slots and some of the rest, per element. The weights' relative
    error, each on its own |v|: scores of hd + 8 additions of 2^-23, as many again in exp, sum and product, and for bf16
    queries 2^-11 (2^-12 of a weight in fp16, its sum, and 2^-16 for each slot with a weight below 2^-32 among scales 2^16 apart, of
    which those tests have few). One rounding of the result."""
    G = q.shape[1] // kv[0].shape[1]
    finite = torch.isfinite(kv[0]).all(-1) & torch.isfinite(kv[1]).all(-1)
    k, v = (torch.where(finite[..., None], x, 0.0).repeat_interleave(G, 1) for x in kv)
    see = torch.tensor([[1] * n + s for s in sees], dtype=torch.bool, device="cuda")
    qd = q.double()
    x = torch.einsum("thd,nhd->thn", qd, k) * scale
    p = torch.softmax(x.masked_fill(~see[:, None], float("-inf")), -1)
    out, size = (torch.einsum("thn,nhd->thd", p, y) for y in (v, v.abs()))
    s_abs = (torch.einsum("thd,nhd->thn", qd.abs(), k.abs()) * scale).masked_fill(~see[:, None], 0.0).amax(-1, keepdim=True)
    e = (2 * (hd + 8) * 2.0 ** -23 * s_abs + (k.shape[0] + 16) * 2.0 ** -23 + (2.0 ** -11 if q.dtype is BF else 0)) * size
    e = e + (2.0 ** -8 if q.dtype is BF else 2.0 ** -24) * out.abs()
    d = (got.double() - out).abs()
    assert torch.isfinite(got).all()
    assert (d <= e).all(), float((d / e).nan_to_num(0).max())


def check(c, layer, q, lens, mask, nodes, scale, got):
    for b in range(len(lens)):
        check_rows(q.shape[3], c.values(layer, b, 0, lens[b] + nodes[b]), q[b, :nodes[b]],
                   [ref.bits_of(mask, b, t, nodes[b]) for t in range(nodes[b])], lens[b], scale, got[b, :nodes[b]])


def problem(cdsl, T, H, kvh, hd, dtype, size, seed, lens=(700, 260)):
    """Queries that share a large first component, keys without it, and values of about `size`; a star of T nodes."""
    g = torch.Generator().manual_seed(seed)
    lens, B, n = list(lens), len(lens), max(lens) + T
    c = i4.Cache(B, n, kvh, hd, 64, layers=2, seed=seed)
    k, v = (torch.randn((B, n, kvh, hd), generator=g) for _ in range(2))
    k[..., 0] = 0
    q = torch.randn((B, T, H, hd), generator=g)
    q[..., 0] = 8
    mask = torch.stack([cdsl.cdsl_tree_mask(ref.tree("star", T, None))[0]] * B)
    return c, q.to(dtype).cuda(), k, v * size, lens, mask, [T] * B


# 1, 4, 8 and 16 vectors a K/V head (slots as the MMA's rows), 24, 36 and 34 (vectors as rows)
HEADS = [(1, 2, 2, 128), (1, 8, 2, 64), (2, 8, 2, 128), (4, 8, 2, 64), (6, 8, 2, 128), (9, 8, 2, 128), (17, 4, 2, 64)]
SHAPES = pytest.mark.parametrize("T,H,kvh,hd", HEADS, ids=[str(i) for i in range(len(HEADS))])
TYPES = pytest.mark.parametrize("dtype", [F32, BF], ids=["q32", "q16"])


@SHAPES
@TYPES
@pytest.mark.parametrize("up", [5, 9, 14, 20, 60])
@pytest.mark.parametrize("at", [5, 259])
@pytest.mark.parametrize("group", [False, True])
def test_a_large_value_without_weight(cdsl, T, H, kvh, hd, dtype, up, at, group):
    """One cached token's V, or one group of it, is 2^up times the others', its weight below 2^-60."""
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, dtype, 1.0, up)
    v[:, at, :, 32 if group else 0:64 if group else hd] *= 2.0 ** up
    k[:, at] = 0
    k[:, at, :, 0] = -7 * hd ** 0.5
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(0, 0))
    check(c, 1, q, lens, mask, nodes, hd ** -0.5, attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0])


@pytest.mark.parametrize("T,H,kvh,hd", HEADS[3:], ids=[str(i) for i in range(len(HEADS) - 3)])
@TYPES
@pytest.mark.parametrize("up", [9, 20, 40])
def test_a_large_value_that_is_not_seen(cdsl, T, H, kvh, hd, dtype, up):
    """A node's V is 2^up times the others'; its siblings' results do not depend on it."""
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, dtype, 1.0, up)
    for b, n in enumerate(lens):
        v[b, n + 2] *= 2.0 ** up
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(0, 0))
    check(c, 1, q, lens, mask, nodes, hd ** -0.5, attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0])


@SHAPES
@TYPES
@pytest.mark.parametrize("size", [100.0, 0.01, 1e-6])
def test_values_and_groups_of_zeros(cdsl, T, H, kvh, hd, dtype, size):
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, dtype, size, 1)
    v[:, 130] = 0
    v[:, 131, :, :32] = 0
    k[:, 132] = 0
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(0, 0))
    check(c, 1, q, lens, mask, nodes, hd ** -0.5, attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0])


@SHAPES
@TYPES
@pytest.mark.parametrize("down", [6, 24])
def test_a_small_value_with_most_of_the_weight(cdsl, T, H, kvh, hd, dtype, down):
    """The first token takes most of the weight and its V is 2^-down of the others'."""
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, dtype, 1.0, down)
    v[:, 0] *= 2.0 ** -down
    k[:, 0] = 0
    k[:, 0, :, 0] = hd ** 0.5
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(0, 0))
    check(c, 1, q, lens, mask, nodes, hd ** -0.5, attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0])


@SHAPES
@TYPES
@pytest.mark.parametrize("q_size,k_size", [(2.0 ** 60, 2.0 ** -60), (2.0 ** -90, 2.0 ** 90), (2.0 ** 118, 2.0 ** -117), (1e-38, 1e34)])
def test_sizes_of_queries_and_keys(cdsl, T, H, kvh, hd, dtype, q_size, k_size):
    """Scores of ordinary size from queries and keys that are not."""
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, dtype, 1.0, 3)
    q = (q.double() / 8 * q_size).to(dtype)
    cdsl.cdsl_kv_write(c.c, 1, (k * k_size).cuda(), v.cuda(), ints(0, 0))
    check(c, 1, q, lens, mask, nodes, hd ** -0.5, attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0])


MIXED = [  # B, T, H, kvh, hd, page: 1, 4, 8, 15, 24, 40 and 128 vectors a K/V head, and 2 blocks of rows
    (6, 1, 4, 4, 128, 16), (6, 2, 8, 4, 64, 32), (5, 2, 8, 2, 64, 64), (6, 3, 10, 2, 128, 16), (6, 6, 8, 2, 128, 256),
    (5, 10, 8, 2, 128, 32), (4, 128, 1, 1, 64, 128), (4, 33, 8, 2, 128, 64)]


@pytest.mark.parametrize("shape", MIXED, ids=[str(i) for i in range(len(MIXED))])
@TYPES
@pytest.mark.parametrize("tail", [1.0, 4.0, 12.0])
def test_heavy_tails_with_all_that_is_rare(cdsl, shape, dtype, tail):
    """Values whose sizes are spread by e^tail from row to row, so that chunks with scales far apart and others take turns
    in an item, together with ragged trees, rows that see nothing, a node whose V and one whose K is not finite, and a page
    that is out of range. Bits are the same in a second call."""
    B, T, H, kvh, hd, page = shape
    rng, g = random.Random(T), torch.Generator().manual_seed(T)
    lens = [rng.choice([0, 1, 127, 128, 129, 300, 700, 1000]) for _ in range(B - 1)] + [1000]
    nodes = [rng.randint((T + 1) // 2, T) for _ in range(B)]
    n = max(lens) + T
    c = i4.Cache(B, n, kvh, hd, page, layers=2, seed=T)
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
            check_rows(hd, c.values(1, b, 0, lens[b] + nodes[b]), q[b, t], [sees[i] for i in t.tolist()], lens[b], scale, got[b, t])
    lost = c.table.clone()
    lost[B - 1, 0] = 1 << 22
    out, ws = torch.empty_like(q), torch.empty(cdsl.cdsl_tree_attention_workspace(c.c, T, H), dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    cdsl.cdsl_tree_attention(c.c.at(lost), 1, q, ints(*lens), mask.cuda(), out, ws, scale=scale, max_len=max(lens),
                             nodes=ints(*nodes), status=st)
    assert int(st) == cdsl.CDSL_ERANGE
    b, t = B - 1, nodes[B - 1]
    part = [x[page:] for x in c.values(1, b, 0, lens[b] + t)]
    check_rows(hd, part, q[b, :t], [ref.bits_of(mask, b, i, t) for i in range(t)], lens[b] - page, scale, out[b, :t])
