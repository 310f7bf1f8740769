"""Attention by rows where a token with most of a row's weight has a far smaller V than thousands that have next to none: what those
have together counts, in whatever chunk the one token lies."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import i4_reference as i4  # noqa: E402
import tree_reference as ref  # noqa: E402
from test_gpu_tree import attend, cdsl, ints  # noqa: E402,F401
from tree_reference import BF, F8  # noqa: E402

I4 = torch.uint8


def check_rows(c, b, q, sees, n, scale, got):
    """Per element, each weight's error on its own |v|: 2^-11 relative (2^-12 of a weight in fp16, or 2^-16 in two planes, and its
    sum). Scores: hd + 8 additions of 2^-23, and over e4m3 queries that are each off by 2^-18 of the row's largest value. Where
    no scale of V is below 2^-16 of the largest (e4m3: 2^-21), a weight may be held to 2^-32 of the row's largest instead: half of fp16's
    smallest step of 2^-24, at a reference that counts as 2^7. One rounding of the result."""
    kv = c.values(1, b, 0, n + len(sees))
    G, hd = q.shape[1] // kv[0].shape[1], q.shape[2]
    k, v = (x.repeat_interleave(G, 1) for x in kv)
    see = torch.tensor([[1] * n + s for s in sees], dtype=torch.bool, device="cuda")
    qd = q.double()
    x = torch.einsum("thd,nhd->thn", qd, k) * scale
    p = torch.softmax(x.masked_fill(~see[:, None], float("-inf")), -1)
    out, size = (torch.einsum("thn,nhd->thd", p, y) for y in (v, v.abs()))
    s_abs = (torch.einsum("thd,nhd->thn", qd.abs(), k.abs()) * scale).amax(-1, keepdim=True)
    ds = (hd + 8) * 2.0 ** -23 * s_abs
    if c.c.pool.dtype is F8:
        ds = ds + 2.0 ** -18 * scale * qd.abs().amax(-1, keepdim=True) * k.abs().sum(-1).amax(0)[None, :, None]
    e = (2 * ds + (k.shape[0] + 16) * 2.0 ** -23 + 2.0 ** -11) * size + 2.0 ** -8 * out.abs()
    s = scales(c, b, n + len(sees))
    if s.amax() <= s.amin() * {I4: 2.0 ** 16, F8: 2.0 ** 21, BF: 0.0}[c.c.pool.dtype]:
        e = e + 2.0 ** -32 * p.amax(-1, keepdim=True) * v.abs().sum(0)
    d = (got.double() - out).abs()
    assert torch.isfinite(got).all()
    assert (d <= e).all(), float((d / e).max())


def scales(c, b, n):
    """V's scales of a sequence's first n slots."""
    slot = torch.arange(n, device="cuda")
    x = c.c.scale[1][c.table[b][slot // c.page].long(), 1, :, slot % c.page].double()
    return x if c.c.pool.dtype is I4 else torch.exp2(x - 127)


# 17 .. 36 vectors a K/V head (vectors as rows; an e4m3 cache: from 33 on); the whole row, or a group of it, is small
SHAPES = [(I4, 17, 2, 2, 128, False), (I4, 6, 8, 2, 128, True), (I4, 34, 2, 2, 64, False), (I4, 20, 2, 2, 64, True),
          (F8, 36, 2, 2, 128, False), (F8, 17, 4, 2, 64, False), (BF, 36, 2, 2, 128, False)]


@pytest.mark.parametrize("cache,T,H,kvh,hd,group", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
@pytest.mark.parametrize("down", [13, 18, 40])
@pytest.mark.parametrize("place", ["first", "middle", "last", "chunk"])
def test_a_heavy_token_with_a_small_value(cdsl, cache, T, H, kvh, hd, group, down, place):
    """Base 2, the others' scores are 33 below the heavy token's. Enough sequences for several chunks a block. "chunk": V of
    a whole chunk is as small, and no chunk has scales far apart."""
    B, n = 80, 1000 if place == "first" else 700
    g = torch.Generator().manual_seed(down)
    c = i4.Cache(B, n + T, kvh, hd, 64, layers=2, seed=down) if cache is I4 else ref.Cache(B, n + T, kvh, hd, 64, cache, layers=2, seed=down)
    k, v = torch.randn((B, n + T, kvh, hd), generator=g) * 0.05, torch.randn((B, n + T, kvh, hd), generator=g)
    heavy = {"middle": n // 2, "last": n - 1}.get(place, 0)
    k[..., 0] = 0
    k[:, heavy] = 0
    k[:, heavy, :, 0] = 33 * 0.6931 * hd ** 0.5 / 8
    v[:, heavy:heavy + (128 if place == "chunk" else 1), :, :32 if group else hd] *= 2.0 ** -down
    q = torch.randn((B, T, H, hd), generator=g)
    q[..., 0] = 8
    q = q.to(BF).cuda()
    mask = torch.stack([cdsl.cdsl_tree_mask(ref.tree("star", T, None))[0]] * B)
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(*[0] * B))
    got = attend(cdsl, c, 1, q, [n] * B, mask, [T] * B, hd ** -0.5)[0]
    sees = [ref.bits_of(mask, 0, t, T) for t in range(T)]
    for b in range(0, B, 3):
        check_rows(c, b, q[b], sees, n, hd ** -0.5, got[b])
