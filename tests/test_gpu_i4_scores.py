"""The attention over a 4-bit cache at the ends of what keys, queries and scales can be: scores of ordinary size, or finite ones at
least, from any of them."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import i4_reference as i4  # noqa: E402
import tree_reference as ref  # noqa: E402
from test_gpu_i4_ranges import HEADS, SHAPES, TYPES, check, problem  # noqa: E402
from test_gpu_tree import attend, cdsl, ints  # noqa: E402,F401
from tree_reference import BF, F32  # noqa: E402


# queries' size, keys' size, scale: scores of ordinary size
ORDINARY = [(2.0 ** -99, 2.0 ** 116, 2.0 ** -20), (2.0 ** -60, 2.0 ** 116, 2.0 ** -59), (2.0 ** 118, 2.0 ** 1, 2.0 ** -122),
            (2.0 ** 20, 2.0 ** -116, 2.0 ** 93), (2.0 ** -97, 2.0 ** -1, 2.0 ** 95)]


@SHAPES
@TYPES
@pytest.mark.parametrize("q_size,k_size,scale", ORDINARY, ids=[str(i) for i in range(len(ORDINARY))])
def test_scores_of_ordinary_size_from_any_scale(cdsl, T, H, kvh, hd, dtype, q_size, k_size, scale):
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, dtype, 1.0, 13)
    q = (q.double() / 8 * q_size).to(dtype)
    cdsl.cdsl_kv_write(c.c, 1, (k * k_size).cuda(), v.cuda(), ints(0, 0))
    check(c, 1, q, lens, mask, nodes, scale, attend(cdsl, c, 1, q, lens, mask, nodes, scale)[0])


@pytest.mark.parametrize("T,H,kvh,hd,dtype", [h + (t,) for h in HEADS for t in (F32, BF) if t is F32 or h[0] * h[1] // h[2] <= 16])
@pytest.mark.parametrize("q_size,scale", [(2.0 ** -100, 2.0 ** 10), (2.0 ** -20, 1.0), (1.0, 2.0 ** -7)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_the_largest_of_huge_scores(cdsl, T, H, kvh, hd, dtype, q_size, scale, sign):
    """Up to 16 bfloat16 vectors a K/V head, or float32 ones. Scores of 2^35 and more, of which one is twice the others, take all the weight: the result is that slot's value."""
    n, top = 300, 137
    c = i4.Cache(1, n + T, kvh, hd, 64, layers=2, seed=3)
    g = torch.Generator().manual_seed(4)
    k, v = torch.full((1, n + T, kvh, hd), 2.0 ** 118 * sign), torch.randn((1, n + T, kvh, hd), generator=g)
    k[:, top] = 2.0 ** 119 if sign > 0 else -2.0 ** 117
    cdsl.cdsl_kv_write(c.c, 1, k.cuda(), v.cuda(), ints(0))
    q = torch.full((1, T, H, hd), q_size, dtype=dtype, device="cuda")
    mask = cdsl.cdsl_tree_mask(ref.tree("star", T, None))[0][None]
    got, lse = attend(cdsl, c, 1, q, [n], mask, [T], scale)[:2]
    want = c.values(1, 0, top, 1)[1][0].repeat_interleave(H // kvh, 0)
    assert torch.equal(got[0].double(), want.expand(T, H, hd))
    dot = c.values(1, 0, top, 1)[0][0, 0, 0].item() * q_size * hd * scale
    assert (lse.double() - dot).abs().max() <= (hd + 8) * 2.0 ** -23 * abs(dot)
