"""The attention over a 4-bit cache with keys and values whose scale is not finite: they stand for NaN."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from test_gpu_i4_ranges import HEADS, SHAPES, TYPES, check, problem  # noqa: E402
from test_gpu_tree import attend, cdsl, ints  # noqa: E402,F401
from tree_reference import BF  # noqa: E402


def at(c, b, slot):
    """Where a sequence's slot is in the pool: page, place."""
    return int(c.table[b, slot // c.page]), slot % c.page


@SHAPES
@TYPES
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("slot", [0, 70, 259])
def test_a_key_whose_scale_is_not_finite(cdsl, T, H, kvh, hd, dtype, value, slot):
    """A caller's own cached key with one such scale: all queries of its head that see it give NaN, whatever their sign."""
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, dtype, 1.0, 11)
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(0, 0))
    for b, group in ((0, 0), (1, hd // 32 - 1)):
        p, i = at(c, b, slot)
        c.c.scale[1, p, 0, 0, i, group] = value
    got = attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0]
    G = H // kvh
    assert torch.isnan(got[:, :, :G]).all()
    assert torch.isfinite(got[:, :, G:]).all()


@pytest.mark.parametrize("T,H,kvh,hd", HEADS[2:], ids=[str(i) for i in range(len(HEADS) - 2)])
@TYPES
@pytest.mark.parametrize("value", [float("inf"), float("-inf")])
def test_a_node_whose_keys_scale_is_not_finite(cdsl, T, H, kvh, hd, dtype, value):
    """Of a star's nodes only itself sees it; others' results are as they are without it."""
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, dtype, 1.0, 12)
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(0, 0))
    for b, n in enumerate(lens):
        p, i = at(c, b, n + T - 1)
        c.c.scale[1, p, 0, :, i, 1] = value
    got = attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0]
    assert torch.isnan(got[:, T - 1]).all()
    got[:, T - 1] = 0
    for b in range(len(lens)):
        mask[b, :, :] = mask[b] & torch.tensor([-1 ^ (1 << (T - 1))], dtype=torch.int64).to(torch.int32)
    one = nodes[0] - 1
    check(c, 1, q[:, :one], lens, mask, [one] * len(lens), hd ** -0.5, got[:, :one])


@SHAPES
@TYPES
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("slot", [0, 70, 259])
def test_a_value_whose_scale_is_not_finite(cdsl, T, H, kvh, hd, dtype, value, slot):
    """V's, alike: NaN in all of the head's dimensions."""
    c, q, k, v, lens, mask, nodes = problem(cdsl, T, H, kvh, hd, dtype, 1.0, 11)
    cdsl.cdsl_kv_write(c.c, 1, k.to(BF).cuda(), v.to(BF).cuda(), ints(0, 0))
    for b, group in ((0, 0), (1, hd // 32 - 1)):
        p, i = at(c, b, slot)
        c.c.scale[1, p, 1, 0, i, group] = value
    got = attend(cdsl, c, 1, q, lens, mask, nodes, hd ** -0.5)[0]
    G = H // kvh
    assert torch.isnan(got[:, :, :G]).all()
    assert torch.isfinite(got[:, :, G:]).all()
