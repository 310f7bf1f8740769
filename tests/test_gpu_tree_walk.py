"""Tree validation (include/cdsl_tree.h) at nodes whose rows are not finite and at nodes without children, by the kernel
that keeps a row in registers and by the one for rows beyond them."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from test_gpu_tree import cdsl, run_verify  # noqa: E402,F401
from tree_reference import BF, F32  # noqa: E402

VOCABS = [300, 5000, 163841]                   # one block, a cluster, beyond the registers


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("dtype", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("bad", ["nan", "+inf", "-inf"])
def test_greedy_walk_ends_without_a_token_at_a_bad_row(cdsl, V, dtype, bad):
    """A chain 0-1-2 of the target's best tokens, the row of node 0, 1 or 2 not finite: the nodes before are taken, and
    no token is drawn. -inf: the whole row."""
    T = 3
    logits = torch.zeros((T + 1, T, V), dtype=dtype)
    best = [V - 1, 11, 7]
    for i, x in enumerate(best):
        logits[:, i, x] = 4
    for b in range(T):
        if bad == "-inf":
            logits[b, b] = float("-inf")
        else:
            logits[b, b, 5] = float(bad)
    tokens = torch.tensor([[0, best[0], best[1]]] * (T + 1), dtype=torch.int32)
    u, u_last = torch.zeros((T + 1, T)), torch.zeros(T + 1)
    for temperature in (0.0, 0.25):
        path, n, emitted, st = run_verify(cdsl, logits, None, tokens, [[0, 0, 1]] * (T + 1), u, u_last, temperature)
        assert st == cdsl.CDSL_ENONFINITE
        assert n == [1, 2, 3, 3]
        assert path.tolist() == [[0, -1, -1], [0, 1, -1], [0, 1, 2], [0, 1, 2]]
        assert emitted[:3].tolist() == [[-1, -1, -1], [best[0], -1, -1], [best[0], best[1], -1]]
        assert emitted[3, :2].tolist() == best[:2] and (temperature > 0 or int(emitted[3, 2]) == best[2])


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("dtype", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("left", ["nan", "+inf", "-inf"])
def test_draft_rows_of_leaves_do_not_matter(cdsl, V, dtype, left):
    """The draft's row of a node without children was never sampled from: whatever is in it, the target's row alone
    decides the draw there. Sequences: a chain taken to its leaf; a chain of which `nodes` leaves out the last, so that
    node 1 is the leaf; the root alone; a node whose only child names a later parent."""
    B, T = 4, 3
    g = torch.Generator().manual_seed(V)
    logits = torch.randn((B, T, V), generator=g).to(dtype)
    draft = torch.randn((B, T, V), generator=g).to(dtype)
    tokens = torch.randint(0, V, (B, T), generator=g, dtype=torch.int32)
    parents = [[0, 0, 1]] * 3 + [[0, 0, 2]]
    nodes = [3, 2, 1, 3]
    u, u_last = torch.zeros((B, T)), torch.rand(B, generator=g)     # (u = 0 takes every child that has a weight)
    want = run_verify(cdsl, logits, draft, tokens, parents, u, u_last, 1.0, nodes)
    assert want[3] == cdsl.CDSL_OK and want[1] == [3, 2, 1, 2]
    for b, i in ((0, 2), (1, 1), (2, 0), (3, 1)):
        if left == "-inf":
            draft[b, i] = float("-inf")
        else:
            draft[b, i, 3] = float(left)
    got = run_verify(cdsl, logits, draft, tokens, parents, u, u_last, 1.0, nodes)
    assert got[3] == cdsl.CDSL_OK and got[1] == want[1]
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
