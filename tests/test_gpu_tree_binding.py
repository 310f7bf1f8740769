"""What the binding of the tree speculation calls (include/cdsl_tree.h) refuses of tensors that are on a GPU."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import tree_reference as ref  # noqa: E402
from test_gpu_tree import cdsl, ints  # noqa: E402,F401
from tree_reference import BF, F8  # noqa: E402


@pytest.fixture
def calls(cdsl):
    """Every call that launches, with arguments that it takes."""
    B, T, H, kvh, hd, V = 2, 5, 4, 2, 64, 100
    c = ref.Cache(B, 20, kvh, hd, 16, F8).c
    rows = torch.zeros((B, T, kvh, hd), dtype=BF, device="cuda")
    back = torch.full((1, B, T, kvh, hd), 7.0, dtype=BF, device="cuda")
    q = torch.zeros((B, T, H, hd), dtype=BF, device="cuda")
    out = torch.full_like(q, 7.0)
    lens, path, n_path = ints(3, 4), torch.zeros((B, T), dtype=torch.int32, device="cuda"), ints(1, 1)
    mask = cdsl.cdsl_tree_mask([0] * T)[0].cuda().expand(B, -1, -1).contiguous()
    ws = torch.empty(cdsl.cdsl_tree_attention_workspace(c, T, H), dtype=torch.uint8, device="cuda")
    logits, u = torch.zeros((B, T, V), device="cuda"), torch.zeros((B, T), device="cuda")
    emitted = torch.full((B, T), 7, dtype=torch.int32, device="cuda")
    return dict(
        outputs=(back, out, emitted),
        write=lambda **kw: cdsl.cdsl_kv_write(c, 0, rows, rows, lens, **kw),
        read=lambda **kw: cdsl.cdsl_kv_read(c, 0, lens, back, back.clone(), **kw),
        commit=lambda **kw: cdsl.cdsl_kv_commit(c, lens, path, n_path, **kw),
        attend=lambda out=out, **kw: cdsl.cdsl_tree_attention(c, 0, q, lens, mask, out, ws, scale=0.1, max_len=4, **kw),
        verify=lambda **kw: cdsl.cdsl_tree_verify(logits, path, path, u, u[:, 0].contiguous(), path.clone(), n_path.clone(),
                                                  emitted, **kw))


@pytest.mark.parametrize("name", ["write", "read", "commit", "attend", "verify"])
def test_tensors_of_a_device_that_is_not_current_are_refused(cdsl, calls, monkeypatch, name):
    """With the stream given or not; nothing is launched. (One GPU is enough: how many
    there are and which is current are made up.)"""
    calls[name]()                              # (taken as it is)
    for x in calls["outputs"]:
        x.fill_(7)
    stream = torch.cuda.current_stream().cuda_stream
    monkeypatch.setattr(cdsl._torch(), "devices", 2, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for kw in ({}, {"stream": stream}):
        with pytest.raises(cdsl.CdslError, match="current device"):
            calls[name](**kw)
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert all((x == 7).all() for x in calls["outputs"])
