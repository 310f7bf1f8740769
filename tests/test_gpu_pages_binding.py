"""What the binding of the 4-bit cache, the page calls and the rotary positions refuses of tensors that are on a GPU."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from test_gpu_tree import cdsl, ints  # noqa: E402,F401
from tree_reference import BF, F32  # noqa: E402

U8 = torch.uint8


@pytest.fixture
def calls(cdsl):
    """Every call that launches, with arguments that it takes (changed by keywords), and what it writes."""
    B, T, kvh, hd, n = 2, 3, 2, 64, 8
    table = torch.tensor([[0, 1], [2, -1]], dtype=torch.int32, device="cuda")
    c = cdsl.KvCache.empty(1, n, kvh, 16, hd, table, U8)
    c.pool.fill_(7)
    refs = ints(1, 1, 1, 0, 0, 0, 0, 0)
    new_table, new_refs, page_map = torch.full_like(table, 7), torch.full_like(refs, 7), torch.full_like(refs, 7)
    new_lens, live = ints(7, 7), ints(7)
    ws = torch.empty(cdsl.cdsl_kv_pages_workspace(c), dtype=U8, device="cuda")
    q, k = torch.ones((B, T, 4, hd), dtype=BF, device="cuda"), torch.ones((B, T, kvh, hd), dtype=BF, device="cuda")
    qo, ko = torch.full_like(q, 7), torch.full_like(k, 7)
    rope = cdsl.Rope(hd)

    def fork(refs=refs, src=ints(0, 1), lens=ints(20, 3), new_table=new_table, new_lens=new_lens, new_refs=new_refs, ws=ws, **kw):
        cdsl.cdsl_kv_fork(c, refs, src, lens, new_table, new_lens, new_refs, ws, **kw)

    def resize(refs=refs, slots=ints(16, 17), new_table=new_table, new_refs=new_refs, ws=ws, **kw):
        cdsl.cdsl_kv_resize(c, refs, slots, new_table, new_refs, ws, **kw)

    def compact(refs=refs, new_table=new_table, new_refs=new_refs, page_map=page_map, live=live, ws=ws, **kw):
        cdsl.cdsl_kv_compact(c, refs, new_table, new_refs, page_map, live, ws, **kw)

    def turn(q=q, qo=qo, start=ints(1, 2), k=k, ko=ko, **kw):
        cdsl.cdsl_rope(rope, q, qo, start, k=k, k_out=ko, **kw)

    outputs = (new_table, new_refs, page_map, new_lens, live, qo, ko)
    return dict(fork=fork, resize=resize, compact=compact, rope=turn, outputs=outputs, q=q, k=k, table=table)


@pytest.mark.parametrize("name", ["fork", "resize", "compact", "rope"])
def test_tensors_of_a_device_that_is_not_current_are_refused(cdsl, calls, monkeypatch, name):
    """With the stream given or not; nothing is launched. (How many devices there are and which is current are made up.)"""
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


def test_wrong_tensors_are_refused(cdsl, calls):
    q, k, table = calls["q"], calls["k"], calls["table"]
    bad = [("fork", dict(refs=ints(1, 1))), ("fork", dict(src=ints(0, 1)[None])), ("fork", dict(lens=ints(1, 2, 3))),
           ("fork", dict(new_table=table[:1])), ("fork", dict(new_table=table)), ("fork", dict(new_lens=ints(1))),
           ("fork", dict(new_refs=torch.zeros(8, device="cuda"))), ("fork", dict(ws=torch.empty(64, dtype=U8, device="cuda"))),
           ("fork", dict(ws=torch.empty(1 << 20, dtype=torch.int8, device="cuda"))), ("resize", dict(slots=ints(1))),
           ("resize", dict(new_table=table.T)), ("resize", dict(refs=ints(*[0] * 8).cpu())), ("compact", dict(live=ints(1, 2))),
           ("compact", dict(page_map=ints(1))), ("compact", dict(status=ints(1, 2))), ("rope", dict(q=q.half())),
           ("rope", dict(q=q[0])), ("rope", dict(qo=k)), ("rope", dict(qo=q.float())), ("rope", dict(ko=None)), ("rope", dict(k=None)),
           ("rope", dict(k=k[:, :2], ko=k[:, :2])), ("rope", dict(k=k[..., :32], ko=k[..., :32])), ("rope", dict(start=ints(1))),
           ("rope", dict(offset=ints(1, 2))), ("rope", dict(qo=q[:, :, :1].expand(-1, -1, 4, -1))),
           ("rope", dict(q=q.transpose(2, 3).contiguous().transpose(2, 3))), ("rope", dict(q=q.cpu(), qo=q.cpu()))]
    for name, kw in bad:
        with pytest.raises(cdsl.CdslError):
            calls[name](**kw)
        assert all((x == 7).all() for x in calls["outputs"]), (name, list(kw))


def test_wrong_caches_are_refused(cdsl, calls):
    pool = torch.zeros((1, 8, 2, 2, 16, 32), dtype=U8, device="cuda")
    scale = torch.zeros((1, 8, 2, 2, 16, 2), dtype=BF, device="cuda")
    table = calls["table"]
    assert cdsl.KvCache(pool, scale, table).head_dim == 64
    for p, s in ((pool, scale.float()), (pool, scale[..., :1].contiguous()), (pool, scale.view(U8)), (pool[..., ::2], scale),
                 (pool.view(torch.int8), scale), (pool, torch.zeros(pool.shape[:5], dtype=U8, device="cuda"))):
        with pytest.raises(cdsl.CdslError):
            cdsl.KvCache(p, s, table)
    with pytest.raises(cdsl.CdslError):        # heads of 192: refused by the first call
        c = cdsl.KvCache.empty(1, 8, 2, 16, 192, table, U8)
        x = torch.zeros((2, 1, 2, 192), dtype=F32, device="cuda")
        cdsl.cdsl_kv_write(c, 0, x, x, ints(0, 0))
