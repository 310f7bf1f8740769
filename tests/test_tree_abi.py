"""Argument checks of the tree speculation entry points (no GPU needed: what is refused launches nothing)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def cdsl():
    from paper_2412_10418_gb300 import build
    build.build()
    import paper_2412_10418_gb300 as pkg
    return pkg


PTR = 1 << 20   # never dereferenced


def cache(cdsl, **kw):
    c = cdsl._KvCacheC(PTR, PTR, PTR, 2, 10, 8, 64, 128, cdsl.DTYPE_F8E4M3, 3, 4)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [dict(d_pool=None), dict(d_pool=PTR + 8), dict(d_scale=None), dict(d_page_table=None), dict(n_layers=0),
              dict(n_pages=0), dict(n_kv_heads=0), dict(page_size=48), dict(page_size=8), dict(page_size=512),
              dict(head_dim=96), dict(dtype=0), dict(dtype=7), dict(batch=0), dict(batch=1025), dict(max_pages=0),
              dict(n_pages=1 << 23), dict(n_pages=1 << 21), dict(max_pages=1 << 28)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=[str(b) for b in BAD_CACHES])
def test_bad_caches_are_refused(cdsl, bad):
    lib, c, n = cdsl.lib(), cache(cdsl, **bad), ctypes.c_size_t(0)
    st = (ctypes.c_int64 * 6)(*[8192, 1024, 128] * 2)
    calls = {"cdsl_kv_write": lambda: lib.cdsl_kv_write(ctypes.addressof(c), 0, PTR, PTR, 1, 4, st, PTR, None, None, None),
             "cdsl_kv_read": lambda: lib.cdsl_kv_read(ctypes.addressof(c), 0, 1, PTR, PTR, 1, 4, PTR, None, None, None),
             "cdsl_kv_commit": lambda: lib.cdsl_kv_commit(ctypes.addressof(c), PTR, PTR, PTR, 4, None, None, None),
             "cdsl_tree_attention": lambda: lib.cdsl_tree_attention(
                 ctypes.addressof(c), 0, PTR, 1, 32, 4, st, PTR, None, PTR, 0.1, 100, PTR, None, PTR, 1 << 30, None, None)}
    if not set(bad) & {"d_pool", "d_scale", "d_page_table"}:
        calls["cdsl_tree_attention_workspace"] = lambda: lib.cdsl_tree_attention_workspace(
            ctypes.addressof(c), 32, 4, ctypes.addressof(n))
    for name, call in calls.items():
        assert call() == cdsl.CDSL_EINVAL, name
        assert name in cdsl.cdsl_last_error(None)


def test_bad_arguments_are_refused(cdsl):
    lib, c = cdsl.lib(), cache(cdsl)
    a, st = ctypes.addressof(c), (ctypes.c_int64 * 6)(*[8192, 1024, 128] * 2)

    def write(layer=0, k=PTR, v=PTR, dtype=1, T=4, strides=st, start=PTR):
        return lib.cdsl_kv_write(a, layer, k, v, dtype, T, strides, start, None, None, None)

    for kw in (dict(layer=-1), dict(layer=2), dict(k=None), dict(v=None), dict(k=PTR + 1), dict(dtype=2), dict(T=0),
               dict(T=257), dict(strides=None), dict(start=None)):
        assert write(**kw) == cdsl.CDSL_EINVAL, kw

    def read(layer=0, n=1, k=PTR, v=PTR, dtype=1, T=4, start=PTR):
        return lib.cdsl_kv_read(a, layer, n, k, v, dtype, T, start, None, None, None)

    for kw in (dict(n=0), dict(n=3), dict(layer=1, n=2), dict(k=None), dict(k=PTR + 8), dict(dtype=2), dict(T=0),
               dict(start=None)):
        assert read(**kw) == cdsl.CDSL_EINVAL, kw

    def commit(lens=PTR, path=PTR, n=PTR, T=4, new=None):
        return lib.cdsl_kv_commit(a, lens, path, n, T, new, None, None)

    for kw in (dict(lens=None), dict(path=None), dict(n=None), dict(T=0), dict(T=129), dict(new=PTR)):
        assert commit(**kw) == cdsl.CDSL_EINVAL, kw

    def attend(layer=0, q=PTR, dtype=1, H=32, T=4, strides=st, lens=PTR, mask=PTR, scale=0.1, max_len=100, out=PTR,
               ws=PTR, n=1 << 30):
        return lib.cdsl_tree_attention(a, layer, q, dtype, H, T, strides, lens, None, mask, scale, max_len, out, None,
                                       ws, n, None, None)

    for kw in (dict(layer=2), dict(q=None), dict(q=PTR + 1), dict(dtype=2), dict(H=0), dict(H=12), dict(H=8 * 65),
               dict(T=0), dict(T=129), dict(strides=None), dict(lens=None), dict(mask=None), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(max_len=-1),
               dict(max_len=253), dict(out=None), dict(ws=None), dict(ws=PTR + 128)):
        assert attend(**kw) == cdsl.CDSL_EINVAL, kw
    assert attend(n=16) == cdsl.CDSL_ENOMEM

    def verify(B=2, T=4, V=100, logits=PTR, draft=None, dtype=0, strides=(ctypes.c_int64 * 4)(400, 100, 0, 0),
               tokens=PTR, parents=PTR, u=PTR, u_last=PTR, t=1.0, path=PTR, n=PTR, emitted=PTR):
        return lib.cdsl_tree_verify(B, T, V, logits, draft, dtype, strides, tokens, parents, None, u, u_last, t, path, n,
                                    emitted, None, None)

    for kw in (dict(B=0), dict(B=1025), dict(T=0), dict(T=129), dict(V=0), dict(V=(1 << 20) + 1), dict(logits=None),
               dict(logits=PTR + 2), dict(draft=PTR + 2), dict(dtype=2), dict(strides=None), dict(tokens=None),
               dict(parents=None), dict(u=None), dict(u_last=None), dict(t=-1.0), dict(t=float("nan")),
               dict(t=float("inf")), dict(path=None), dict(n=None), dict(emitted=None)):
        assert verify(**kw) == cdsl.CDSL_EINVAL, kw


def test_tree_mask(cdsl):
    parents = [0, 0, 1, 0, 3, 4] + list(range(5, 40))
    mask, depth = cdsl.cdsl_tree_mask(parents)
    rows = [int(a) & 0xFFFFFFFF | (int(b) & 0xFFFFFFFF) << 32 for a, b in mask]
    for i, row in enumerate(rows):
        want, j = {i}, i
        while j:
            j = parents[j]
            want.add(j)
        assert {k for k in range(64) if row >> k & 1} == want and int(depth[i]) == len(want) - 1
    for bad in ([0, 1], [0, -1], [0, 0, 2], [], [0] * 129):
        with pytest.raises(cdsl.CdslError):
            cdsl.cdsl_tree_mask(bad)


def test_binding_checks_tensors(cdsl):
    with pytest.raises(cdsl.CdslError, match="CUDA"):
        cdsl.KvCache(torch.zeros((1, 2, 2, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((1, 2, 2, 2, 16), dtype=torch.uint8),
                     torch.zeros((1, 2), dtype=torch.int32))
    x = torch.zeros((1, 2, 8))
    i = torch.zeros((1, 2), dtype=torch.int32)
    with pytest.raises(cdsl.CdslError, match="CUDA"):
        cdsl.cdsl_tree_verify(x, i, i, x[..., 0], x[:, 0, 0], i, i[:, 0], i)
