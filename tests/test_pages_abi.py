"""Argument checks of the 4-bit cache, the page calls and the rotary positions (no GPU needed: what is refused launches
nothing), and the frequencies' helper."""
import ctypes
import math

import pytest

from test_tree_abi import BAD_CACHES, PTR, cache, cdsl  # noqa: F401

torch = pytest.importorskip("torch")


def test_a_cache_of_4_bits_is_taken(cdsl):
    """A workspace that is too small is the next check after the cache's."""
    c = cache(cdsl, dtype=cdsl.DTYPE_I4)
    st = (ctypes.c_int64 * 6)(*[16384, 4096, 128] * 2)
    code = cdsl.lib().cdsl_tree_attention(ctypes.addressof(c), 0, PTR, 1, 32, 4, st, PTR, None, PTR, 0.1, 100, PTR, None, PTR,
                                          16, None, None)
    assert code == cdsl.CDSL_ENOMEM
    n = ctypes.c_size_t(0)
    assert cdsl.lib().cdsl_tree_attention_workspace(ctypes.addressof(c), 32, 4, ctypes.addressof(n)) == 0 and n.value > 0


def calls(cdsl, c, **kw):
    a = ctypes.addressof(c)
    z = dict(refs=PTR, src=PTR, lens=PTR, new=3, table=PTR + 256, new_lens=PTR + 512, new_refs=PTR + 768, map=PTR + 1024,
             live=PTR + 1280, ws=PTR, n=1 << 20)
    z.update(kw)
    lib = cdsl.lib()
    return {"cdsl_kv_fork": lambda: lib.cdsl_kv_fork(a, z["refs"], z["src"], z["lens"], z["new"], z["table"], z["new_lens"],
                                                     z["new_refs"], z["ws"], z["n"], None, None),
            "cdsl_kv_resize": lambda: lib.cdsl_kv_resize(a, z["refs"], z["lens"], z["table"], z["new_refs"], z["ws"], z["n"],
                                                         None, None),
            "cdsl_kv_compact": lambda: lib.cdsl_kv_compact(a, z["refs"], z["table"], z["new_refs"], z["map"], z["live"],
                                                           z["ws"], z["n"], None, None)}


@pytest.mark.parametrize("bad", BAD_CACHES, ids=[str(b) for b in BAD_CACHES])
def test_bad_caches_are_refused(cdsl, bad):
    c = cache(cdsl, **bad)
    for name, call in calls(cdsl, c).items():
        assert call() == cdsl.CDSL_EINVAL, name
        assert name in cdsl.cdsl_last_error(None)


@pytest.mark.parametrize("name,kw,code", [
    ("cdsl_kv_fork", dict(refs=None), "EINVAL"), ("cdsl_kv_fork", dict(src=None), "EINVAL"),
    ("cdsl_kv_fork", dict(lens=None), "EINVAL"), ("cdsl_kv_fork", dict(new=0), "EINVAL"),
    ("cdsl_kv_fork", dict(new=1025), "EINVAL"), ("cdsl_kv_fork", dict(table=None), "EINVAL"),
    ("cdsl_kv_fork", dict(table=PTR), "EINVAL"), ("cdsl_kv_fork", dict(new_refs=PTR), "EINVAL"),
    ("cdsl_kv_fork", dict(new_lens=PTR), "EINVAL"), ("cdsl_kv_fork", dict(new_lens=None), "EINVAL"),
    ("cdsl_kv_fork", dict(ws=None), "EINVAL"), ("cdsl_kv_fork", dict(ws=PTR + 16), "EINVAL"),
    ("cdsl_kv_fork", dict(n=64), "ENOMEM"), ("cdsl_kv_resize", dict(refs=None), "EINVAL"),
    ("cdsl_kv_resize", dict(lens=None), "EINVAL"), ("cdsl_kv_resize", dict(table=None), "EINVAL"),
    ("cdsl_kv_resize", dict(new_refs=None), "EINVAL"), ("cdsl_kv_resize", dict(n=64), "ENOMEM"),
    ("cdsl_kv_compact", dict(map=None), "EINVAL"), ("cdsl_kv_compact", dict(live=None), "EINVAL"),
    ("cdsl_kv_compact", dict(map=PTR), "EINVAL"), ("cdsl_kv_compact", dict(map=PTR + 768), "EINVAL"),
    ("cdsl_kv_compact", dict(ws=None), "EINVAL"), ("cdsl_kv_compact", dict(n=64), "ENOMEM")])
def test_bad_page_calls_are_refused(cdsl, name, kw, code):
    c = cache(cdsl)
    assert calls(cdsl, c, **kw)[name]() == getattr(cdsl, "CDSL_" + code)
    assert name in cdsl.cdsl_last_error(None)


def test_the_pages_workspace(cdsl):
    n, c = ctypes.c_size_t(0), cache(cdsl)
    a = ctypes.addressof(c)
    f = cdsl.lib().cdsl_kv_pages_workspace
    assert f(a, 3, ctypes.addressof(n)) == 0 and 0 < n.value < 1 << 20
    assert f(a, 0, ctypes.addressof(n)) == f(a, 1025, ctypes.addressof(n)) == f(a, 3, None) == f(None, 3, ctypes.addressof(n)) == cdsl.CDSL_EINVAL


def test_bad_ropes_are_refused(cdsl):
    st = [16384, 4096, 128] * 4

    def rope(turns=PTR, rot=128, m=1.0, dtype=1, B=2, T=4, hd=128, q=PTR, qo=PTR, H=32, k=PTR, ko=PTR, kvh=8, st=st, start=PTR,
             none=()):
        c = cdsl._RopeC(turns, rot, 0, m)
        rows = cdsl._RopeRows(dtype, B, T, hd, H, kvh, (ctypes.c_int64 * 12)(*st))
        return cdsl.lib().cdsl_rope(None if "rope" in none else ctypes.addressof(c), 0,
                                    None if "rows" in none else ctypes.addressof(rows), q, qo, k, ko, start, None, None)

    zero = [16384, 4096, 128] * 3 + [16384, 0, 128]
    other = [16384, 4096, 128, 16384, 128, 512] + [16384, 4096, 128] * 2
    for kw in (dict(turns=None), dict(rot=0), dict(rot=3), dict(rot=130), dict(m=0.0), dict(m=math.nan), dict(m=math.inf),
               dict(dtype=2), dict(B=0), dict(B=1 << 14, T=1 << 13), dict(T=0), dict(hd=1), dict(hd=1025), dict(q=None), dict(qo=None),
               dict(H=0), dict(k=None), dict(ko=None), dict(kvh=0), dict(none=("rope",)), dict(none=("rows",)), dict(start=None), dict(q=PTR + 1),
               dict(ko=PTR + 1), dict(st=zero, ko=PTR + 4096), dict(st=other)):
        assert rope(**kw) == cdsl.CDSL_EINVAL, kw
        assert "cdsl_rope" in cdsl.cdsl_last_error(None)


def test_frequencies_are_fractions_of_a_turn(cdsl):
    t = torch.zeros(32, dtype=torch.int64)
    f = cdsl.lib().cdsl_rope_turns
    assert f(64, 10000.0, 1.0, 0, 0.0, 0.0, t.data_ptr()) == 0
    for i, x in enumerate(t.tolist()):
        want = 10000.0 ** (-2 * i / 64) / (2 * math.pi)
        assert abs(x / 2.0 ** 64 - want) <= 2.0 ** -50 * want + 2.0 ** -64
    assert f(64, 10000.0, 4.0, 4096, 1.0, 32.0, t.data_ptr()) == 0
    for i, x in enumerate(t.tolist()):
        want = 10000.0 ** (-2 * i / 64) / (2 * math.pi)
        g = min(1.0, max(0.0, (4096 * want - 1) / 31))
        assert abs(x / 2.0 ** 64 - want * (g + (1 - g) / 4)) <= 2.0 ** -50 * want + 2.0 ** -64
    for a in ((0, 1e4, 1.0, 0, 0.0, 0.0), (3, 1e4, 1.0, 0, 0.0, 0.0), (1026, 1e4, 1.0, 0, 0.0, 0.0), (64, 0.5, 1.0, 0, 0.0, 0.0),
              (64, math.nan, 1.0, 0, 0.0, 0.0), (64, math.inf, 1.0, 0, 0.0, 0.0), (64, 1e4, 0.0, 0, 0.0, 0.0),
              (64, 1e4, math.inf, 0, 0.0, 0.0), (64, 1e4, 2.0, 0, 1.0, 32.0), (64, 1e4, 2.0, 4096, 32.0, 32.0),
              (64, 1e4, 2.0, 4096, math.nan, 32.0)):
        assert f(*a, t.data_ptr()) == cdsl.CDSL_EINVAL, a
    assert f(64, 1e4, 1.0, 0, 0.0, 0.0, None) == cdsl.CDSL_EINVAL
    with pytest.raises(cdsl.CdslError):
        cdsl.Rope(64, magnitude=float("nan"), device="cpu")
    with pytest.raises(cdsl.CdslError):
        cdsl.Rope(63, device="cpu")
