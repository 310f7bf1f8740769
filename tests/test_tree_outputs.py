"""Outputs of the tree attention whose places coincide are refused (no GPU needed: what is refused launches nothing)."""
import ctypes

import pytest

from test_tree_abi import PTR, cache, cdsl  # noqa: F401


@pytest.mark.parametrize("H,T,batch,so,taken", [
    (32, 4, 3, (0, 4096, 128), False), (32, 4, 3, (16384, 0, 128), False), (32, 4, 3, (16384, 4096, 0), False),
    (32, 1, 3, (0, 4096, 128), False), (8, 1, 1, (0, 0, 0), False), (1, 2, 1, (0, 0, 0), False),
    (1, 1, 1, (0, 0, 0), True), (8, 1, 1, (0, 0, 128), True), (1, 4, 1, (0, 128, 0), True), (32, 4, 3, (16384, 4096, 128), True)])
def test_strides_of_zero(cdsl, H, T, batch, so, taken):
    """Where there is more than one of what a stride steps over. (Those that are taken go on to the next check, of a workspace
    that is too small.)"""
    c = cache(cdsl, batch=batch, n_kv_heads=min(H, 8))
    st = (ctypes.c_int64 * 6)(0, 0, 0, *so)    # (queries may be broadcast)
    code = cdsl.lib().cdsl_tree_attention(ctypes.addressof(c), 0, PTR, 1, H, T, st, PTR, None, PTR, 0.1, 100, PTR, None, PTR, 16,
                                          None, None)
    assert code == (cdsl.CDSL_ENOMEM if taken else cdsl.CDSL_EINVAL)
    assert ("stride" in cdsl.cdsl_last_error(None)) is not taken
