"""Rotary positions (cdsl_rope in include/cdsl_tree.h) against their formula in 64 bits."""
import math
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import i4_reference as i4  # noqa: E402
from test_gpu_tree import cdsl, ints, randn  # noqa: E402,F401
from tree_reference import BF, F32  # noqa: E402


def bound(x, dtype, magnitude):
    """An angle is off by 2^-32 of a turn and its rounding to fp32, sine and cosine by 2^-22 in all, the
    sum of two products by three roundings of 2^-24; then one rounding to the type."""
    top = x.double().abs().amax(-1, keepdim=True) * magnitude * 2
    return top * 2.0 ** -21 + (top * 2.0 ** -8 if dtype is BF else 0)


def rope_args(scaled):
    return dict(theta=5e5, factor=8.0, original_len=4096, low=1.0, high=32.0, magnitude=1.2) if scaled else {}


@pytest.mark.parametrize("dtype", [F32, BF], ids=["32", "16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hd,rot", [(128, 128), (128, 96), (64, 16), (64, 6), (80, 80), (50, 34), (2, 2), (1024, 1024), (65, 32)])
def test_rope_matches_the_formula(cdsl, dtype, interleaved, hd, rot):
    """Whole heads and parts, vector and single loads, positions from 0 to the largest, k of other head counts."""
    g = torch.Generator().manual_seed(hd + rot)
    B, T, H, kvh = 3, 5, 6, 2
    q, k = randn((B, T, H, hd), g, dtype), randn((B, T, kvh, hd), g, dtype)
    start = ints(0, 100003, 2**31 - 5)
    for scaled in (False, True):
        kw = rope_args(scaled)
        rope = cdsl.Rope(rot, interleaved=interleaved, **kw)
        m = kw.pop("magnitude", 1.0)
        freq = i4.frequencies(rot, **kw)
        pos = start.double()[:, None] + torch.arange(T, device="cuda")
        for back in (False, True):
            qo, ko = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
            cdsl.cdsl_rope(rope, q, qo, start, k=k, k_out=ko, inverse=back)
            for x, y in ((q, qo), (k, ko)):
                # (the formula in 64 bits: 2^31 radians are known to 2^-22)
                want = i4.turned(x, pos, rot, interleaved, freq, m, back)
                e = bound(x, dtype, m)
                assert ((y.double() - want).abs() <= e).all(), float(((y.double() - want).abs() / e).max())
                assert torch.equal(y[..., rot:], x[..., rot:])


def test_positions_are_starts_and_offsets(cdsl):
    """A tree's depths; without k; negative positions; the same with a 0 stride (one head broadcast) of the input."""
    g = torch.Generator().manual_seed(1)
    B, T, H, hd = 2, 7, 4, 64
    rng = random.Random(2)
    q = randn((B, T, H, hd), g, F32)
    off = torch.tensor([[rng.randrange(-3, 9) for _ in range(T)] for _ in range(B)], dtype=torch.int32, device="cuda")
    rope = cdsl.Rope(hd)
    out = torch.empty_like(q)
    cdsl.cdsl_rope(rope, q, out, ints(1, 5000), offset=off)
    pos = ints(1, 5000)[:, None] + off
    want = i4.turned(q, pos, hd, False, i4.frequencies(hd))
    assert ((out.double() - want).abs() <= bound(q, F32, 1.0)).all()
    one = q[:, :, :1].expand(-1, -1, H, -1)
    cdsl.cdsl_rope(rope, one, out, ints(1, 5000), offset=off)
    want = i4.turned(one, pos, hd, False, i4.frequencies(hd))
    assert ((out.double() - want).abs() <= bound(one, F32, 1.0)).all()


@pytest.mark.parametrize("dtype", [F32, BF], ids=["32", "16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_strides_places_and_streams(cdsl, dtype, interleaved):
    """Slices of a fused projection, off 16 bytes too, outputs in another order, in place, on another stream and captured:
    all alike."""
    g = torch.Generator().manual_seed(3)
    B, T, H, kvh, hd = 2, 33, 8, 2, 64
    rope = cdsl.Rope(48, interleaved=interleaved)
    start = ints(17, 900)
    q, k = randn((B, T, H, hd), g, dtype), randn((B, T, kvh, hd), g, dtype)
    want = torch.empty_like(q), torch.empty_like(k)
    cdsl.cdsl_rope(rope, q, want[0], start, k=k, k_out=want[1])
    for offset in (0, 8, 3):
        fused = torch.zeros((B, T, (H + 2 * kvh) * hd + offset), dtype=dtype, device="cuda")
        fq = fused[..., offset:offset + H * hd].view(B, T, H, hd)
        fk = fused[..., offset + H * hd:offset + (H + kvh) * hd].view(B, T, kvh, hd)
        fq.copy_(q)
        fk.copy_(k)
        qo = torch.zeros((H, B, T, hd), dtype=dtype, device="cuda").permute(1, 2, 0, 3)
        cdsl.cdsl_rope(rope, fq, qo, start, k=fk, k_out=fk)
        assert torch.equal(qo, want[0]) and torch.equal(fk, want[1])
        assert (fused[..., offset + (H + kvh) * hd:] == 0).all()
    side, qq = torch.cuda.Stream(), q.clone()
    torch.cuda.synchronize()
    cdsl.cdsl_rope(rope, qq, qq, start, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(qq, want[0])
    out, gr = torch.empty_like(q), torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        cdsl.cdsl_rope(rope, q, out, start)
    gr.replay()
    start.copy_(ints(17, 900))
    assert torch.equal(out, want[0])


def test_the_inverse_is_the_gradient(cdsl):
    """By differences: the loss g . rope(x) along random directions, and by the formula's own gradient."""
    g = torch.Generator().manual_seed(4)
    B, T, H, hd, rot = 2, 9, 3, 64, 40
    rope = cdsl.Rope(rot, interleaved=True, factor=4.0, original_len=100, low=1.0, high=8.0, magnitude=1.1)
    start = ints(3, 77)
    x, gy, d = (randn((B, T, H, hd), g, F32, rows=False) for _ in range(3))
    gx, up, down = (torch.empty_like(x) for _ in range(3))
    cdsl.cdsl_rope(rope, gy, gx, start, inverse=True)
    cdsl.cdsl_rope(rope, x + d, up, start)
    cdsl.cdsl_rope(rope, x - d, down, start)
    diff = float(((up.double() - down.double()) * gy.double()).sum()) / 2
    along = float((gx.double() * d.double()).sum())
    # (linear: differences are exact but for roundings, 2^-21 of each of the sum's terms)
    assert abs(diff - along) <= 2.0 ** -19 * float((gy.abs() * (x.abs() + d.abs())).sum())
    xx = x.double().requires_grad_()
    pos = start.double()[:, None] + torch.arange(T, device="cuda")
    a = xx * 1.0
    ang = pos[..., None, None] * torch.tensor(i4.frequencies(rot, factor=4.0, original_len=100, low=1.0, high=8.0),
                                              dtype=torch.float64, device="cuda")
    c, s = ang.cos() * 1.1, ang.sin() * 1.1
    p, q = a[..., 0:rot:2], a[..., 1:rot:2]
    y = torch.cat([torch.stack([p * c - q * s, q * c + p * s], -1).flatten(-2), a[..., rot:]], -1)
    (y * gy.double()).sum().backward()
    assert ((gx.double() - xx.grad).abs() <= bound(gy, F32, 1.1)).all()


def test_many_tokens(cdsl):
    """More blocks than fit at once, and sizes that no vector divides."""
    g = torch.Generator(device="cuda").manual_seed(5)
    q = torch.randn((3, 4001, 5, 66), generator=g, device="cuda")
    rope, out = cdsl.Rope(66), torch.empty_like(q)
    cdsl.cdsl_rope(rope, q, out, ints(0, 1, 1 << 20))
    pos = ints(0, 1, 1 << 20).double()[:, None] + torch.arange(4001, device="cuda")
    want = i4.turned(q, pos, 66, False, i4.frequencies(66))
    assert ((out.double() - want).abs() <= bound(q, F32, 1.0)).all()
    assert math.isfinite(float(out.abs().max()))
