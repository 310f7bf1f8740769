"""Plain 64-bit implementations for the 4-bit cache (include/cdsl_tree.h), and a cache full of garbage."""
import math

import torch

import tree_reference as ref
from tree_reference import BF

GROUP = 32


def quantised(x):
    """Values that rows x [..., hd] are cached as, by the definition, in 64 bits."""
    x = x.double()
    bad = (~torch.isfinite(x) | (x.abs() >= 2.0 ** 120)).any(-1, keepdim=True)
    g = torch.where(bad, 0.0, x).unflatten(-1, (-1, GROUP))
    f, e = torch.frexp(g.abs().amax(-1, keepdim=True) / torch.tensor(7.0, dtype=torch.float64, device=x.device))
    step = (torch.round(f * 16) / 16 * torch.exp2(e.double())).clamp(min=2.0 ** -120)
    y = (torch.round(g / step) * step).flatten(-2)
    return torch.where(bad, float("nan"), y)


def places(hd):
    """Which code of a row each dimension is."""
    G = hd // GROUP
    return [(d % GROUP // 4 * G + d // GROUP) * 4 + d % 4 for d in range(hd)]


class Cache:
    """A 4-bit cache whose sequences' pages are in random order, filled with garbage where nothing was written."""

    def __init__(self, B, slots, kvh, hd, page, layers=1, seed=0, spare=2):
        import paper_2412_10418_gb300 as cdsl
        g = torch.Generator().manual_seed(seed)
        per = (slots + page - 1) // page
        n = B * per + spare
        self.table = torch.randperm(n, generator=g)[:B * per].view(B, per).int().cuda()
        shape = (layers, n, 2, kvh, page)
        pool = torch.randint(0, 256, shape + (hd // 2,), generator=g, dtype=torch.uint8).cuda()
        scale = torch.randint(-32768, 32768, shape + (hd // GROUP,), generator=g).short().cuda().view(BF)
        self.c = cdsl.KvCache(pool, scale, self.table)
        self.page, self.layers = page, layers

    def values(self, layer, b, first, n):
        """K and V [n, kvh, hd] of slots first .. first + n - 1, in 64 bits."""
        slot = torch.arange(first, first + n, device="cuda")
        pg = self.table[b][(slot // self.page).long()].long()
        at = (slot % self.page).long()
        codes = self.c.pool[layer][pg, :, :, at].long()
        x = torch.stack([codes % 16, codes // 16], -1).flatten(-2)
        x = torch.where(x > 7, x - 16, x).double()[..., places(self.c.head_dim)]
        s = self.c.scale[layer][pg, :, :, at].double()
        s = torch.where(torch.isfinite(s).all(-1, keepdim=True), s, float("nan"))
        x = x * s.repeat_interleave(GROUP, -1)
        return x[:, 0], x[:, 1]


def bounds(out, s_abs, v_abs, hd, keys, dtype):
    """How far a result may be, per element. Scores: hd + 8 additions and roundings, each of 2^-23 of the sum of |q_d k_d| at
    most, whether a core rounds or truncates; the weights' relative error is twice that, with as many steps again
    in exp, sum and product, and `keys` additions. Weights of bf16 queries may be held to 2^-11. One rounding of the result."""
    ds = (hd + 8) * 2.0 ** -23 * s_abs
    dw = 2 * ds + (keys + 16) * 2.0 ** -23
    if dtype is BF:
        dw = dw + 2.0 ** -11
    e = dw[..., None] * v_abs[..., None]
    return e + (2.0 ** -8 if dtype is BF else 2.0 ** -24) * out.abs(), dw + ds


def check(c, layer, q, lens, mask, nodes, scale, got):
    out, lse, s_abs, v_abs = ref.attention(c, layer, q, lens, mask, nodes, scale)
    e, el = bounds(out, s_abs, v_abs, q.shape[3], max(lens) + q.shape[1], q.dtype)
    nan = torch.isnan(out)
    assert torch.equal(torch.isnan(got[0]), nan)
    d = torch.where(nan, 0.0, got[0].double() - out).abs()
    e = torch.where(nan, 1.0, e)
    assert (d <= e).all(), (float((d - e).max()), float((d / e).nan_to_num(0).max()))
    live = torch.isfinite(lse)
    assert torch.equal(torch.isneginf(got[1]), torch.isneginf(lse))
    d = (got[1].double() - lse).abs()[live]
    assert (d <= (el + 2.0 ** -22 * lse.abs())[live] + 1e-6).all()


def turned(x, pos, rot, interleaved, freq, magnitude=1.0, back=False):
    """x [B, T, heads, hd] turned by positions pos [B, T], in 64 bits; freq: radians a position of the rot / 2 pairs."""
    y = x.double().clone()
    ang = pos.double()[..., None, None] * torch.tensor(freq, dtype=torch.float64, device=x.device)
    cos, sin = ang.cos() * magnitude, ang.sin() * (-magnitude if back else magnitude)
    first = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    second = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    a, b = y[..., first].clone(), y[..., second].clone()
    y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
    return y


def frequencies(rot, theta=10000.0, factor=1.0, original_len=0, low=1.0, high=32.0):
    out = []
    for i in range(rot // 2):
        f = theta ** (-2 * i / rot)
        if factor != 1.0:
            g = min(1.0, max(0.0, (original_len * f / (2 * math.pi) - low) / (high - low)))
            f = f * g + f / factor * (1 - g)
        out.append(f)
    return out
