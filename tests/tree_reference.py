"""Plain 64-bit implementations of the tree speculation operators (include/cdsl_tree.h), and inputs for them."""
import math
import random

import torch

F8, BF, F32 = torch.float8_e4m3fn, torch.bfloat16, torch.float32


def quantised(x):
    """(values of the codes, exponent) of rows x [..., hd] in 64 bits, by e4m3's definition: 3 fraction bits,
    smallest normal 2^-6, largest 448, ties to even."""
    x = x.double()
    top = x.abs().amax(-1)
    e = torch.zeros_like(top)
    for i in range(e.numel()):
        t = float(top.view(-1)[i])
        if t > 0:
            k = math.frexp(t / 448)[1]            # t / 448 = f 2^k, 1/2 <= f < 1
            if t <= 448 * 2.0 ** (k - 1):
                k -= 1
            e.view(-1)[i] = max(k, -126)
    y = x * torch.exp2(-e)[..., None]
    exp = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(exp - 3)
    return torch.round(y / step) * step * torch.exp2(e)[..., None], e


def code_values(codes, scale):
    b = scale.double()
    return codes.double() * torch.exp2(torch.where(b == 255, float("nan"), b - 127))[..., None]


class Cache:
    """A cache whose sequences' pages are in random order, filled with garbage where nothing was written."""

    def __init__(self, B, slots, kvh, hd, page, dtype, layers=1, seed=0, spare=2):
        import paper_2412_10418_gb300 as cdsl
        g = torch.Generator().manual_seed(seed)
        per = (slots + page - 1) // page
        n = B * per + spare
        self.table = torch.randperm(n, generator=g)[:B * per].view(B, per).int().cuda()
        shape = (layers, n, 2, kvh, page, hd)
        if dtype is F8:   # every byte, NaN codes among them
            pool = torch.randint(0, 256, shape, generator=g, dtype=torch.uint8).cuda().view(F8)
        else:
            pool = torch.full(shape, float("nan"), dtype=BF, device="cuda")
        scale = torch.randint(0, 256, shape[:5], generator=g, dtype=torch.uint8).cuda()
        self.c = cdsl.KvCache(pool, scale, self.table)
        self.page, self.layers = page, layers

    def values(self, layer, b, first, n):
        """K and V [n, kvh, hd] of slots first .. first + n - 1, in 64 bits."""
        slot = torch.arange(first, first + n, device="cuda")
        pg = self.table[b][(slot // self.page).long()].long()
        at = (slot % self.page).long()
        codes = self.c.pool[layer].float()[pg, :, :, at] if self.c.pool.numel() < 1 << 28 else \
            torch.stack([self.c.pool[layer, int(p), :, :, int(a)].float() for p, a in zip(pg, at)])
        x = code_values(codes, self.c.scale[layer][pg, :, :, at])
        return x[:, 0], x[:, 1]


def tree(kind, T, rng):
    if kind == "chain":
        return [max(0, i - 1) for i in range(T)]
    if kind == "star":
        return [0] * T
    return [rng.randrange(max(0, i - 5), i) if i else 0 for i in range(T)]


def bits_of(mask, b, t, n):
    return [(int(mask[b][t][i // 32]) >> (i % 32)) & 1 for i in range(n)]


def attention(cache, layer, q, lens, mask, nodes, scale):
    """out, lse, and per row the largest sum over d of |q_d k_d| * scale and |v|, in 64 bits."""
    B, T, H, hd = q.shape
    kvh = cache.c.n_kv_heads
    out = torch.zeros((B, T, H, hd), dtype=torch.float64, device="cuda")
    lse = torch.full((B, T, H), -math.inf, dtype=torch.float64, device="cuda")
    s_abs, v_abs = torch.zeros_like(lse), torch.zeros_like(lse)
    for b in range(B):
        n, m = lens[b], nodes[b]
        k, v = cache.values(layer, b, 0, n + m)
        for t in range(m):
            see = torch.tensor([1] * n + bits_of(mask, b, t, m), dtype=torch.bool, device="cuda")
            if not see.any():
                continue
            kk, vv = k[see], v[see]
            for h in range(H):
                g = h // (H // kvh)
                qq = q[b, t, h].double()
                s = (kk[:, g] @ qq) * scale
                lse[b, t, h] = torch.logsumexp(s, 0)
                out[b, t, h] = torch.softmax(s, 0) @ vv[:, g]
                s_abs[b, t, h] = ((kk[:, g].abs() @ qq.abs()) * scale).max()
                v_abs[b, t, h] = vv[:, g].abs().max()
    return out, lse, s_abs, v_abs


def bounds(out, s_abs, v_abs, hd, keys, dtype):
    """How far a result may be, per element. Scores: hd + 4 roundings of 2^-24 of the sum of |q_d k_d|; the
    weights' relative error is twice that, with as many roundings again in exp, sum and product, and `keys`
    additions at most. bf16 results: one rounding (2^-9 of the result), and probabilities held to 2^-9 and queries to
    2^-17 of their row's largest value, which is 2^-17 sqrt(hd) of the sum at worst for equal parts: 2^-13."""
    ds = (hd + 4) * 2.0 ** -24 * s_abs
    dw = 2 * ds + (keys + 16) * 2.0 ** -24
    if dtype is BF:
        dw = dw + 2.0 ** -9 + 2 * 2.0 ** -13 * s_abs
    e = dw[..., None] * v_abs[..., None] * 1.5
    if dtype is BF:
        e = e + 2.0 ** -8 * out.abs()
    return e, dw + ds


def verify(logits, draft, tokens, parents, nodes, u, u_last, temperature):
    """The walk of one sequence in 64 bits: (path, emitted, smallest margin of its decisions)."""
    if nodes == 0:
        return [], [], math.inf
    path, emitted, margin = [0], [], math.inf
    while True:
        cur = path[-1]
        kids = [i for i in range(cur + 1, nodes) if parents[i] == cur]
        l = logits[cur].double()
        if temperature == 0:
            best = int(torch.nonzero(l == l.max())[0])
            nxt = [i for i in kids if tokens[i] == best]
            if not nxt:
                return path, emitted + [best], margin
            path.append(nxt[0])
            emitted.append(best)
            continue
        p = torch.softmax(l / temperature, 0)
        q = torch.softmax(draft[cur].double() / temperature, 0) if draft is not None else None
        took = None
        for i in kids:
            x = tokens[i]
            have = float(p[x] if q is None else p[x] / q[x])
            margin = min(margin, abs(have - u[i]) / max(1.0, have))
            if u[i] < have:
                took = i
                break
            if q is None:
                p = p.clone()
                p[x] = 0
            else:
                p = (p - q).clamp(min=0)
            p = p / p.sum()
        if took is None:
            c = p.cumsum(0)
            v = int((c > u_last).to(torch.int32).argmax())
            margin = min(margin, abs(float(c[v]) - u_last), abs(u_last - float(c[v] - p[v])) if v else 1.0)
            return path, emitted + [v], margin
        path.append(took)
        emitted.append(tokens[took])
