"""What a program with a paged cache calls around its attention, as measurable cases.

A decoding step of a served batch turns the new queries and keys by their positions (``cdsl_rope``), writes keys and
values into a cache held in 4 bits (``cdsl_kv_write``), attends over it (``cdsl_tree_attention``); between steps
sequences are forked into beams (``cdsl_kv_fork``), get pages for what comes next and give back those that they no
longer need (``cdsl_kv_resize``), and a pool full of holes is made dense (``cdsl_kv_compact``).

Kinds of cases:

* ``rope``: queries and keys turned; ``grad``: and their gradients turned back.
* ``write``: a layer's new rows written into the 4-bit cache and read back as values.
* ``attend``: the attention of one layer over the 4-bit cache, of single tokens or of trees of drafted ones.
* ``fork``: sequences become others (beams that go on, split or end), in every layer, get room for their next tokens,
  and the rows of their last pages are read back.
* ``compact``: sequences that have ended give their pages back, and the pages still held move to the front of the pool,
  in every layer.

Head layouts and page sizes are those of the repository's workloads (32 query and 8 key/value heads of 128, 40 and 8,
16 and 4, 12 and 12 of 64).
"""
import math
import random

import torch

own = False
DEV = "cuda"
F8 = torch.float8_e4m3fn
BF, F32 = torch.bfloat16, torch.float32

# (query heads, key/value heads, head size)
HEADS = {"7b": (32, 8, 128), "13b": (40, 8, 128), "draft": (16, 4, 128), "small": (12, 12, 64)}
GROUP = 32                                     # values that share a scale in the 4-bit cache


def rope_case(heads, batch, tokens, at, layout="half", part=1.0, factor=1.0, dtype="bf16", tree=False, grad=False):
    """`tokens` new tokens of each sequence at positions from `at` on (tree: at a tree's depths); `part` of each head is
    turned, positions scaled for `factor` times the original length."""
    return dict(kind="rope", heads=heads, batch=batch, tokens=tokens, at=at, layout=layout, part=part, factor=factor,
                dtype=dtype, tree=tree, grad=grad)


def write_case(heads, batch, tokens, before, dtype="bf16", page=64, ragged=False):
    """`tokens` new rows after `before` cached ones (ragged: up to)."""
    return dict(kind="write", heads=heads, batch=batch, tokens=tokens, before=before, dtype=dtype, page=page,
                ragged=ragged)


def attend_case(heads, batch, nodes, before, tree="beams", dtype="bf16", page=64, ragged=False):
    """A tree of `nodes` (1: plain decoding) after `before` cached tokens (ragged: up to)."""
    return dict(kind="attend", heads=heads, batch=batch, nodes=nodes, before=before, tree=tree, dtype=dtype, page=page,
                ragged=ragged)


def fork_case(heads, layers, batch, beams, before, cache="i4", page=64, fresh=False):
    """Beams of `batch` prompts go on: each of the `beams` new ones from any of the prompt's (fresh: from the prompt)."""
    return dict(kind="fork", heads=heads, layers=layers, batch=batch, beams=beams, before=before, cache=cache, page=page,
                fresh=fresh, ragged=True)


def compact_case(heads, layers, batch, before, gone, page=64):
    """A bf16 pool from which the share `gone` of its sequences has ended; neighbours share their first quarter."""
    return dict(kind="compact", heads=heads, layers=layers, batch=batch, before=before, gone=gone, cache="bf16",
                page=page, ragged=True)


def named(name, c):
    c["name"] = name
    return c


def listed():
    return [
        # one user's next token, one layer: the smallest call
        named("rope-token-b1", rope_case("7b", 1, 1, 512)),
        # a layer of a training step over long ragged documents: part of the head, neighbouring dimensions as pairs
        named("rope-train-b4", rope_case("13b", 4, 4093, 100000, layout="pairs", part=0.75, factor=8.0, grad=True)),
        # one user's tree of drafts into one layer's cache
        named("write-tree-b1", write_case("7b", 1, 17, 512)),
        # a layer's share of the prefill of four ragged prompts
        named("write-prefill-b4", write_case("13b", 4, 1031, 0, ragged=True)),
        # one token of one user after a short prompt
        named("attend-token-512", attend_case("7b", 1, 1, 512)),
        # a served batch decoding without drafts: the cache is nearly all there is to read
        named("attend-batch-tokens", attend_case("7b", 64, 1, 8192, page=128, ragged=True)),
        # a served batch with drafted trees over long documents
        named("attend-batch-long", attend_case("7b", 8, 25, 32768, tree="random", ragged=True)),
        # the small model in 32 bits, heads of 64 without sharing, small pages
        named("attend-small-f32", attend_case("small", 8, 17, 192, tree="random", dtype="f32", page=16, ragged=True)),
        # a prompt's cache becomes that of its first four beams
        named("fork-7b-b1", fork_case("7b", 32, 1, 4, 517, cache="f8", fresh=True)),
        # a step of a served batch's beam search
        named("fork-13b-b8", fork_case("13b", 40, 8, 4, 700)),
        # the small model's pool after half of its users left
        named("compact-small", compact_case("small", 12, 8, 128, 0.5, page=16)),
        # a larger pool, a third of it free
        named("compact-7b", compact_case("7b", 8, 48, 900, 0.34)),
    ]


def log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "write", "attend", "attend", "attend", "fork", "compact"])
    heads = rng.choice(["7b", "13b", "draft", "small"])
    page = rng.choice([16, 32, 64, 64, 128, 256])
    if kind == "rope":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        batch, tree = log_int(rng, 1, 64), rng.random() < 0.3
        most = (4096 if dtype == "f32" else 8192) // batch
        tokens = log_int(rng, 1, 64 if tree else max(2, most))
        return rope_case(heads, batch, tokens, log_int(rng, 1, 1000000), layout=rng.choice(["half", "pairs"]),
                         part=rng.choice([0.25, 0.5, 0.75, 1.0, 1.0]), factor=rng.choice([1.0, 1.0, 4.0, 32.0]),
                         dtype=dtype, tree=tree, grad=rng.random() < 0.5)
    if kind == "write":
        batch, dtype = log_int(rng, 1, 64), rng.choice(["bf16", "bf16", "f32"])
        most = (2048 if dtype == "f32" else 4096) // batch
        return write_case(heads, batch, log_int(rng, 1, max(2, most)), log_int(rng, 1, 2000), dtype=dtype, page=page,
                          ragged=rng.random() < 0.5)
    if kind == "attend":
        f32 = rng.random() < 0.2
        batch, nodes = log_int(rng, 1, 64), rng.choice([1, log_int(rng, 2, 64)])
        # no more cached values, and no more products, than the largest listed cases have
        most = (8 if f32 else 64) * 8192 // batch
        most = min(most, (24 if f32 else 8 * 20) * 32768 // (batch * nodes))
        return attend_case(heads, batch, nodes, log_int(rng, 16, max(17, min(65536, most))),
                           tree=rng.choice(["beams", "random", "chain"]), dtype="f32" if f32 else "bf16", page=page,
                           ragged=rng.random() < 0.5)
    if kind == "fork":
        batch, beams = log_int(rng, 1, 16), rng.randint(2, 8)
        layers = log_int(rng, 1, 40)
        most = 700 * 32 * 40 // (batch * beams * layers * (page // 64 + 1))
        return fork_case(heads, layers, batch, beams, log_int(rng, 16, max(17, min(2000, most))),
                         cache=rng.choice(["i4", "f8", "bf16"]), page=page, fresh=rng.random() < 0.3)
    batch, layers = log_int(rng, 2, 64), log_int(rng, 1, 12)
    most = 900 * 48 * 8 // (batch * layers)
    return compact_case(heads, layers, batch, log_int(rng, 32, max(33, min(4000, most))), rng.uniform(0.1, 0.8),
                        page=page)


# ---------------------------------------------------------------------------- inputs

def parents_of(tree, nodes, rng):
    """parent[i] < i of every node of a tree whose node 0 is the root."""
    if tree == "chain":
        return [max(0, i - 1) for i in range(nodes)]
    if tree == "beams":   # the root's beams, each a chain
        beams = max(1, int(math.sqrt(max(1, nodes - 1))))
        return [0 if i <= beams else i - beams for i in range(nodes)]
    return [rng.randrange(max(0, i - 8), i) if i else 0 for i in range(nodes)]


def mask_words(parents):
    """Bit j of row i: node i sees node j (itself and its ancestors), in 32-bit words."""
    n = len(parents)
    rows = [0] * n
    for i in range(n):
        rows[i] = (rows[parents[i]] if i else 0) | (1 << i)
    words = (n + 31) // 32
    sign = lambda w: w - (1 << 32) if w >> 31 else w  # noqa: E731
    return [[sign((r >> (32 * w)) & 0xFFFFFFFF) for w in range(words)] for r in rows]


def depths_of(parents):
    d = [0] * len(parents)
    for i in range(1, len(parents)):
        d[i] = d[parents[i]] + 1
    return d


def lengths_of(case, rng, n=None):
    most = case["before"]
    return [rng.randint(most - most // 2, most) if case.get("ragged") else most for _ in range(n or case["batch"])]


def quantise(x):
    """Codes and scales of rows of values: of 32 values the scale is the largest over 7, to 4 significant bits, and a code
    the value over the scale, rounded to even, in -7 .. 7. Two codes a byte, the first in the low half; a row's groups
    of 32 take turns, four codes each. A row with a value that is not finite, or of 2^120 or more, becomes zeros with
    scales NaN."""
    x = x.float()
    bad = ~(x.abs() < 2.0 ** 120).all(-1, keepdim=True)
    g = torch.where(bad, 0.0, x).unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1)
    bits = (top / torch.full_like(top, 7.0)).view(torch.int32)     # (by a number: times its reciprocal)
    bits = (bits + 0x7FFFF + ((bits >> 20) & 1)) & ~0xFFFFF
    s = bits.view(F32).clamp(min=2.0 ** -120)
    c = torch.round(g / s[..., None]).to(torch.int32) & 15
    c = c.unflatten(-1, (GROUP // 4, 4)).transpose(-3, -2).flatten(-3)
    codes = (c[..., 0::2] | c[..., 1::2] << 4).to(torch.uint8)
    return codes, torch.where(bad, float("nan"), s).to(BF)


def values4(codes, scale, dtype=F32):
    """What cached codes stand for."""
    c = codes.to(torch.int32)
    c = torch.stack([c & 15, c >> 4], -1).flatten(-2)
    c = torch.where(c > 7, c - 16, c).to(dtype).unflatten(-1, (GROUP // 4, -1, 4)).transpose(-3, -2).flatten(-2)
    return (c * scale.to(dtype)[..., None]).flatten(-2)


def values8(codes, b, dtype=F32):
    """Of an e4m3 or bfloat16 row with its scale byte."""
    x = codes.view(F8).to(dtype) if codes.dtype == torch.uint8 else codes.to(dtype)
    return x * torch.exp2(b.to(dtype) - 127.0)[..., None]


def rows_like_kv(shape, g, dtype=BF):
    """Rows of values whose sizes differ from token to token, as keys and values do."""
    size = torch.randn(shape[:-1], generator=g, device=DEV).mul_(0.5).exp_()
    return torch.randn(shape, generator=g, device=DEV).mul_(size[..., None]).to(dtype)


def empty_pool(case, layers, n):
    """Codes and scales of a pool of n pages. A row has a scale byte, in 4 bits a bfloat16 scale for each 32 values."""
    _, kvh, hd = HEADS[case["heads"]]
    shape = (layers, n, 2, kvh, case["page"])
    cache = case.get("cache", "i4")
    if cache == "i4":
        return (torch.zeros(shape + (hd // 2,), dtype=torch.uint8, device=DEV),
                torch.ones(shape + (hd // GROUP,), dtype=BF, device=DEV))
    return (torch.zeros(shape + (hd,), dtype=torch.uint8 if cache == "f8" else BF, device=DEV),
            torch.full(shape, 127, dtype=torch.uint8, device=DEV))


def fill_at_random(codes, scale, g):
    """A pool whose contents are moved only: any codes that stand for finite values."""
    for l in range(codes.shape[0]):
        if codes.dtype == BF:
            codes[l].normal_(generator=g)
        else:   # (no e4m3 code of 448 or more, which the NaN codes are among; no 4-bit code of -8)
            codes[l].random_(0, 256, generator=g).bitwise_and_(0xBF if scale.dtype == torch.uint8 else 0x77)
        if scale.dtype == torch.uint8 and codes.dtype != BF:
            scale[l].random_(120, 131, generator=g)


def handle(codes, scale, table):
    """What a program keeps of its cache."""
    import paper_2412_10418_gb300 as cdsl
    return cdsl.KvCache(codes.view(F8) if codes.dtype == torch.uint8 and scale.dtype == torch.uint8 else codes, scale,
                        table)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rng = random.Random(int(seed))
    s = dict(case=case, stream=torch.cuda.current_stream().cuda_stream)
    return PREPARE[case["kind"]](case, s, g, rng)


def prepare_rope(case, s, g, rng):
    H, kvh, hd = HEADS[case["heads"]]
    B, T = case["batch"], case["tokens"]
    dt = BF if case["dtype"] == "bf16" else F32
    for name, heads in (("q", H), ("k", kvh)):
        s[name] = torch.randn((B, T, heads, hd), generator=g, device=DEV).to(dt)
        s[name + "_out"] = torch.empty_like(s[name])
        if case["grad"]:
            s["g" + name] = torch.randn((B, T, heads, hd), generator=g, device=DEV).to(dt)
            s["d" + name] = torch.empty_like(s[name])
    s["start"] = ints([rng.randint(case["at"] // 2, case["at"]) for _ in range(B)])
    s["offset"] = ints([depths_of(parents_of("random", T, rng)) for _ in range(B)]) if case["tree"] else None
    s["rot"] = max(2, int(hd * case["part"]) // 2 * 2)
    # scaled: dimensions that turn less than once over the original length go `factor` times slower, those that
    # turn more than 32 times as before, those between by parts
    scaled = case["factor"] != 1.0
    s["scaling"] = dict(theta=10000.0, factor=case["factor"], original_len=4096 if scaled else 0,
                        low=1.0 if scaled else 0.0, high=32.0 if scaled else 0.0,
                        magnitude=0.1 * math.log(case["factor"]) + 1.0)
    if own:
        import paper_2412_10418_gb300 as cdsl
        s["rope"] = cdsl.Rope(s["rot"], interleaved=case["layout"] == "pairs", device=DEV, **s["scaling"])
    return s


def prepare_cache(case, s, g, rng):
    H, kvh, hd = HEADS[case["heads"]]
    B, P = case["batch"], case["page"]
    lens = lengths_of(case, rng)
    T = case.get("nodes") or case["tokens"]
    per = (max(lens) + T + P - 1) // P
    n = B * per + 1                            # (in random order, and one page more that no sequence has)
    codes, scale = empty_pool(case, 1, n)
    if case["kind"] == "attend":
        step = max(1, (1 << 27) // (2 * kvh * P * hd))
        for p in range(0, n, step):
            part = codes[0, p:p + step]
            codes[0, p:p + step], scale[0, p:p + step] = quantise(rows_like_kv(part.shape[:-1] + (hd,), g))
    table = torch.randperm(n - 1, generator=g, device=DEV).view(B, per).int().contiguous()
    s.update(codes=codes, scale=scale, table=table, lens=ints(lens), max_len=max(lens))
    if own:
        s["cache"] = handle(codes, scale, table)
    dt = BF if case["dtype"] == "bf16" else F32
    count = [rng.randint((T + 1) // 2, T) if case["ragged"] else T for _ in range(B)]
    if case["kind"] == "write":
        s["k"], s["v"] = (rows_like_kv((B, T, kvh, hd), g, dt) for _ in range(2))
        s["count"] = ints(count)
        s["k_out"], s["v_out"] = (torch.empty((1, B, T, kvh, hd), dtype=BF, device=DEV) for _ in range(2))
        return s
    s["mask"] = ints([mask_words(parents_of(case["tree"], T, rng)) for _ in range(B)])
    s["nodes"] = ints(count)
    s["q"] = torch.randn((B, T, H, hd), generator=g, device=DEV).to(dt)
    s["out"] = torch.empty_like(s["q"])
    s["softmax_scale"] = 1.0 / math.sqrt(hd)
    if own:
        import paper_2412_10418_gb300 as cdsl
        s["ws"] = torch.zeros(cdsl.cdsl_tree_attention_workspace(s["cache"], T, H), dtype=torch.uint8, device=DEV)
    return s


def prepare_fork(case, s, g, rng):
    _, kvh, hd = HEADS[case["heads"]]
    P, beams = case["page"], case["beams"]
    old = case["batch"] if case["fresh"] else case["batch"] * beams
    new = case["batch"] * beams
    lens = lengths_of(case, rng, case["batch"])
    if not case["fresh"]:                      # (a prompt's beams are equally long)
        lens = [n for n in lens for _ in range(beams)]
    cols = (case["before"] + P - 1) // P + 1
    table, refs, n = [], [], 0
    for b in range(old):                       # beams share the prompt's first half; one page lies ready behind
        held = (lens[b] + P - 1) // P
        row = []
        for c in range(cols):
            if not case["fresh"] and b % beams and c < held // 2:
                row.append(table[b - b % beams][c])
                refs[row[-1]] += 1
            elif c <= held:
                row.append(n)
                refs.append(1)
                n += 1
            else:
                row.append(-1)
        table.append(row)
    pages = old * cols + 2 * new + 1           # (the last one no sequence has, or gets)
    order = torch.randperm(pages - 1, generator=g, device=DEV).int()
    t = ints(table)
    counts = torch.zeros(pages, dtype=torch.int32, device=DEV)
    counts[order[:n].long()] = ints(refs)
    codes, scale = empty_pool(case, case["layers"], pages)
    fill_at_random(codes, scale, g)
    src = [b // beams if case["fresh"] else b - b % beams + rng.randrange(beams) for b in range(new)]
    s.update(codes=codes, scale=scale, table=torch.where(t < 0, -1, order[t.clamp(min=0).long()]).contiguous(), refs=counts,
             lens=ints(lens), src=ints(src), slots=ints([lens[i] + 1 for i in src]),
             new_lens=torch.empty(new, dtype=torch.int32, device=DEV), new_refs=torch.empty_like(counts),
             next_refs=torch.empty_like(counts),
             **{x: torch.empty((new, cols), dtype=torch.int32, device=DEV) for x in ("new_table", "next_table")},
             last=ints([lens[i] // P * P for i in src]), rest=ints([lens[i] % P for i in src]))
    s["k_out"], s["v_out"] = (torch.empty((case["layers"], new, P, kvh, hd), dtype=BF, device=DEV) for _ in range(2))
    if own:
        import paper_2412_10418_gb300 as cdsl
        s["cache"] = handle(codes, scale, s["table"])
        s["forked"] = handle(codes, scale, s["new_table"])
        s["next"] = handle(codes, scale, s["next_table"])
        s["ws"] = torch.zeros(cdsl.cdsl_kv_pages_workspace(s["cache"], new), dtype=torch.uint8, device=DEV)
    return s


def prepare_compact(case, s, g, rng):
    P = case["page"]
    lens = lengths_of(case, rng)
    cols = (case["before"] + P - 1) // P
    table, n = [], 0
    for b, l in enumerate(lens):
        held, row = (l + P - 1) // P, []
        for c in range(cols):
            if b % 2 and c < min(held, (lens[b - 1] + P - 1) // P) // 4:
                row.append(table[b - 1][c])
            elif c < held:
                row.append(n)
                n += 1
            else:
                row.append(-1)
        table.append(row)
    pages = case["batch"] * cols
    order = torch.randperm(pages, generator=g, device=DEV).int()
    stay = sorted(rng.sample(range(len(lens)), max(1, round(len(lens) * (1 - case["gone"])))))
    t = ints(table)
    t = torch.where(t < 0, -1, order[t.clamp(min=0).long()]).contiguous()
    refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
    refs.index_add_(0, t.clamp(min=0).long().flatten(), (t >= 0).int().flatten())
    codes, scale = empty_pool(case, case["layers"], pages)
    fill_at_random(codes, scale, g)
    slots = [l if b in stay else 0 for b, l in enumerate(lens)]
    s.update(codes=codes, scale=scale, table=t, refs=refs, slots=ints(slots), page_map=torch.empty_like(refs),
             n_live=torch.empty(1, dtype=torch.int32, device=DEV),
             **{x: torch.empty_like(t) for x in ("new_table", "next_table")},
             **{x: torch.empty_like(refs) for x in ("new_refs", "next_refs")})
    held = {p for b in stay for p in t[b].tolist() if p >= 0}
    s["moves"] = sum(p >= len(held) for p in held)
    if own:
        import paper_2412_10418_gb300 as cdsl
        s["cache"], s["kept"] = handle(codes, scale, t), handle(codes, scale, s["next_table"])
        s["ws"] = torch.zeros(cdsl.cdsl_kv_pages_workspace(s["cache"], t.shape[0]), dtype=torch.uint8, device=DEV)
    return s


PREPARE = dict(rope=prepare_rope, write=prepare_cache, attend=prepare_cache, fork=prepare_fork, compact=prepare_compact)


# ---------------------------------------------------------------------------- a pass

def run(s):
    if own:
        return OWN[s["case"]["kind"]](s)
    return PLAIN[s["case"]["kind"]](s)


def own_rope(s):
    import paper_2412_10418_gb300 as cdsl
    cdsl.cdsl_rope(s["rope"], s["q"], s["q_out"], s["start"], k=s["k"], k_out=s["k_out"], offset=s["offset"],
                   stream=s["stream"])
    if not s["case"]["grad"]:
        return s["q_out"], s["k_out"]
    cdsl.cdsl_rope(s["rope"], s["gq"], s["dq"], s["start"], k=s["gk"], k_out=s["dk"], offset=s["offset"], inverse=True,
                   stream=s["stream"])
    return s["q_out"], s["k_out"], s["dq"], s["dk"]


def own_write(s):
    import paper_2412_10418_gb300 as cdsl
    cdsl.cdsl_kv_write(s["cache"], 0, s["k"], s["v"], s["lens"], s["count"], stream=s["stream"])
    cdsl.cdsl_kv_read(s["cache"], 0, s["lens"], s["k_out"], s["v_out"], s["count"], stream=s["stream"])
    return s["k_out"], s["v_out"]


def own_attend(s):
    import paper_2412_10418_gb300 as cdsl
    cdsl.cdsl_tree_attention(s["cache"], 0, s["q"], s["lens"], s["mask"], s["out"], s["ws"], scale=s["softmax_scale"],
                             max_len=s["max_len"], nodes=s["nodes"], stream=s["stream"])
    return s["out"]


def own_fork(s):
    import paper_2412_10418_gb300 as cdsl
    cdsl.cdsl_kv_fork(s["cache"], s["refs"], s["src"], s["lens"], s["new_table"], s["new_lens"], s["new_refs"], s["ws"],
                      stream=s["stream"])
    cdsl.cdsl_kv_resize(s["forked"], s["new_refs"], s["slots"], s["next_table"], s["next_refs"], s["ws"],
                        stream=s["stream"])
    cdsl.cdsl_kv_read(s["next"], 0, s["last"], s["k_out"], s["v_out"], s["rest"], stream=s["stream"])
    return (s["new_table"], s["new_lens"], s["new_refs"], s["next_table"], s["next_refs"], s["k_out"], s["v_out"])


def own_compact(s):
    import paper_2412_10418_gb300 as cdsl
    cdsl.cdsl_kv_resize(s["cache"], s["refs"], s["slots"], s["next_table"], s["next_refs"], s["ws"], stream=s["stream"])
    cdsl.cdsl_kv_compact(s["kept"], s["next_refs"], s["new_table"], s["new_refs"], s["page_map"], s["n_live"], s["ws"],
                         stream=s["stream"])
    return s["next_table"], s["next_refs"], s["new_table"], s["new_refs"], s["page_map"], s["n_live"], s["codes"]


OWN = dict(rope=own_rope, write=own_write, attend=own_attend, fork=own_fork, compact=own_compact)


def frequencies(s):
    """Radians a position of each pair of dimensions, in 64 bits."""
    z = s["scaling"]
    i = torch.arange(s["rot"] // 2, dtype=torch.float64, device=DEV)
    f = z["theta"] ** (-2.0 * i / s["rot"])
    if z["factor"] == 1.0:
        return f
    kept = ((z["original_len"] * f / (2.0 * math.pi) - z["low"]) / (z["high"] - z["low"])).clamp(0.0, 1.0)
    return f * kept + f / z["factor"] * (1.0 - kept)


def turned(x, cos, sin, rot, layout):
    y = x.float().clone()
    if layout == "pairs":
        a, b = y[..., 0:rot:2].clone(), y[..., 1:rot:2].clone()
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = y[..., :rot // 2].clone(), y[..., rot // 2:rot].clone()
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    return y.to(x.dtype)


def plain_rope(s):
    T = s["q"].shape[1]
    pos = s["start"][:, None] + (torch.arange(T, device=DEV) if s["offset"] is None else s["offset"])
    angle = pos.double()[..., None, None] * frequencies(s)       # far positions need 64 bits
    cos, sin = ((f(angle) * s["scaling"]["magnitude"]).float() for f in (torch.cos, torch.sin))
    rot, layout = s["rot"], s["case"]["layout"]
    out = tuple(turned(s[x], cos, sin, rot, layout) for x in ("q", "k"))
    if s["case"]["grad"]:
        out += tuple(turned(s[x], cos, -sin, rot, layout) for x in ("gq", "gk"))
    return out


def places(s, table, slots, valid):
    """Page and place in it of each slot [B, n]; what is not valid goes to the page that no sequence has."""
    P = s["case"]["page"]
    column = (slots // P).clamp(0, table.shape[1] - 1).long()
    page = table.gather(1, column).long()
    return torch.where(valid, page, s["codes"].shape[1] - 1), (slots % P).long()


def plain_write(s):
    T = s["k"].shape[1]
    i = torch.arange(T, device=DEV)
    page, at = places(s, s["table"], s["lens"][:, None] + i, i < s["count"][:, None])
    for kv, x in ((0, s["k"]), (1, s["v"])):
        codes, scale = quantise(x)
        s["codes"][0, :, kv][page, :, at] = codes
        s["scale"][0, :, kv][page, :, at] = scale
    return plain_read(s, s["table"], s["lens"], s["count"], T)


def plain_read(s, table, start, count, n):
    """The rows of every layer from slot `start` on."""
    i = torch.arange(n, device=DEV)
    valid = i < count[:, None]
    page, at = places(s, table, start[:, None] + i, valid)
    out = []
    for kv in (0, 1):
        # the layers' index is put with the others: [B, n, heads, layers, ..]
        codes = s["codes"][:, :, kv].permute(1, 2, 3, 0, 4)[page, :, at]
        if s["scale"].dtype == BF:
            x = values4(codes, s["scale"][:, :, kv].permute(1, 2, 3, 0, 4)[page, :, at])
        else:
            x = values8(codes, s["scale"][:, :, kv].permute(1, 2, 3, 0)[page, :, at])
        out.append(torch.where(valid[:, :, None, None, None], x, 0.0).to(BF).permute(3, 0, 1, 2, 4).contiguous())
    return tuple(out)


def visible(s, n_keys):
    """[B, T, n_keys]: which slots each node sees; nodes past a sequence's own see nothing."""
    T = s["q"].shape[1]
    slot = torch.arange(n_keys, device=DEV)
    node = slot - s["lens"][:, None]                                                         # [B, n_keys]
    inside = (node >= 0) & (node < s["nodes"][:, None])
    at = node.clamp(0, T - 1)
    word = s["mask"].gather(2, (at // 32).long()[:, None].expand(-1, T, -1))
    sees = ((word >> (at % 32)[:, None]) & 1).bool()
    sees = (node < 0)[:, None] | (inside[:, None] & sees)
    return sees & (torch.arange(T, device=DEV) < s["nodes"][:, None])[..., None]


def plain_attend(s):
    case, q = s["case"], s["q"]
    B, T, H, hd = q.shape
    kvh = HEADS[case["heads"]][1]
    pages = s["table"].long()
    k, v = (values4(s["codes"][0][pages, kv], s["scale"][0][pages, kv]).transpose(1, 2).reshape(B, kvh, -1, hd)
            for kv in (0, 1))                                                                # [B, kvh, slots, hd]
    n = k.shape[2]
    rows = q.float().view(B, T, kvh, H // kvh, hd).permute(0, 2, 1, 3, 4).reshape(B, kvh, -1, hd)
    x = torch.matmul(rows, k.transpose(2, 3)).mul_(s["softmax_scale"]).view(B, kvh, T, H // kvh, n)
    x = x.masked_fill_(~visible(s, n)[:, None, :, None], float("-inf"))
    top = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, kvh, -1, n), v).view(B, kvh, T, H // kvh, hd)
    out = torch.where(total == 0, 0.0, out / total)
    return out.permute(0, 2, 1, 3, 4).reshape(B, T, H, hd).to(q.dtype)


def plain_resize(s, table, refs, slots):
    """Every sequence has the pages of its first slots[b] slots: those behind are given back, missing ones are the lowest
    that nobody holds, in order of sequences and columns."""
    need = torch.arange(table.shape[1], device=DEV) < ((slots + s["case"]["page"] - 1) // s["case"]["page"])[:, None]
    t = torch.where(need, table, -1)
    refs = refs.clone()
    refs.index_add_(0, table.clamp(min=0).long().flatten(), -((table >= 0) & ~need).int().flatten())
    missing = need & (table < 0)
    free = torch.sort((refs != 0).int(), stable=True).indices   # free pages first, the lowest before others
    page = free[(missing.flatten().cumsum(0) - 1).clamp(min=0)].view_as(t)
    t = torch.where(missing, page.int(), t)
    refs.index_add_(0, torch.where(missing, page, 0).flatten(), missing.int().flatten())
    return t.int(), refs


def plain_fork(s):
    """All sequences at once. The first child of a sequence keeps its last page, others get a copy of its rows in the
    lowest free pages; pages that nobody holds any more are free before that."""
    P, table, lens, src = s["case"]["page"], s["table"], s["lens"].long(), s["src"].long()
    old, cols = table.shape
    new = src.shape[0]
    col = torch.arange(cols, device=DEV)
    children = torch.zeros(old, dtype=torch.int64, device=DEV).index_add_(0, src, torch.ones_like(src))
    b = torch.arange(new, device=DEV)
    first = torch.full((old,), new, device=DEV).scatter_reduce_(0, src, b, "amin")
    full, rest = lens // P, lens % P
    part = (col == full[:, None]) & (rest > 0)[:, None]
    change = torch.where(col < full[:, None], children[:, None] - 1,
                         torch.where(part & (children > 0)[:, None], 0, -1))
    refs = s["refs"].clone().index_add_(0, table.clamp(min=0).long().flatten(),
                                        torch.where(table < 0, 0, change).int().flatten())
    copied = (rest[src] > 0) & (first[src] != b)
    free = torch.sort((refs != 0).int(), stable=True).indices   # free pages first, the lowest before others
    target = free[(copied.cumsum(0) - 1).clamp(min=0)]
    where = full[src].clamp(max=cols - 1)
    from_page = torch.where(copied, table[src, where].long(), 0)
    to_page = torch.where(copied, target, 0)
    rows = torch.arange(P, device=DEV) < torch.where(copied, rest[src], 0)[:, None]             # [new, P]
    for x in (s["codes"], s["scale"]):
        keep = rows.view(1, new, 1, 1, P, *[1] * (x.dim() - 5))
        y = torch.where(keep, x[:, from_page], x[:, to_page])
        # (what is not copied goes to the last page, which no sequence has)
        x[:, torch.where(copied, to_page, x.shape[1] - 1)] = y
    held = col < ((lens + P - 1) // P)[src][:, None]
    t = torch.where(held, table[src], -1)
    t = torch.where(copied[:, None] & (col == where[:, None]), target[:, None].int(), t)
    refs.index_add_(0, to_page, copied.int())
    next_table, next_refs = plain_resize(s, t, refs, s["slots"])
    return (t, s["lens"][src], refs, next_table, next_refs) + plain_read(s, next_table, s["last"], s["rest"], P)


def plain_compact(s):
    """The k-th held page at or past n goes to the k-th free page below n, n the number of held pages."""
    table, refs = plain_resize(s, s["table"], s["refs"], s["slots"])
    m = s["moves"]
    live = refs > 0
    n = live.sum()
    page = torch.arange(refs.shape[0], device=DEV)
    mover, hole = live & (page >= n), ~live & (page < n)
    src = torch.sort((~mover).int(), stable=True).indices[:m]
    dst = torch.sort((~hole).int(), stable=True).indices[:m]
    s["codes"][:, dst] = s["codes"][:, src]
    s["scale"][:, dst] = s["scale"][:, src]
    page_map = torch.where(live, page, -1)
    page_map[src] = dst
    new_refs = torch.where(live, refs, 0)
    new_refs[dst] = refs[src]
    new_refs[src] = 0
    new_table = torch.where(table < 0, -1, page_map[table.clamp(min=0).long()])
    return table, refs, new_table.int(), new_refs, page_map.int(), n.int().view(1), s["codes"]


PLAIN = dict(rope=plain_rope, write=plain_write, attend=plain_attend, fork=plain_fork, compact=plain_compact)


# ---------------------------------------------------------------------------- work and exact values

def row_bytes(case):
    hd = HEADS[case["heads"]][2]
    return {"i4": hd // 2 + hd // GROUP * 2, "f8": hd + 1, "bf16": hd * 2 + 1}[case.get("cache", "i4")]


def work(case):
    B = case["batch"]
    mean = lambda n: n * 3 / 4 if case.get("ragged") and n > 1 else n  # noqa: E731  of ragged sizes
    H, kvh, hd = HEADS[case["heads"]]
    eb = 2 if case.get("dtype") == "bf16" else 4
    if case["kind"] == "rope":
        n = B * case["tokens"] * (H + kvh) * hd * (2 if case["grad"] else 1)
        return dict(bytes=2 * n * eb, flops=3 * n * case["part"])
    row, P = row_bytes(case), case["page"]
    if case["kind"] == "write":
        n = mean(case["tokens"]) * B * 2 * kvh
        whole = B * case["tokens"] * 2 * kvh
        return dict(bytes=n * (hd * eb + row) + whole * hd * 2, flops=4 * n * hd)
    if case["kind"] == "attend":
        keys = mean(case["before"]) + mean(case["nodes"])
        q = B * case["nodes"] * H * hd
        return dict(bytes=B * keys * kvh * 2 * row + 2 * q * eb + B * case["nodes"] * 4,
                    flops=4 * B * mean(case["nodes"]) * H * hd * keys)
    if case["kind"] == "fork":
        new = B * case["beams"]
        # half a page's rows of each copied one; all new sequences' last rows read back
        copies = new - B if case["fresh"] else new * (1 - 1 / case["beams"]) ** case["beams"]
        tables = (new * mean(case["before"]) / P + case["batch"]) * 20
        n = case["layers"] * 2 * kvh
        return dict(bytes=n * (copies * P / 2 * 2 * row + new * P * hd * 2) + tables, flops=n * new * P / 2 * hd)
    pages = B * case["before"] / P
    live = pages * 7 / 8 * 3 / 4 * (1 - case["gone"])        # neighbours share some
    moved = live * (1 - live / pages)
    return dict(bytes=case["layers"] * moved * 2 * kvh * P * row * 2 + pages * 24, flops=pages)


def exact(case, seed):
    """In 64 bits. What only moves, and whole numbers, have none."""
    if case["kind"] in ("fork", "compact"):
        return None
    s = prepare(case, seed)
    H, kvh, hd = HEADS[case["heads"]]
    if case["kind"] == "rope":
        z, rot = s["scaling"], s["rot"]
        freq = []
        for i in range(rot // 2):
            f = z["theta"] ** (-2 * i / rot)
            if z["factor"] != 1.0:
                r = (z["original_len"] / (2 * math.pi / f) - z["low"]) / (z["high"] - z["low"])
                r = min(1.0, max(0.0, r))
                f = (1 - r) * f / z["factor"] + r * f
            freq.append(f)
        T = case["tokens"]
        offset = torch.arange(T, device=DEV).expand(case["batch"], T) if s["offset"] is None else s["offset"]
        ang = (s["start"].double()[:, None] + offset)[..., None] * torch.tensor(freq, dtype=torch.float64, device=DEV)
        phase = torch.polar(torch.full_like(ang, z["magnitude"]), ang)[:, :, None]

        def turn(x, phase):
            y = x.double()
            head, tail = y[..., :rot], y[..., rot:]
            if case["layout"] == "pairs":
                c = torch.view_as_complex(head.reshape(*head.shape[:-1], rot // 2, 2).contiguous()) * phase
                head = torch.view_as_real(c).flatten(-2)
            else:
                c = torch.complex(head[..., :rot // 2].contiguous(), head[..., rot // 2:].contiguous()) * phase
                head = torch.cat([c.real, c.imag], -1)
            return torch.cat([head, tail], -1)

        out = (turn(s["q"], phase), turn(s["k"], phase))
        return out + (turn(s["gq"], phase.conj()), turn(s["gk"], phase.conj())) if case["grad"] else out
    if case["kind"] == "write":
        count = s["count"].cpu().tolist()
        out = []
        for x in (s["k"].double(), s["v"].double()):
            g = x.view(*x.shape[:-1], hd // GROUP, GROUP)
            top = g.abs().amax(-1, keepdim=True)
            mant, exp = torch.frexp(top / torch.full_like(top, 7.0))   # 1/2 <= mant < 1
            step = (torch.round(mant * 16) / 16 * torch.exp2(exp.double())).clamp(min=2.0 ** -120)
            y = (torch.round(g / step) * step).flatten(-2)
            for b, n in enumerate(count):
                y[b, n:] = 0
            out.append(y[None])
        return tuple(out)
    P = case["page"]
    table, lens = s["table"].cpu().tolist(), s["lens"].cpu().tolist()
    nodes, T = s["nodes"].cpu().tolist(), case["nodes"]
    out = torch.zeros((case["batch"], T, H, hd), dtype=torch.float64, device=DEV)
    words = s["mask"].cpu().tolist()
    nibble = torch.tensor(list(range(8)) + list(range(-8, 0)), dtype=torch.float64, device=DEV)
    for b in range(case["batch"]):
        n, m = lens[b], nodes[b]
        page = torch.tensor([table[b][i // P] for i in range(n + m)], device=DEV)
        at = torch.tensor([i % P for i in range(n + m)], device=DEV)
        codes = s["codes"][0][page, :, :, at].long()
        kv = torch.empty(codes.shape[:-1] + (hd,), dtype=torch.float64, device=DEV)
        for d in range(hd):                    # where dimension d lies: 4 codes of each group in turn
            at4 = (d % GROUP // 4 * (hd // GROUP) + d // GROUP) * 4 + d % 4
            kv[..., d] = nibble[codes[..., at4 // 2] // (16 if at4 % 2 else 1) % 16]
        kv *= s["scale"][0][page, :, :, at].double().repeat_interleave(GROUP, -1)
        kv = kv.permute(1, 2, 0, 3)                                                          # [2, heads, n, size]
        sees = torch.ones((m, n + m), dtype=torch.bool)
        for t in range(m):
            for i in range(m):
                sees[t, n + i] = (words[b][t][i // 32] >> (i % 32)) & 1
        sees = sees.to(DEV)
        for h in range(kvh):
            q = s["q"][b, :m, h * (H // kvh):(h + 1) * (H // kvh)].double()
            x = torch.einsum("tgd,nd->tgn", q, kv[0, h]) * s["softmax_scale"]
            x = x.masked_fill(~sees[:, None], float("-inf"))
            out[b, :m, h * (H // kvh):(h + 1) * (H // kvh)] = torch.softmax(x, -1) @ kv[1, h]
    return out
