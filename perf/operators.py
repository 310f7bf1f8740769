"""Tree speculation over a quantised paged cache, as measurable cases.

One decoding step of a model that drafts a tree of tokens is, for every layer, ``cdsl_kv_write``
(the tree's K/V into the cache) and ``cdsl_tree_attention`` (the tree's queries over prefix and
ancestors), then ``cdsl_tree_verify`` (which drafted path the target takes, and the next token) and
``cdsl_kv_commit`` (the taken path's K/V to their places). ``cdsl_kv_read`` gives cached rows back.

Kinds of cases:

* ``write``: a layer's new rows written into the cache and read back as values.
* ``attend``: the attention of one layer.
* ``verify``: the decision of one step.
* ``commit``: the taken paths' rows moved in every layer, and read back.

Head layouts, page sizes and vocabulary are those of the repository's workloads (32 query and 8
key/value heads of 128, 40 and 8, 16 and 4, 12 and 12 of 64; 32000 tokens).
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


def write_case(heads, batch, tokens, before, cache="f8", dtype="bf16", page=64, ragged=False):
    """`tokens` new rows after `before` cached ones (ragged: up to)."""
    return dict(kind="write", heads=heads, batch=batch, tokens=tokens, before=before, cache=cache, dtype=dtype,
                page=page, ragged=ragged)


def attend_case(heads, batch, nodes, before, tree="beams", cache="f8", dtype="bf16", page=64, ragged=False):
    """A tree of `nodes` (1: plain decoding) after `before` cached tokens (ragged: up to)."""
    return dict(kind="attend", heads=heads, batch=batch, nodes=nodes, before=before, tree=tree, cache=cache,
                dtype=dtype, page=page, ragged=ragged)


def verify_case(batch, nodes, vocab, tree="beams", dtype="f32", drafts=False, temperature=1.0):
    """drafts: the draft's own logits are given, and its tokens were sampled from them."""
    return dict(kind="verify", batch=batch, nodes=nodes, vocab=vocab, tree=tree, dtype=dtype, drafts=drafts,
                temperature=temperature)


def commit_case(heads, layers, batch, nodes, before, tree="beams", cache="f8", page=64):
    return dict(kind="commit", heads=heads, layers=layers, batch=batch, nodes=nodes, before=before, tree=tree,
                cache=cache, page=page)


def named(name, c):
    c["name"] = name
    return c


def listed():
    return [
        # one user's decoding step: the root and 4 beams of 4 drafted tokens into one layer's cache
        named("write-tree-b1", write_case("7b", 1, 17, 512)),
        # a layer's share of the prefill of four ragged prompts
        named("write-prefill-b4", write_case("13b", 4, 1031, 0, ragged=True)),
        # the smallest call: one token of one user after a short prompt
        named("attend-token-512", attend_case("7b", 1, 1, 512)),
        # one user's tree over a longer document
        named("attend-tree-4k", attend_case("7b", 1, 17, 4096)),
        # four users of the larger model, 8 beams of 6, cache in 16 bits
        named("attend-13b-tree-bf16", attend_case("13b", 4, 49, 1024, cache="bf16", ragged=True)),
        # a served batch decoding without drafts: the cache is nearly all there is to read
        named("attend-batch-tokens", attend_case("7b", 64, 1, 8192, page=128, ragged=True)),
        # a served batch with drafted trees over long documents
        named("attend-batch-long", attend_case("7b", 8, 25, 32768, tree="random", ragged=True)),
        # the small model in 32 bits, heads of 64 without sharing, small pages
        named("attend-small-f32", attend_case("small", 8, 17, 192, tree="random", dtype="f32", page=16, ragged=True)),
        # one user's decision over drafted beams
        named("verify-b1", verify_case(1, 17, 32000)),
        # a served batch whose drafts were sampled from the draft's distribution
        named("verify-drafts-b32", verify_case(32, 49, 32000, tree="random", dtype="bf16", drafts=True, temperature=0.8)),
        # the end of one user's step, all layers
        named("commit-7b-b1", commit_case("7b", 32, 1, 17, 512)),
        # the same of a served batch
        named("commit-13b-b16", commit_case("13b", 40, 16, 49, 1000, tree="random")),
    ]


def log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["write", "attend", "attend", "attend", "verify", "commit"])
    heads = rng.choice(["7b", "13b", "draft", "small"])
    tree = rng.choice(["beams", "random", "chain"])
    cache = rng.choice(["f8", "f8", "f8", "bf16"])
    page = rng.choice([16, 32, 64, 64, 128, 256])
    if kind == "write":
        batch, dtype = log_int(rng, 1, 64), rng.choice(["bf16", "bf16", "f32"])
        most = (2048 if dtype == "f32" else 4096) // batch
        return write_case(heads, batch, log_int(rng, 1, max(2, most)), log_int(rng, 1, 2000), cache=cache, dtype=dtype,
                          page=page, ragged=rng.random() < 0.5)
    if kind == "attend":
        f32 = rng.random() < 0.2
        batch, nodes = log_int(rng, 1, 64), rng.choice([1, log_int(rng, 2, 64)])
        # no more cached values, and no more products, than the largest listed cases have
        most = (4 if f32 else 32 if cache == "bf16" else 64) * 8192 // batch
        most = min(most, (24 if f32 else 8 * 20) * 32768 // (batch * nodes))
        return attend_case(heads, batch, nodes, log_int(rng, 16, max(17, min(65536, most))), tree=tree, cache=cache,
                           dtype="f32" if f32 else "bf16", page=page, ragged=rng.random() < 0.5)
    if kind == "verify":
        batch, drafts = log_int(rng, 1, 32), rng.random() < 0.5
        return verify_case(batch, log_int(rng, 2, max(3, min(64, 1536 // batch))),
                           rng.choice([512, 31999, 32000, log_int(rng, 500, 32768)]), tree=tree,
                           dtype=rng.choice(["bf16", "f32"]), drafts=drafts,
                           temperature=rng.choice([0.0, 0.6, 1.0, 1.0]))
    return commit_case(heads, log_int(rng, 1, 40), log_int(rng, 1, 16), log_int(rng, 2, 49), log_int(rng, 16, 1000),
                       tree=tree, cache=cache, page=page)


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


def most_taken(case):
    """Nodes of the longest path that a commit moves: all of a beam, or a quarter of another tree."""
    n = case["nodes"]
    return 1 + (-(-(n - 1) // max(1, int(math.sqrt(n - 1)))) if case["tree"] == "beams" else n // 4)


def lengths_of(case, rng):
    n = case["before"]
    if not case.get("ragged"):
        return [n] * case["batch"]
    return [rng.randint(n - n // 2, n) for _ in range(case["batch"])]


def quantise(x):
    """e4m3 codes (as bytes) and scale bytes of rows of values: a scale is the smallest power of two with which
    the row's largest value is at most 448; a row with a value that is not finite becomes zeros and byte 255."""
    x = x.float()
    bad = (x - x != 0).any(-1)
    x = torch.where(bad[..., None], 0.0, x)
    bits = x.abs().amax(-1).view(torch.int32)
    e = ((bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000)).clamp(-126, 127)
    e = torch.where(bits == 0, 0, e)
    codes = (x * ((127 - e) << 23).view(F32)[..., None]).to(F8).view(torch.uint8)
    return codes, torch.where(bad, 255, e + 127).to(torch.uint8)


def to_cache(x, cache):
    if cache == "f8":
        return quantise(x)
    bad = (x.float() - x.float() != 0).any(-1)
    return torch.where(bad[..., None], 0.0, x.float()).to(BF), torch.where(bad, 255, 127).to(torch.uint8)


def scale_values(b):
    return torch.where(b == 255, float("nan"), (b.int() << 23).view(F32))


def values(codes, b):
    """What cached codes stand for, in 32 bits."""
    x = codes.view(F8).float() if codes.dtype == torch.uint8 else codes.float()
    return x * scale_values(b)[..., None]


def rows_like_kv(shape, g, dtype=BF):
    """Rows of values whose sizes differ from token to token, as keys and values do."""
    size = torch.randn(shape[:-1], generator=g, device=DEV).mul_(0.5).exp_()
    return torch.randn(shape, generator=g, device=DEV).mul_(size[..., None]).to(dtype)


def cache_of(case, g, rng, slots, layers, fill):
    """Pages for `slots` tokens of each sequence in random order, and one page more that no sequence has."""
    _, kvh, hd = HEADS[case["heads"]]
    B, P = case["batch"], case["page"]
    per = (slots + P - 1) // P
    n = B * per + 1
    shape = (layers, n, 2, kvh, P)
    codes = torch.zeros(shape + (hd,), dtype=torch.uint8 if case["cache"] == "f8" else BF, device=DEV)
    scale = torch.full(shape, 127, dtype=torch.uint8, device=DEV)
    if fill:
        step = max(1, (1 << 28) // (2 * kvh * P * hd))
        for l in range(layers):
            for p in range(0, n, step):
                part = codes[l, p:p + step]
                codes[l, p:p + step], scale[l, p:p + step] = to_cache(rows_like_kv(part.shape, g), case["cache"])
    table = torch.randperm(n - 1, generator=g, device=DEV).view(B, per).int().contiguous()
    return codes, scale, table


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rng = random.Random(int(seed))
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    s = dict(case=case, stream=torch.cuda.current_stream().cuda_stream)
    B = case["batch"]
    if case["kind"] == "verify":
        return prepare_verify(case, s, g, rng, ints)
    H, kvh, hd = HEADS[case["heads"]]
    lens = lengths_of(case, rng)
    T = case.get("nodes") or case["tokens"]
    layers = case.get("layers", 1)
    codes, scale, table = cache_of(case, g, rng, max(lens) + T, layers, case["kind"] != "write")
    s.update(codes=codes, scale=scale, table=table, lens=ints(lens), max_len=max(lens))
    if own:   # the handle that a program keeps of its cache
        import paper_2412_10418_gb300 as cdsl
        s["cache"] = cdsl.KvCache(codes.view(F8) if case["cache"] == "f8" else codes, scale, table)
    if case["kind"] == "write":
        dt = BF if case["dtype"] == "bf16" else F32
        s["k"], s["v"] = (rows_like_kv((B, T, kvh, hd), g, dt) for _ in range(2))
        n = [rng.randint((T + 1) // 2, T) if case["ragged"] else T for _ in range(B)]
        s["count"] = ints(n)
        s["k_out"], s["v_out"] = (torch.empty((1, B, T, kvh, hd), dtype=BF, device=DEV) for _ in range(2))
    elif case["kind"] == "attend":
        dt = BF if case["dtype"] == "bf16" else F32
        trees = [parents_of(case["tree"], T, rng) for _ in range(B)]
        s["mask"] = ints([mask_words(p) for p in trees])
        n = [rng.randint((T + 1) // 2, T) if case["ragged"] else T for _ in range(B)]
        s["nodes"] = ints(n)
        s["q"] = torch.randn((B, T, H, hd), generator=g, device=DEV).to(dt)
        s["out"] = torch.empty_like(s["q"])
        s["softmax_scale"] = 1.0 / math.sqrt(hd)
        if own:
            s["ws"] = torch.zeros(cdsl.cdsl_tree_attention_workspace(s["cache"], T, H), dtype=torch.uint8, device=DEV)
    else:
        paths, D = [], most_taken(case)
        for _ in range(B):   # a path from the root towards a random node
            parents, i, path = parents_of(case["tree"], T, rng), rng.randrange(T), []
            while i:
                path.append(i)
                i = parents[i]
            paths.append(([0] + path[::-1])[:D])
        s["path"] = ints([p + [-1] * (T - len(p)) for p in paths])
        s["n_path"] = ints([len(p) for p in paths])
        s["new_lens"] = torch.empty_like(s["lens"])
        s["k_out"], s["v_out"] = (torch.empty((layers, B, D, kvh, hd), dtype=BF, device=DEV) for _ in range(2))
    return s


def prepare_verify(case, s, g, rng, ints):
    B, T, V = case["batch"], case["nodes"], case["vocab"]
    dt = BF if case["dtype"] == "bf16" else F32
    trees = [parents_of(case["tree"], T, rng) for _ in range(B)]
    logits = torch.randn((B, T, V), generator=g, device=DEV).mul_(3.0)
    near = torch.empty_like(logits).copy_(logits).add_(torch.randn((B, T, V), generator=g, device=DEV).mul_(0.7))
    parents = ints(trees)
    rows = parents.long()[..., None].expand(B, T, V)
    if case["drafts"]:   # sampled from the parent's row of the draft
        t = case["temperature"] or 1.0
        p = torch.softmax(near / t, -1).gather(1, rows).view(B * T, V)
        tokens = torch.multinomial(p, 1, generator=g).view(B, T)
    else:                # the k-th child has the draft's k-th choice
        kth = [[sum(t[j] == t[i] for j in range(1, i)) for i in range(T)] for t in trees]
        best = near.topk(min(T, V), dim=-1).indices
        tokens = best.gather(1, rows[..., :best.shape[-1]]).gather(2, ints(kth).long()[..., None])[..., 0]
    s.update(logits=logits.to(dt), draft=near.to(dt) if case["drafts"] else None, tokens=tokens.int().contiguous(),
             parents=parents, u=torch.rand((B, T), generator=g, device=DEV),
             u_last=torch.rand(B, generator=g, device=DEV),
             path=torch.empty((B, T), dtype=torch.int32, device=DEV),
             n_path=torch.empty(B, dtype=torch.int32, device=DEV),
             emitted=torch.empty((B, T), dtype=torch.int32, device=DEV))
    return s


# ---------------------------------------------------------------------------- a pass

def run(s):
    if own:
        return OWN[s["case"]["kind"]](s)
    return PLAIN[s["case"]["kind"]](s)


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


def own_verify(s):
    import paper_2412_10418_gb300 as cdsl
    cdsl.cdsl_tree_verify(s["logits"], s["tokens"], s["parents"], s["u"], s["u_last"], s["path"], s["n_path"],
                          s["emitted"], draft_logits=s["draft"], temperature=s["case"]["temperature"],
                          stream=s["stream"])
    return s["path"], s["n_path"], s["emitted"]


def own_commit(s):
    import paper_2412_10418_gb300 as cdsl
    cdsl.cdsl_kv_commit(s["cache"], s["lens"], s["path"], s["n_path"], s["new_lens"], stream=s["stream"])
    cdsl.cdsl_kv_read(s["cache"], 0, s["lens"], s["k_out"], s["v_out"], s["n_path"], stream=s["stream"])
    return s["k_out"], s["v_out"], s["new_lens"]


OWN = dict(write=own_write, attend=own_attend, verify=own_verify, commit=own_commit)


def places(s, slots, valid):
    """Page and place in it of each slot [B, n]; what is not valid goes to the page that no sequence has."""
    P = s["case"]["page"]
    column = (slots // P).clamp(0, s["table"].shape[1] - 1).long()
    page = s["table"].gather(1, column).long()
    return torch.where(valid, page, s["codes"].shape[1] - 1), (slots % P).long()


def plain_write(s):
    T = s["k"].shape[1]
    i = torch.arange(T, device=DEV)
    page, at = places(s, s["lens"][:, None] + i, i < s["count"][:, None])
    for kv, x in ((0, s["k"]), (1, s["v"])):
        codes, scale = to_cache(x, s["case"]["cache"])
        s["codes"][0, :, kv][page, :, at] = codes
        s["scale"][0, :, kv][page, :, at] = scale
    return plain_read(s, s["count"], T)


def plain_read(s, count, n):
    """The rows of every layer from slot `lens` on."""
    i = torch.arange(n, device=DEV)
    valid = i < count[:, None]
    page, at = places(s, s["lens"][:, None] + i, valid)
    out = []
    for kv in (0, 1):
        # the layers' index is put with the others: [B, n, heads, layers, size]
        codes = s["codes"][:, :, kv].permute(1, 2, 3, 0, 4)[page, :, at]
        scale = s["scale"][:, :, kv].permute(1, 2, 3, 0)[page, :, at]
        x = values(codes, scale)
        out.append(torch.where(valid[:, :, None, None, None], x, 0.0).to(BF).permute(3, 0, 1, 2, 4).contiguous())
    return tuple(out)


def plain_commit(s):
    T = s["path"].shape[1]
    i = torch.arange(T, device=DEV)
    valid = i < s["n_path"][:, None]
    page, at = places(s, s["lens"][:, None] + s["path"].clamp(min=0), valid)
    to_page, to_at = places(s, s["lens"][:, None] + i, valid)
    codes, scale = s["codes"].permute(1, 4, 0, 2, 3, 5), s["scale"].permute(1, 4, 0, 2, 3)   # views: page, place first
    moved, moved_scale = codes[page, at], scale[page, at]
    codes[to_page, to_at] = moved
    scale[to_page, to_at] = moved_scale
    return plain_read(s, s["n_path"], s["k_out"].shape[2]) + (s["lens"] + s["n_path"],)


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
    k, v = (values(s["codes"][0][pages, kv], s["scale"][0][pages, kv]).transpose(1, 2).reshape(B, kvh, -1, hd)
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


TWO31, TWO24 = float(1 << 31), 1 << 24


def share(u, total):
    """floor(floor(u 2^24) total / 2^24) of whole numbers, total below 2^56."""
    k = (u * TWO24).long()
    return k * (total >> 24) + ((k * (total & (TWO24 - 1))) >> 24)


def weights(logits, inv_t):
    x = logits.float()
    return ((x - x.amax(-1, keepdim=True)) * inv_t).exp()


def plain_verify(s):
    """The walk over all sequences at once, node after node: a parent comes before its children."""
    case = s["case"]
    B, T, V = s["logits"].shape
    path = torch.full((B, T), -1, dtype=torch.int32, device=DEV)
    emitted = torch.full((B, T), -1, dtype=torch.int32, device=DEV)
    path[:, 0] = 0
    n = torch.ones(B, dtype=torch.int32, device=DEV)
    cur = torch.zeros(B, dtype=torch.int32, device=DEV)
    every = torch.arange(B, device=DEV)
    greedy = case["temperature"] == 0
    drafts = s["draft"] is not None and not greedy
    inv_t = 0.0 if greedy else float(torch.tensor(1.0) / torch.tensor(case["temperature"]))
    units = lambda w: (w * TWO31).long()  # noqa: E731

    def start(node):
        if greedy:
            return [s["logits"][every, node].float()]
        w = weights(s["logits"][every, node], inv_t)
        W = units(w)
        Z = W.sum(-1)
        r = [W, Z]
        if drafts:
            wq = weights(s["draft"][every, node], inv_t)
            r += [w * (1.0 / (Z.float() / TWO31))[:, None], wq * (1.0 / (units(wq).sum(-1).float() / TWO31))[:, None]]
        return r

    state = start(cur.long())
    for i in range(1, T):
        child = s["parents"][:, i] == cur
        x = s["tokens"][:, i].long()[:, None]
        if greedy:
            took = child & (state[0].argmax(-1) == x[:, 0])
            rejected = state
        elif drafts:
            W, Z, p, q = state
            took = child & (s["u"][:, i] * q.gather(1, x)[:, 0] < p.gather(1, x)[:, 0])
            r = (p - q).clamp(min=0.0)
            R = units(r)
            ZR = R.sum(-1)
            none = (ZR == 0)
            inv = 1.0 / (ZR.float() / TWO31)
            rejected = [torch.where(none[:, None], W, R), torch.where(none, Z, ZR),
                        torch.where(none[:, None], p, r * inv[:, None]), q]
        else:
            W, Z = state
            mine = W.gather(1, x)[:, 0]
            took = child & (share(s["u"][:, i], Z) < mine)
            rejected = [W.scatter(1, x, 0), Z - mine]
        path[every, torch.where(took, n, 0).long()] = torch.where(took, i, 0).int()
        emitted[every, (n - 1).long()] = torch.where(took, x[:, 0].int(), emitted[every, (n - 1).long()])
        n = n + took.int()
        cur = torch.where(took, i, cur)
        fresh = start(cur.long())
        wide = lambda c, like: c.view((B,) + (1,) * (like.dim() - 1))  # noqa: E731
        state = [torch.where(wide(took, a), a, torch.where(wide(child, a), b, c))
                 for a, b, c in zip(fresh, rejected, state)]
    if greedy:
        last = state[0].argmax(-1)
    else:
        last = (state[0].cumsum(-1) > share(s["u_last"], state[1])[:, None]).int().argmax(-1)
    emitted[every, (n - 1).long()] = last.int()
    return path, n, emitted


PLAIN = dict(write=plain_write, attend=plain_attend, verify=plain_verify, commit=plain_commit)


# ---------------------------------------------------------------------------- work and exact values

def work(case):
    B = case["batch"]
    mean = lambda n: n * 3 / 4 if case.get("ragged") and n > 1 else n  # noqa: E731  of ragged sizes
    if case["kind"] == "verify":
        # the rows of the nodes on the way taken: the root and about two more
        rows = B * min(case["nodes"], 3)
        eb = 2 if case["dtype"] == "bf16" else 4
        n = rows * case["vocab"] * (2 if case["drafts"] else 1)
        return dict(bytes=n * eb + B * case["nodes"] * 20, flops=4 * n)
    H, kvh, hd = HEADS[case["heads"]]
    row = hd * (1 if case["cache"] == "f8" else 2) + 1
    if case["kind"] == "write":
        n = mean(case["tokens"]) * B * 2 * kvh
        whole = B * case["tokens"] * 2 * kvh
        return dict(bytes=n * (hd * (2 if case["dtype"] == "bf16" else 4) + row) + whole * hd * 2, flops=4 * n * hd)
    if case["kind"] == "commit":
        most = most_taken(case)   # about half of them are taken; the others' values are zeros
        n = case["layers"] * B * 2 * kvh
        return dict(bytes=n * (most / 2 * 2 * row + most * hd * 2), flops=n * most / 2 * hd)
    keys = mean(case["before"]) + mean(case["nodes"])
    eb = 2 if case["dtype"] == "bf16" else 4
    q = B * case["nodes"] * H * hd
    return dict(bytes=B * keys * kvh * 2 * row + 2 * q * eb + B * case["nodes"] * 4,
                flops=4 * B * mean(case["nodes"]) * H * hd * keys)


def exact(case, seed):
    """In 64 bits, sequence by sequence; the decisions are whole numbers and have none."""
    if case["kind"] == "verify":
        return None
    s = prepare(case, seed)
    H, kvh, hd = HEADS[case["heads"]]
    P = case["page"]
    table, lens = s["table"].cpu().tolist(), s["lens"].cpu().tolist()

    def stored(layer, b, slots):
        """[2, heads, n, size] of the slots as cached."""
        page = torch.tensor([table[b][i // P] for i in slots], device=DEV)
        at = torch.tensor([i % P for i in slots], device=DEV)
        codes = s["codes"][layer][page, :, :, at]
        b8 = s["scale"][layer][page, :, :, at].double()
        x = codes.view(F8).double() if codes.dtype == torch.uint8 else codes.double()
        return (x * torch.exp2(torch.where(b8 == 255, float("nan"), b8 - 127))[..., None]).permute(1, 2, 0, 3)

    if case["kind"] == "write":
        count = s["count"].cpu().tolist()
        out = []
        for x in (s["k"].double(), s["v"].double()):
            y = x
            if case["cache"] == "f8":
                top = x.abs().amax(-1, keepdim=True)
                e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 448)).clamp(-126, 127)
                e = e + (top > 448 * torch.exp2(e)).double() - (top <= 224 * torch.exp2(e)).double()
                z = x * torch.exp2(-e)
                step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
                y = torch.round(z / step) * step * torch.exp2(e)
            else:
                y = x.to(BF).double()
            for b, n in enumerate(count):
                y[b, n:] = 0
            out.append(y[None])
        return tuple(out)
    if case["kind"] == "commit":
        n_path, path = s["n_path"].cpu().tolist(), s["path"].cpu().tolist()
        k = torch.zeros(s["k_out"].shape, dtype=torch.float64, device=DEV)
        v = torch.zeros_like(k)
        for l in range(case["layers"]):
            for b in range(case["batch"]):
                x = stored(l, b, [lens[b] + i for i in path[b][:n_path[b]]])
                k[l, b, :n_path[b]], v[l, b, :n_path[b]] = x[0].transpose(0, 1), x[1].transpose(0, 1)
        return k, v, None
    nodes, T = s["nodes"].cpu().tolist(), case["nodes"]
    out = torch.zeros((case["batch"], T, H, hd), dtype=torch.float64, device=DEV)
    words = s["mask"].cpu().tolist()
    for b in range(case["batch"]):
        n, m = lens[b], nodes[b]
        kv = stored(0, b, range(n + m))
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
