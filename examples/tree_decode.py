"""Tree-speculative decoding with a draft model, over quantised paged caches.

A decoding step of `TreeDecoder`, for every sequence of the batch:

1. M_q drafts a tree of tokens, level by level: the children of a node are M_q's most likely tokens after it.
2. M_p runs once over the tree: per layer `cdsl_kv_write` and `cdsl_tree_attention`.
3. `cdsl_tree_verify` walks the tree by M_p's distributions and draws the token after the path.
4. `cdsl_kv_commit` moves the path's K/V in both caches to their places.

Both models are the synthetic decoders of `synth` with PyTorch's products for their projections; nothing of a step
is read on the host, and a step is one CUDA graph. The prompt goes through the same calls, as chains of up to 128
tokens.

    python examples/tree_decode.py --workload small-bf16 --new 64
"""
import argparse
import os
import sys
import time

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2412_10418_gb300 as cdsl  # noqa: E402
import synth  # noqa: E402


def rope(x, pos, theta):
    """x [B, T, heads, hd] turned by the angles of positions pos [B, T]; dimension i goes with i + hd / 2."""
    half = x.shape[-1] // 2
    freq = theta ** (-torch.arange(half, device=x.device, dtype=torch.float32) / half)
    ang = pos[..., None, None].float() * freq
    cos, sin = ang.cos(), ang.sin()
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(x.dtype)


class Model:
    """A decoder whose K/V live in a paged cache of its own, `slots` tokens for each of `batch` sequences."""

    def __init__(self, shape, weights, batch, slots, page_size=64, cache_dtype=None):
        self.shape, self.w = shape, weights
        dev = weights["embed"].device
        pages = -(-slots // page_size)
        table = torch.arange(batch * pages, dtype=torch.int32, device=dev).view(batch, pages)
        self.cache = cdsl.KvCache.empty(shape.n_layers, batch * pages, shape.n_kv_heads, page_size, shape.head_dim, table,
                                        cache_dtype)
        self.max_len = pages * page_size - cdsl.TREE_MAX_NODES
        self.work = torch.empty(cdsl.cdsl_tree_attention_workspace(self.cache, cdsl.TREE_MAX_NODES, shape.n_heads),
                                dtype=torch.uint8, device=dev)

    def forward(self, tokens, lens, depth, mask, nodes=None, head=True, status=None):
        """Nodes tokens [B, T] at positions lens + depth: their K/V into slots lens .. lens + T - 1, and the logits of
        the tokens after them [B, T, vocab]."""
        s, w = self.shape, self.w
        B, T = tokens.shape
        pos = lens[:, None] + depth
        h = F.embedding(tokens.clamp(0, s.vocab - 1), w["embed"])
        for l in range(s.n_layers):
            a = self.norm(h, w[f"l{l}.attn_norm"])
            q, k, v = (F.linear(a, w[f"l{l}.w{x}"]).view(B, T, -1, s.head_dim) for x in "qkv")
            q, k = rope(q, pos, s.rope_theta), rope(k, pos, s.rope_theta)
            cdsl.cdsl_kv_write(self.cache, l, k, v, lens, count=nodes, status=status)
            out = torch.empty_like(q)
            cdsl.cdsl_tree_attention(self.cache, l, q, lens, mask, out, self.work, scale=s.head_dim ** -0.5,
                                     max_len=self.max_len, nodes=nodes, status=status)
            h = h + F.linear(out.flatten(2), w[f"l{l}.wo"])
            a = self.norm(h, w[f"l{l}.ffn_norm"])
            h = h + F.linear(F.silu(F.linear(a, w[f"l{l}.w_gate"])) * F.linear(a, w[f"l{l}.w_up"]), w[f"l{l}.w_down"])
        return F.linear(self.norm(h, w["final_norm"]), w["lm_head"]) if head else None

    def norm(self, x, g):
        y = x.float()
        return (y * (y.square().mean(-1, keepdim=True) + self.shape.norm_eps).rsqrt() * g.float()).to(x.dtype)


class TreeDecoder:
    """Decodes `batch` sequences with trees whose nodes at depth d have widths[d] children each; () drafts nothing."""

    def __init__(self, target, draft, widths, temperature=1.0, seed=0):
        self.target, self.draft, self.temperature = target, draft, temperature
        dev = target.cache.device
        B = target.cache.batch
        levels, parents = [[0]], [0]           # nodes by depth: parents before children, siblings by M_q's choice
        for n in widths:
            levels.append([])
            for p in levels[-2]:
                for _ in range(n):
                    levels[-1].append(len(parents))
                    parents.append(p)
        self.T, self.levels, self.widths = len(parents), levels, widths
        mask, depth = cdsl.cdsl_tree_mask(parents)
        self.mask = mask.to(dev).expand(B, -1, -1).contiguous()
        self.depth = depth.to(dev)
        self.parents = torch.tensor(parents, dtype=torch.int32, device=dev).expand(B, -1).contiguous()
        self.known = [torch.full((B,), l[-1] + 1, dtype=torch.int32, device=dev) for l in levels]
        self.tokens = torch.zeros((B, self.T), dtype=torch.int32, device=dev)
        self.path, self.emitted = torch.empty_like(self.tokens), torch.empty_like(self.tokens)
        self.n_path = torch.empty(B, dtype=torch.int32, device=dev)
        self.lens = torch.zeros_like(self.n_path)
        self.new_lens = torch.zeros_like(self.n_path)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.u, self.u_last = torch.empty((B, self.T), device=dev), torch.empty(B, device=dev)
        self.rng = torch.Generator(device=dev).manual_seed(seed)
        self.graph, self.steps = None, 0

    def prefill(self, prompts, lengths):
        """prompts [B, n] int32 of lengths [B] tokens (1 at least): all but the last token into both caches; the last is
        the first step's node 0."""
        B, n = prompts.shape
        self.lens.zero_()
        for first in range(0, n - 1, cdsl.TREE_MAX_NODES):
            part = prompts[:, first:min(n - 1, first + cdsl.TREE_MAX_NODES)].contiguous()
            T = part.shape[1]
            mask, depth = cdsl.cdsl_tree_mask([max(0, i - 1) for i in range(T)])
            mask, depth = mask.to(part.device).expand(B, -1, -1).contiguous(), depth.to(part.device)
            nodes = (lengths - 1 - first).clamp(0, T).int()
            for m in (self.target, self.draft):
                m.forward(part, self.lens, depth, mask, nodes, head=False, status=self.status)
            self.lens += nodes
        self.tokens[:, 0] = prompts.gather(1, (lengths - 1).long()[:, None])[:, 0]

    def step(self):
        """One step: `emitted` [B, T] (filled up with -1) and `n_path` [B], the number of tokens in it. The third step is
        captured, and it and the later ones are replayed."""
        self.steps += 1
        for u in (self.u, self.u_last):
            u.uniform_(generator=self.rng)
        if self.steps == 3:
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self.run()
        if self.graph is None:
            self.run()
        else:
            self.graph.replay()
        return self.emitted, self.n_path

    def run(self):
        for l, nodes in enumerate(self.levels):      # (the last level's K/V too: its nodes may be taken)
            last = l + 1 == len(self.levels)
            logits = self.draft.forward(self.tokens, self.lens, self.depth, self.mask, self.known[l], not last, self.status)
            if not last:
                best = logits[:, nodes[0]:nodes[-1] + 1].topk(self.widths[l], dim=-1).indices
                self.tokens[:, self.levels[l + 1][0]:self.levels[l + 1][-1] + 1] = best.flatten(1).int()
        logits = self.target.forward(self.tokens, self.lens, self.depth, self.mask, status=self.status)
        cdsl.cdsl_tree_verify(logits, self.tokens, self.parents, self.u, self.u_last, self.path, self.n_path,
                              self.emitted, temperature=self.temperature, status=self.status)
        for m in (self.target, self.draft):
            cdsl.cdsl_kv_commit(m.cache, self.lens, self.path, self.n_path, self.new_lens, self.status)
        self.lens.copy_(self.new_lens)
        self.tokens[:, 0] = self.emitted.gather(1, (self.n_path - 1).clamp(min=0).long()[:, None])[:, 0]


def build(workload, widths, slots, self_draft=False, cache_dtype=None, **kw):
    """A decoder of a `synth` workload's models; self_draft: M_p drafts for itself."""
    target = synth.model_weights(workload, "target", device="cuda")
    model = Model(workload.target, target, workload.batch, slots, cache_dtype=cache_dtype)
    if self_draft:
        draft = Model(workload.target, target, workload.batch, slots, cache_dtype=cache_dtype)
    else:
        draft = Model(workload.draft, synth.model_weights(workload, "draft", device="cuda"), workload.batch, slots,
                      cache_dtype=cache_dtype)
    return TreeDecoder(model, draft, widths, **kw)


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--workload", default="small-bf16", choices=sorted(synth.WORKLOADS))
    p.add_argument("--widths", default="3,2,1,1", help="children of the nodes at each depth")
    p.add_argument("--temperature", type=float, default=0.0)
    p.add_argument("--new", type=int, default=64, help="tokens to decode per sequence")
    p.add_argument("--self-draft", action="store_true", help="the target drafts for itself")
    a = p.parse_args()
    wl = synth.WORKLOADS[a.workload]
    widths = tuple(int(x) for x in a.widths.split(",") if x)
    d = build(wl, widths, wl.prompt_len + a.new + 2 * cdsl.TREE_MAX_NODES, a.self_draft, temperature=a.temperature)
    prompts = torch.from_numpy(synth.prompts(wl)).cuda()
    d.prefill(prompts, torch.full((wl.batch,), wl.prompt_len, dtype=torch.int32, device="cuda"))
    out = [[] for _ in range(wl.batch)]
    steps, times = 0, []
    while min(len(o) for o in out) < a.new:
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        emitted, n = d.step()
        steps += 1
        for o, e, m in zip(out, emitted.tolist(), n.tolist()):
            o += e[:m]
        times.append(time.perf_counter() - t0)
    if int(d.status):
        raise cdsl.CdslError(int(d.status), "a step")
    print(f"{wl.name}: {d.T}-node trees, {steps} steps, {sum(map(len, out)) / steps / wl.batch:.2f} tokens a step and "
          f"sequence, {sorted(times)[steps // 2] * 1e3:.2f} ms a step (the median)")


if __name__ == "__main__":
    main()
