"""Several answers to one prompt over the 8-bit paged cache: shared pages, draft-and-verify steps, all layers run by this program.

The prompt is processed once; the answers fork its cache, so that they share its pages until each writes to its last one. A step of all answers: the extra heads' candidates fill a
tree, one pass of the base model verifies every node (rows of the pass stay in 16 bits and see the cached tokens and their own ancestors), the accepted path of each answer, of its own length, goes
into the cache. Nothing of a step waits for the host except the tokens that are printed.

    python examples/forked_answers.py [--answers 4] [--steps 8] [--temperature 0.8]

Seeded synthetic weights of a small shape; projections by spec_op_linear, norms and the feed-forward product by plain torch.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2503_14153_b200 import SpecCache, build_tree, spec_op_linear, spec_rotary, spec_rotary_table, upload_weights  # noqa: E402
from synthetic import draw_prompt, draw_weights, get_config  # noqa: E402


def small_config():
    return get_config("c0", name="forked_answers", n_layers=2, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ffn=704, dtype="bf16", seed=5, n_medusa=3, topk=(4, 2, 2), tree_nodes=16)


class Model:
    """The base model's layers over a SpecCache."""

    def __init__(self, cfg, weights, cache, span=4096):
        self.cfg, self.w, self.cache = cfg, weights, cache
        self.table = spec_rotary_table(span, cfg.head_dim, cfg.rope_base)

    def norm(self, x, gain):
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + self.cfg.rms_eps) * gain).bfloat16()

    def linear(self, x, w):
        """y = x w^T; the projection takes rows in sixteens."""
        rows = -x.shape[0] % 16
        return spec_op_linear(torch.cat([x, x.new_zeros(rows, x.shape[1])]) if rows else x, w)[: x.shape[0]]

    def forward(self, tokens, positions, batch, seqs=None, mask=None):
        """Hidden states after the final norm [rows, d_model], and every layer's K and V rows [layers, rows, kv heads, D], not yet cached."""
        cfg, w = self.cfg, self.w
        H, kv, D = cfg.n_heads, cfg.n_kv_heads, cfg.head_dim
        x = w["embed"][tokens.long()].float()
        ks, vs = [], []
        for l in range(cfg.n_layers):
            p = f"layers.{l}."
            qkv = self.linear(self.norm(x, w[p + "attn_norm"]), w[p + "wqkv"]).view(-1, H + 2 * kv, D)
            q, k, v = spec_rotary(*qkv.split((H, kv, kv), dim=1), positions, self.table, dtype=torch.bfloat16)
            o = self.cache.attention(l, q, k, v, batch=batch, seqs=seqs, mask=mask)
            x = x + self.linear(o.flatten(1), w[p + "wo"])
            u = self.norm(x, w[p + "ffn_norm"])
            x = x + self.linear((torch.nn.functional.silu(self.linear(u, w[p + "w_gate"])) * self.linear(u, w[p + "w_up"])).bfloat16(), w[p + "w_down"])
            ks.append(k)
            vs.append(v)
        return self.norm(x, w["final_norm"]), torch.stack(ks), torch.stack(vs)

    def logits(self, h):
        return self.linear(h, self.w["lm_head"])

    def candidates(self, h):
        """The extra heads' largest tokens [rows, heads, kmax] from the hidden state h."""
        out = []
        for i in range(self.cfg.n_medusa):
            r = h.float() + torch.nn.functional.silu(self.linear(h, self.w[f"medusa.{i}.w"]) + self.w[f"medusa.{i}.b"].float())
            out.append(self.logits(r.bfloat16()).topk(self.cfg.kmax, dim=-1)[1])
        return torch.stack(out, dim=1)


def answer(model, prompt, answers, steps, temperature, seed=0):
    """Tokens of every answer (a list of lists). The answers' first tokens are drawn at `temperature`, the rest is greedy."""
    cfg, cache = model.cfg, model.cache
    tree = build_tree(cfg.topk, cfg.tree_nodes)
    dev = cache.device
    ints = lambda v: torch.as_tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    depth, parent, rank = (torch.as_tensor(tree[k], device=dev).long() for k in ("depth", "parent", "rank"))
    T, K = len(depth), cfg.n_medusa
    sees = torch.eye(T, dtype=torch.int64, device=dev)
    for v in range(1, T):
        sees[v] |= sees[parent[v]]
    mask = (sees << torch.arange(T, device=dev)).sum(1).to(torch.int32).view(T, 1).repeat(answers, 1)     # (16 nodes: one word a row)

    # the prompt, as sequence 0
    n = len(prompt)
    one = ints([n])
    h, k, v = model.forward(ints(prompt), torch.arange(n, dtype=torch.int32, device=dev), 1, seqs=ints([0]))
    cache.store(k, v, cache.reserve(one, seqs=ints([0])), seqs=ints([0]))
    last = h[-1:].repeat(answers, 1)
    g = torch.Generator(device=dev).manual_seed(seed)
    root = torch.multinomial(torch.softmax(model.logits(last) / max(temperature, 1e-4), dim=-1), 1, generator=g).view(-1)

    # the answers share its pages
    seqs = torch.arange(1, answers + 1, dtype=torch.int32, device=dev)
    cache.fork(torch.zeros_like(seqs), seqs)
    emitted = []
    for _ in range(steps):
        cand = torch.cat([root.view(-1, 1, 1).expand(-1, 1, cfg.kmax), model.candidates(last)], dim=1)   # [answers, 1 + heads, kmax]
        tokens = cand[:, depth, rank]                                                                     # [answers, T]
        positions = cache.lens[seqs.long()].view(-1, 1) + depth.to(torch.int32)
        h, k, v = model.forward(tokens.reshape(-1), positions.reshape(-1).contiguous(), answers, seqs=seqs, mask=mask)
        best = model.logits(h).argmax(-1).view(answers, T)
        ok = torch.zeros((answers, T), dtype=torch.bool, device=dev)
        ok[:, 0] = True
        for node in range(1, T):
            ok[:, node] = ok[:, parent[node]] & (tokens[:, node] == best[:, parent[node]])
        end = torch.where(ok, depth * T - torch.arange(T, device=dev), torch.full_like(depth, -T * T)).argmax(-1)   # the deepest accepted node, the lowest of them
        path = torch.zeros((answers, K + 1), dtype=torch.int64, device=dev)
        at = end
        for j in range(K, -1, -1):
            path[:, j] = torch.where(depth[at] >= j, at, path[:, j])
            at = torch.where(depth[at] >= j, parent[at].clamp(min=0), at)
        counts = (depth[end] + 1).to(torch.int32)
        cache.store(k, v, cache.reserve(counts, seqs=seqs), seqs=seqs, path=path.to(torch.int32))
        emitted.append((tokens.gather(1, path), counts))
        root = best.gather(1, end.view(-1, 1)).view(-1)
        last = h.view(answers, T, -1)[torch.arange(answers, device=dev), end]
    cache.check()
    return [[t for toks, c in emitted for t in toks[b, : int(c[b])].tolist()] for b in range(answers)]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--answers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--temperature", type=float, default=0.8)
    ap.add_argument("--format", default="int8", choices=("int8", "e4m3"))
    a = ap.parse_args(argv)
    cfg = small_config()
    prompt = draw_prompt(cfg, 60).tolist()
    room = -(-(len(prompt) + a.steps * (cfg.n_medusa + 1)) // 16)
    cache = SpecCache(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, 4 + (a.answers + 1) * room, a.answers + 1, room, fmt=a.format)
    model = Model(cfg, upload_weights(cfg, draw_weights(cfg)), cache)
    got = answer(model, prompt, a.answers, a.steps, a.temperature)
    held = int((cache.refs > 0).sum())
    print(f"{a.answers} answers, {sum(len(x) for x in got)} tokens in {a.steps} steps; {held} pages held for {int(cache.lens.sum())} cached tokens ({int(cache.refs.sum())} without sharing)")
    for i, x in enumerate(got):
        print(f"  {i}: {x}")
    cache.truncate()
    return got, cache


if __name__ == "__main__":
    main()
