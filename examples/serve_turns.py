"""Routing and serving agent turns on one GPU: the router sends each request
to the instance whose KV$ blocks make it cheapest, and that instance prefills
only what its cache does not hold. One attention layer of random weights
stands in for the model.

    python examples/serve_turns.py [4]

With 4 the caches are held in 4 bits. Every turn's output is compared with the same prompt prefilled from nothing."""

from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_08565_gb300 as pkg  # noqa: E402

HQ, HK, D, BLOCK, VOCAB, WIDTH = 16, 2, 128, 32, 4096, 256
dev = torch.device("cuda")


class Layer:
    """Token embedding, a fused query/key/value projection, head norms, rotation."""

    def __init__(self, longest: int):
        g = torch.Generator(device=dev)
        g.manual_seed(0)
        rnd = lambda *s: torch.randn(*s, generator=g, device=dev, dtype=torch.bfloat16)  # noqa: E731
        self.embed, self.proj = rnd(VOCAB, WIDTH), rnd(WIDTH, (HQ + 2 * HK) * D) / WIDTH ** 0.5
        self.norms = dict(q_norm=1 + 0.1 * rnd(D), k_norm=1 + 0.1 * rnd(D))
        f = 10000.0 ** (-torch.arange(0, D, 2, device=dev, dtype=torch.float64) / D)
        a = torch.arange(longest, device=dev, dtype=torch.float64)[:, None] * f
        self.cos_sin = torch.cat([a.cos(), a.sin()], 1).float()

    def __call__(self, kv, cache, tokens):
        qkv = self.embed[tokens] @ self.proj
        q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([HQ * D, HK * D, HK * D], 1))
        q = kv.append(*cache, k, v, q=q, cos_sin=self.cos_sin, **self.norms)
        return kv.paged_attention(q, *cache)


class Instance:
    """A serving instance: a paged cache whose full blocks are found by their chain hash."""

    def __init__(self, pages: int, requests: int, tokens: int, bits: int = 16):
        kind = pkg.SMetricKV4 if bits == 4 else pkg.SMetricKV
        self.kv = kind(head_dim=D, num_q_heads=HQ, num_kv_heads=HK, page_size=BLOCK, num_pages=pages,
                       max_batch_requests=requests, max_batch_tokens=tokens)
        self.cache = (self.kv.new_cache() if bits == 4 else
                      [torch.empty(pages, BLOCK, HK, D, dtype=torch.bfloat16, device=dev) for _ in range(2)])
        self.free, self.held = list(range(pages)), {}

    def prefill(self, layer, prompts, hits, hashes):
        """prompts: token lists; hits: tokens that the route found here; hashes:
        their full blocks' chain hashes. The outputs of the tokens that were
        computed, prompt after prompt, and how many of each."""
        rows, new = [], []
        for prompt, hit, hs in zip(prompts, hits, hashes):
            hit = min(hit, (len(prompt) - 1) // BLOCK * BLOCK)  # one token at least is computed
            pages = [self.held[h] for h in hs[:hit // BLOCK]]
            pages += [self.free.pop() for _ in range(-(-len(prompt) // BLOCK) - len(pages))]
            rows.append(pages)
            new.append(len(prompt) - hit)
        table = torch.full((len(rows), max(map(len, rows))), -1, dtype=torch.int32)
        for r, pages in enumerate(rows):
            table[r, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
        offsets = torch.tensor([0] + new).cumsum(0).to(dev)
        lens = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device=dev)
        self.kv.plan(offsets, lens, table.to(dev), sum(new), max_new=max(new))
        tokens = torch.cat([torch.tensor(p[len(p) - n:]) for p, n in zip(prompts, new)]).to(dev)
        out = layer(self.kv, self.cache, tokens)
        self.kv.check()
        for pages, hs in zip(rows, hashes):
            for h, page in zip(hs, pages):
                self.held.setdefault(h, page)
        return out, new


def serve(sessions=12, turns=4, instances=3, seed=0, say=print, bits=16):
    """Returns (tokens prefilled, tokens of all prompts, largest difference from prefilling from nothing)."""
    g = torch.Generator().manual_seed(seed)
    text = lambda n: torch.randint(0, VOCAB, (n,), generator=g).tolist()  # noqa: E731
    system = text(500)
    prompts = [system + text(50 + 17 * i) for i in range(sessions)]
    most = sessions * (len(system) + 300 * (turns + 1) + 17 * sessions)
    layer = Layer(most)
    ix = pkg.SMetricIndex(instances, BLOCK, 1, capacity_slots=1 << 16, max_batch_requests=sessions, max_batch_tokens=most)
    nodes = [Instance(8192, sessions, most, bits) for _ in range(instances)]
    load = torch.zeros(instances, dtype=torch.int64, device=dev)
    done = total = 0
    worst = 0.0
    for turn in range(turns):
        offsets = torch.tensor([0] + [len(p) for p in prompts]).cumsum(0)
        tokens = torch.tensor([t for p in prompts for t in p], dtype=torch.int32, device=dev)
        offsets = offsets.to(dev)
        out = ix.route_batch_sequential(tokens, offsets, load, weights=(1, 8, 2))
        out["block_hashes"] = ix.block_hashes(tokens, offsets)[0]
        ix.commit_batch(offsets, out, load=load)
        ix.check()
        where, hit, hashes = (out[k].tolist() for k in ("instance", "local_hit", "block_hashes"))
        at = [0] + torch.tensor([len(p) // BLOCK for p in prompts]).cumsum(0).tolist()
        for i, node in enumerate(nodes):
            mine = [r for r in range(sessions) if where[r] == i]
            if not mine:
                continue
            ps, hs = [prompts[r] for r in mine], [hashes[at[r]:at[r + 1]] for r in mine]
            got, new = node.prefill(layer, ps, [hit[r] for r in mine], hs)
            whole, all_new = Instance(8192, sessions, most, bits).prefill(layer, ps, [0] * len(mine), [[]] * len(mine))
            a = b = 0
            for n, m in zip(new, all_new):
                worst = max(worst, (got[a:a + n].float() - whole[b + m - n:b + m].float()).abs().max().item())
                a, b = a + n, b + m
            done, total = done + sum(new), total + sum(all_new)
        say(f"turn {turn}: {done} of {total} prompt tokens prefilled so far, largest difference {worst:.2g}")
        prompts = [p + text(100 + 13 * r) for r, p in enumerate(prompts)]
    return done, total, worst


if __name__ == "__main__":
    serve(bits=int(sys.argv[1]) if len(sys.argv) > 1 else 16)
