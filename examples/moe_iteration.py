"""Serving iterations of a small mixture-of-experts model whose experts live on
the host, with the expert-map search deciding what the expert cache holds.

    python examples/moe_iteration.py

One iteration of a batch of requests, as the library's operators make it up:

  1. embed_pool            each prompt's mean embedding, the semantic query
  2. match_semantic_select the most similar stored iteration of each request and
                           the experts it foretells for every layer
  3. embed_lookup          the last token of every request
  4. per layer:
       moe_route           gate probabilities, written as this layer's row of
                           the batch's expert maps, and the chosen experts
       TrajPass.step       stored iterations by the layers seen so far, and
       select_prefetch     the experts they foretell for the layers ahead
       ExpertCache.load    chosen experts that no prefetch brought in
       moe_experts         the chosen experts' products, added to the stream
  5. Store.insert          the finished iterations enter the store

Model.tune moves the embeddings of some tokens with embed_grad.  Weights are random and attention is left out: the layers are residual MoE blocks.
"""
from __future__ import annotations

import dataclasses
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2502_05370_amd as fm  # noqa: E402


@dataclasses.dataclass
class Config:
    V: int = 1000         # vocabulary
    d: int = 256          # hidden size
    f: int = 128          # expert width
    L: int = 6            # layers
    E: int = 16           # experts per layer
    K: int = 2            # experts per token
    slots: int = 10       # experts of a layer that fit the GPU
    distance: int = 2     # layers between a search and the prefetch it guides
    store: int = 256      # iterations the store holds
    tau: float = 0.9      # share of probability that a prefetch set covers


class Layer:
    """One MoE layer: its gate and expert cache on the GPU, its experts on the host."""

    def __init__(self, c: Config, g: torch.Generator):
        bf = torch.bfloat16
        self.gate = (torch.randn(c.E, c.d, generator=g) * 2 / c.d ** 0.5).to(bf).cuda()
        self.host = [[(torch.randn(*s, generator=g) / s[1] ** 0.5).to(bf) for s in ((c.f, c.d), (c.f, c.d), (c.d, c.f))]
                     for _ in range(c.E)]
        self.cache = fm.ExpertCache(c.slots, c.E, c.d, c.f, "bf16")
        self.held = {}    # expert -> slot, in the order of their last use
        self.loads = 0

    def bring_in(self, experts, keep=()) -> int:
        """Load the experts that the cache lacks, over the least recently used others.  Returns how many were
        loaded; experts that do not fit beside the ones to keep are left out."""
        loaded = 0
        for e in experts:
            if e in self.held:
                self.held[e] = self.held.pop(e)
                continue
            if len(self.held) < self.cache.slots:
                slot = len(self.held)
            else:
                victim = next((v for v in self.held if v not in keep and v not in experts), None)
                if victim is None:
                    continue
                slot = self.held.pop(victim)
            self.cache.load(e, slot, *self.host[e])
            self.held[e] = slot
            loaded += 1
        self.loads += loaded
        return loaded


def experts_of(masks: torch.Tensor):
    """The experts in any of a batch's 64-bit sets, the most wanted first."""
    bits = masks.reshape(-1).cpu().numpy().view(np.uint64)
    votes = [(int(((bits >> np.uint64(e)) & np.uint64(1)).sum()), -e) for e in range(64)]
    return [-e for n, e in sorted(votes, reverse=True) if n]


def normed(x: torch.Tensor) -> torch.Tensor:
    y = x.float()
    return (y * torch.rsqrt(y.square().mean(dim=1, keepdim=True) + 1e-6)).to(x.dtype)


class Model:
    def __init__(self, c: Config = Config(), seed: int = 0):
        g = torch.Generator().manual_seed(seed)
        self.c = c
        self.table = torch.randn(c.V, c.d, generator=g).to(torch.bfloat16).cuda()
        self.layers = [Layer(c, g) for _ in range(c.L)]
        self.store = fm.Store(c.store, c.L, c.E, c.d, "f32")

    def iteration(self, prompts):
        """One iteration of a batch: prompts is a list of token lists.  Returns the hidden states [B][d], the
        expert maps [B][L][E], and how many chosen experts were found in the cache and loaded on demand."""
        c, B = self.c, len(prompts)
        tokens = torch.tensor([t for p in prompts for t in p], dtype=torch.int32, device="cuda")
        offsets = torch.tensor(np.cumsum([0] + [len(p) for p in prompts]), dtype=torch.int32, device="cuda")
        last = torch.tensor([p[-1] if p else -1 for p in prompts], dtype=torch.int32, device="cuda")
        active = (last >= 0).to(torch.uint8)
        scale = c.d ** 0.5
        select = dict(tau=c.tau, k_min=c.K, k_max=c.E)
        maps = torch.empty(B, c.L, c.E, device="cuda")
        whole = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B,), c.L, dtype=torch.int32, device="cuda")

        query = fm.embed_pool(self.table, tokens, offsets, scale)
        known = self.store.size > 0
        if known:
            _, _, masks, _ = fm.match_semantic_select(self.store, query, *whole, **select)
            for l in range(min(c.distance, c.L)):
                self.layers[l].bring_in(experts_of(masks[:, l])[: c.slots])
        x = fm.embed_lookup(self.table, last, scale)
        search = fm.TrajPass(self.store, B)
        found = loaded = 0
        for l, layer in enumerate(self.layers):
            h = normed(x)
            _, ids, weight, chosen = fm.moe_route(h, layer.gate, c.K, renorm=True, active=active,
                                                  out=(maps[:, l], *self._choice(B)))
            ahead = l + c.distance
            if known and ahead < c.L:
                idx, score = search.step(maps[:, l].contiguous(), l)
                masks, _ = fm.select_prefetch(self.store, idx, score, whole[0] + ahead, whole[0] + ahead + 1, **select)
                self.layers[ahead].bring_in(experts_of(masks[:, ahead])[: c.slots])
            # what the batch needs now; more experts than slots take several rounds
            need = experts_of(chosen)
            found += sum(e in layer.held for e in need)
            x = self._experts(layer, h, ids, weight, need, x)
            loaded += len(need)
        # (a batch slot without a request has no iteration: its map of zeros would be the best match of any request
        # that is unlike all others)
        live = [b for b, p in enumerate(prompts) if p]
        done, keys = (maps, query) if len(live) == B else (maps[live], query[live])
        if live and self.store.size + len(live) <= c.store:
            self.store.insert(done, keys)
        elif live:
            self.store.insert_dedup(done, keys, c.distance)
        return x, maps, found, loaded - found

    def tune(self, tokens, wanted, rate: float) -> float:
        """One step of gradient descent on the embedding table that draws the tokens' embeddings to the rows of
        wanted [T][d] (half the squared distance).  Returns the loss before the step."""
        scale = self.c.d ** 0.5
        off = fm.embed_lookup(self.table, tokens, scale).float() - wanted
        grad = fm.embed_grad(off, tokens, self.c.V, scale)
        self.table = (self.table.float() - rate * grad).to(self.table.dtype)
        return 0.5 * float(off.square().sum())

    def _choice(self, B):
        c = self.c
        return (torch.empty(B, c.K, dtype=torch.int32, device="cuda"), torch.empty(B, c.K, device="cuda"),
                torch.empty(B, dtype=torch.int64, device="cuda"))

    def _experts(self, layer, h, ids, weight, need, x):
        done = 0
        need = sorted(need, key=lambda e: e not in layer.held)   # the ones held first
        while done < len(need):
            part = need[done:done + layer.cache.slots]
            layer.bring_in(part, keep=part)
            now = torch.tensor(part, dtype=torch.int32, device="cuda")
            mine = torch.where(torch.isin(ids, now), ids, -1)
            x = fm.moe_experts(layer.cache, h, mine, weight, residual=x)
            done += len(part)
        assert layer.cache.check() == 0
        return x


def main():
    model = Model()
    rng = np.random.default_rng(0)
    topics = [rng.integers(0, model.c.V, 40) for _ in range(6)]   # prompts repeat their topic's words
    for it in range(5):
        prompts = [list(map(int, rng.choice(topics[rng.integers(6)], rng.integers(5, 30)))) for _ in range(8)]
        _, _, found, missed = model.iteration(prompts)
        torch.cuda.synchronize()
        print(f"iteration {it}: {found} of {found + missed} chosen experts were in the cache, {missed} loaded on "
              f"demand; {model.store.size} iterations stored")


if __name__ == "__main__":
    main()
