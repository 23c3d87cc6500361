"""From prompts' tokens to placements on model instances, all on one GPU.

A small decoder-only text model (random weights) reads a batch of prompts one
token a step.  Its layers call the library for what is not a plain matrix
product: the norms with the residual's addition (apc_norm_rows), the paged
key-value cache in e4m3 (apc_kv_write) and the attention over it (apc_attend).
All prompts begin with the same instruction, whose pages are filled once and
stand in every prompt's page table.  The last norm leaves each prompt's
embedding as an e4m3 row with its scale, which is what the matching step takes:
nearest cached prompts, skip level, placement and the cached latents
(MatchStep).

    python examples/embed_and_match.py
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2502_06798_amd as apc  # noqa: E402
from paper_2502_06798_amd import synth  # noqa: E402


class TextModel:
    """Weights, drawn from a seed: `layers` blocks of width q_heads * d, key-value heads shared by query heads."""

    def __init__(self, vocab=1000, places=512, layers=2, q_heads=12, heads=4, d=64, ff=2048, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        w = q_heads * d
        rand = lambda *s: (torch.randn(*s, generator=g) * s[-1] ** -0.5).to(torch.bfloat16).to(device)
        self.layers, self.q_heads, self.heads, self.d, self.width = layers, q_heads, heads, d, w
        self.emb, self.pos = rand(vocab, w) * w ** 0.5, rand(places, w) * w ** 0.5
        self.blocks = [dict(n1=1 + rand(w), qkv=rand((q_heads + 2 * heads) * d, w), o=rand(w, w), n2=1 + rand(w),
                            up=rand(ff, w), down=rand(w, ff)) for _ in range(layers)]
        self.last = 1 + rand(w)


class Reader:
    """A batch of sequences over paged caches (one pool a layer): pages, lengths and the buffers of a step."""

    def __init__(self, model: TextModel, b: int, pages: int, per_sequence: int, page: int = 16, device="cuda"):
        self.m, self.b, self.page = model, b, page
        m, shape = model, (pages, model.heads, page, model.d)
        e4m3 = lambda: torch.zeros(shape, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)
        scale = lambda: torch.zeros(shape[:3], device=device)
        self.caches = [apc.KvCache(e4m3(), e4m3(), scale(), scale()) for _ in range(m.layers)]
        self.free = list(range(pages - 1, -1, -1))
        self.rows = [[] for _ in range(b)]                              # pages of each sequence (host)
        self.table = torch.full((b, per_sequence), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(b, dtype=torch.int32, device=device)
        self.ws = apc.attend_workspace_tensor(self.caches[0], b, m.q_heads, per_sequence)
        half = dict(dtype=torch.bfloat16, device=device)
        self.x, self.heads_out = torch.empty((b, m.width), **half), torch.empty((b, m.q_heads, m.d), **half)
        self.embedding = torch.empty((b, m.width), dtype=torch.float8_e4m3fn, device=device)
        self.embedding_scale = torch.empty(b, device=device)

    def share(self, other: "Reader"):
        """Starts every sequence with the whole pages of `other`'s only sequence, in `other`'s pools."""
        assert other.b == 1 and int(other.lengths[0]) % self.page == 0
        self.caches, self.free = other.caches, other.free
        for row in self.rows:
            row.extend(other.rows[0])
        self.table[:, :len(other.rows[0])] = other.table[:, :len(other.rows[0])]
        self.lengths += other.lengths

    def step(self, ids: torch.Tensor, live: np.ndarray):
        """One token of each sequence that has one (live): its keys and values into the cache, its state through the
        blocks; embeddings of the last tokens in self.embedding, self.embedding_scale."""
        m, place = self.m, self.lengths.cpu().numpy()
        slots = np.full(self.b, -1, np.int32)                           # -1: nothing is written
        for i in np.flatnonzero(live):
            if place[i] % self.page == 0:
                self.rows[i].append(self.free.pop())
                self.table[i, len(self.rows[i]) - 1] = self.rows[i][-1]
            slots[i] = self.rows[i][-1] * self.page + place[i] % self.page
        slots = torch.from_numpy(slots).to(self.table.device)
        here = torch.from_numpy(live.astype(np.int32)).to(self.table.device)
        r = m.emb[ids] + m.pos[self.lengths.long()]                     # the residual, updated in place by the norms
        self.lengths += here
        y = None
        for block, cache in zip(m.blocks, self.caches):
            apc.apc_norm_rows(r if y is None else y, self.x, block["n1"], None if y is None else r, None if y is None else r)
            qkv = (self.x @ block["qkv"].t()).view(self.b, -1, m.d)     # queries, keys and values side by side
            q, k, v = qkv.split([m.q_heads, m.heads, m.heads], dim=1)
            apc.apc_kv_write(cache, k, v, slots)
            apc.apc_attend(cache, q, self.table, self.lengths, m.d ** -0.5, self.heads_out, self.ws)
            y = self.heads_out.view(self.b, -1) @ block["o"].t()
            apc.apc_norm_rows(y, self.x, block["n2"], r, r)
            y = torch.nn.functional.silu(self.x @ block["up"].t()) @ block["down"].t()
        apc.apc_norm_rows(y, self.embedding, m.last, r, r, self.embedding_scale)

    def read(self, prompts):
        """Reads whole prompts (lists of token numbers, one for each sequence); returns copies of their embeddings."""
        out, scale = torch.zeros_like(self.embedding), torch.ones_like(self.embedding_scale)
        for t in range(max(len(p) for p in prompts)):
            live = np.array([t < len(p) for p in prompts])
            ids = torch.tensor([p[min(t, len(p) - 1)] for p in prompts], device=self.table.device)
            self.step(ids, live)
            last = torch.tensor([t == len(p) - 1 for p in prompts], device=self.table.device)
            out.view(torch.uint8)[last] = self.embedding.view(torch.uint8)[last]
            scale[last] = self.embedding_scale[last]
        return out, scale


def embed(model: TextModel, instruction, prompts, shared=True):
    """e4m3 embeddings and scales of the prompts after the instruction, its pages shared or read by every sequence."""
    page, b = 16, len(prompts)
    most = len(instruction) + max(len(p) for p in prompts)
    per = -(-most // page)
    first = Reader(model, 1, (b + 1) * per, per)
    if not shared:
        return Reader(model, b, (b + 1) * per, per).read([list(instruction) + list(p) for p in prompts])
    first.read([instruction])
    rest = Reader(model, b, 1, per)
    rest.share(first)
    return rest.read(prompts)


def main(n_cached=256, b=32, seed=1):
    apc.load()
    rng = np.random.default_rng(seed)
    model = TextModel()
    instruction = rng.integers(0, 1000, 32).tolist()
    cached = [rng.integers(0, 1000, rng.integers(5, 30)).tolist() for _ in range(n_cached)]
    source = rng.choice(n_cached, b, replace=False)
    # new prompts: cached ones, every other with one of its first tokens changed
    prompts = [list(cached[s]) for s in source]
    for p in prompts[1::2]:
        p[rng.integers(0, 3)] = int(rng.integers(0, 1000))

    e, es = embed(model, instruction, cached)
    pool = torch.zeros((n_cached, 32768), dtype=torch.uint8, device="cuda")
    cache = apc.apc_build_cache(e, es, pool)
    step = apc.MatchStep(cache, b, 5, synth.THETA5, synth.K5, [0, 1, 2, 3, 4, 5], [b] * 6, latent_bytes=32768)
    q, qs = embed(model, instruction, prompts)
    step.run(q, qs)
    torch.cuda.synchronize()
    top = step.top_idx[:, 0].cpu().numpy()
    found = int((top == source).sum())
    print(f"{b} prompts of {min(map(len, prompts))} to {max(map(len, prompts))} tokens against {n_cached} cached ones: "
          f"{found} nearest to the prompt they came from, levels {np.bincount(step.out_level.cpu().numpy(), minlength=6).tolist()}, "
          f"{int(step.hit.sum())} latents gathered")
    cache.close()
    return found, source, top, step.top_score[:, 0].cpu().numpy()


if __name__ == "__main__":
    main()
