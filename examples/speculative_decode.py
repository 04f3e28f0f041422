"""Speculative decoding with a small random decoder: rotary positions, attention over a paged cache, MoE layers with
expert skipping, verification of drafted trees. Run on a GPU:

    python examples/speculative_decode.py [--dtype bf16|f32] [--format fp8|plain|int4] [--tokens 64] [--temperature 0.8]

One step, for all requests together: a drafter proposes a small tree of tokens after each request's last one; the
decoder runs all trees' nodes as one batch (requests get pages for them, their rotated K and their V go into the cache at
once, each node attends to the request's prefix and its own ancestors); the verification accepts a path of each tree and
picks the next token; the cache keeps the path's rows.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_05228_gb300 import ace, offline, synth  # noqa: E402

VOCAB, LAYERS, HEADS, KV_HEADS, DIM, PAGE = 512, 2, 8, 2, 64, 16
MAX_NODES = 8
TREE = [-1, 0, 0, 1, 1, 3]          # a drafted tree's parents


class Decoder:
    """Embedding, blocks of attention and an MoE layer, logits. Random weights of the layer's own recipe."""

    def __init__(self, dtype: str = "bf16", fmt: str = "fp8", requests: int = 4, max_len: int = 512, skip: float = 0.25, seed: int = 0):
        spec = synth.LayerSpec(256, 16, 4, 128, dtype=dtype)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        d = spec.hidden

        def w(*shape, scale):
            return (torch.randn(*shape, generator=g, device="cuda") * scale).to(self.dt)

        self.embed = w(VOCAB, d, scale=1.0)
        self.head = w(VOCAB, d, scale=3.0 / d ** 0.5)
        self.qkv = [w((HEADS + 2 * KV_HEADS) * DIM, d, scale=d ** -0.5) for _ in range(LAYERS)]
        self.out = [w(d, HEADS * DIM, scale=(HEADS * DIM) ** -0.5) for _ in range(LAYERS)]
        self.moe = []
        for i in range(LAYERS):
            weights = synth.make_layer(spec, seed=seed + 10 + i)
            self.moe.append(ace.AceLayer(weights, *offline.tables(weights), max_tokens=requests * MAX_NODES, residual=True))
        self.skip = skip
        # the cache: requests get pages as they grow
        per = -(-max_len // PAGE)
        self.kv = ace.AceKvCache(KV_HEADS, DIM, PAGE, requests * per, LAYERS, dtype, fmt)
        self.pages = torch.full((requests, per), -1, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(requests * per, dtype=torch.int32, device="cuda")
        self.missing = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.rope = ace.AceRope(DIM, layout="interleaved", dtype=dtype)

    @staticmethod
    def _norm(x):
        f = x.float()
        return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def forward(self, tokens, parents, offsets, max_nodes: int):
        """Logits [T, VOCAB] of all requests' nodes, whose K and V are in the cache afterwards."""
        T, B = tokens.shape[0], offsets.shape[0] - 1
        mask = torch.empty(T, (max_nodes + 63) // 64, dtype=torch.int64, device="cuda")
        depth = torch.empty(T, dtype=torch.int32, device="cuda")
        ace.ace_tree_mask(parents, offsets, B, max_nodes, mask, depth)
        self.kv.reserve(self.pages, self.lens, offsets[1:] - offsets[:-1], self.refs, self.missing)
        request = torch.repeat_interleave(torch.arange(B, device="cuda"), (offsets[1:] - offsets[:-1]).long(), output_size=T)
        at = self.lens[request].long() + torch.arange(T, device="cuda") - offsets[request].long()
        slots = self.pages[request, at // PAGE].long() * PAGE + at % PAGE
        pos = self.lens[request] + depth
        x = self.embed[tokens.long()]
        for i in range(LAYERS):
            rows = (self._norm(x) @ self.qkv[i].T).view(T, HEADS + 2 * KV_HEADS, DIM)
            q = torch.empty(T, HEADS, DIM, dtype=self.dt, device="cuda")
            self.kv.write_rotated(i, self.rope, pos, rows[:, :HEADS], q, rows[:, HEADS: HEADS + KV_HEADS], rows[:, HEADS + KV_HEADS:], slots)
            o = torch.empty_like(q)
            self.kv.attend(i, q, self.pages, self.lens, offsets, o, mask, max_nodes)
            x = x + o.flatten(1) @ self.out[i].T
            y = torch.empty_like(x)
            self.moe[i].forward(x, y, T, "ratio", self.skip)
            x = y
        return (self._norm(x) @ self.head.T).contiguous()

    def reorder(self, parents):
        """Request b goes on from request parents[b] (int32, negative: it ends and gives its pages back)."""
        pages, lens = torch.empty_like(self.pages), torch.empty_like(self.lens)
        self.kv.fork(self.pages, self.lens, parents, self.refs, pages, lens)
        self.pages, self.lens = pages, lens

    def keep(self, path, n_keep):
        new = torch.empty_like(self.lens)
        self.kv.keep(self.pages, self.lens, path, n_keep, new)
        self.lens = new


def draft_trees(last, decoder, drafted: bool):
    """A tree after each request's last token: two children by a bigram drafter, two below the first, one below that.
    Returns tokens, parents, offsets and the drafter's probabilities. `drafted` False: the last token alone."""
    B = last.shape[0]
    shape = TREE if drafted else [-1]
    n = len(shape)
    tokens = torch.empty(B, n, dtype=torch.int32, device="cuda")
    probs = torch.empty(B, n, VOCAB, device="cuda")
    tokens[:, 0] = last
    for i in range(n):
        # a drafter that sees one token: the decoder's own logits of its embedding
        probs[:, i] = torch.softmax((decoder._norm(decoder.embed[tokens[:, i].long()]) @ decoder.head.T).float(), -1)
        kids = [j for j in range(n) if shape[j] == i]
        if kids:
            race = probs[:, i] / torch.empty_like(probs[:, i]).exponential_()        # draws without replacement
            tokens[:, kids] = race.topk(len(kids), -1).indices.int()
    parents = torch.tensor(shape, dtype=torch.int32, device="cuda").repeat(B)
    offsets = torch.arange(0, B * n + 1, n, dtype=torch.int32, device="cuda")
    return tokens.view(-1), parents, offsets, probs.view(-1, VOCAB), n


def positions(count: int, drafted: bool = True) -> int:
    """Cache rows that `count` tokens of the slowest request may take of the fastest: a token a step and a whole path a step,
    and the tree of the last step."""
    depth = [1] * len(TREE)
    for i, p in enumerate(TREE[1:], 1):
        depth[i] = depth[p] + 1
    return max((count - 1) * max(depth) + len(TREE), count * max(depth)) if drafted else count


def generate(decoder: Decoder, first, count: int, temperature: float, drafted: bool = True):
    """`count` tokens (or a few more) of every request after its `first` one: [B] lists, and the steps taken."""
    B = first.shape[0]
    have = decoder.pages.shape[1] * PAGE - int(decoder.lens.max())
    if positions(count, drafted) > have:
        raise ValueError(f"{count} tokens may take {positions(count, drafted)} positions of a request, which has {have} left")
    out = [[] for _ in range(B)]
    temps = torch.full((B,), temperature, device="cuda")
    last, steps = first.int(), 0
    while min(len(o) for o in out) < count:
        tokens, parents, offsets, probs, n = draft_trees(last, decoder, drafted)
        logits = decoder.forward(tokens, parents, offsets, MAX_NODES)
        path = torch.empty(B, MAX_NODES, dtype=torch.int32, device="cuda")
        n_keep, nxt = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
        noise = torch.empty(B, VOCAB, device="cuda").exponential_().clamp_(min=1e-30)
        ace.ace_verify_tree(logits, tokens, parents, offsets, MAX_NODES, torch.rand(B * n, device="cuda"), noise, path, n_keep, nxt,
                            probs, temps)
        if short := int(decoder.missing):               # the step's rows had no place (a wait, as for its tokens below)
            raise RuntimeError(f"the cache's pool is {short} pages short of what the requests need")
        decoder.keep(path, n_keep)
        for b, (p, k, t) in enumerate(zip(path.tolist(), n_keep.tolist(), nxt.tolist())):
            out[b] += [int(tokens[b * n + i]) for i in p[1:k]] + [t]
        last = nxt
        steps += 1
    decoder.kv.sync()
    return out, steps


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--dtype", default="bf16", choices=("bf16", "f32"))
    ap.add_argument("--format", default="fp8", choices=("fp8", "plain", "int4"))
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--temperature", type=float, default=0.8)
    a = ap.parse_args()
    torch.manual_seed(0)
    decoder = Decoder(a.dtype, a.format, max_len=positions(a.tokens))
    out, steps = generate(decoder, torch.arange(4, device="cuda"), a.tokens, a.temperature)
    made = np.mean([len(o) for o in out])
    print(f"{made:.1f} tokens a request in {steps} steps ({made / steps:.2f} a step)")
    for o in out:
        print(" ".join(map(str, o[:16])), "...")


if __name__ == "__main__":
    main()
