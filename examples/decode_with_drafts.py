"""A text model's decoding loop over a key/value cache in the store's pages.

A toy transformer with random weights (there is nothing to download) takes ragged
prompts, then decodes step by step: a cheap guess drafts a tree of tokens, one
pass of the model attends over the tree, and the longest path that the model
agrees with is kept. The cache grows in pages of the same store that hands
tensors between model functions.

    python examples/decode_with_drafts.py [--steps 8]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_26566_gb300 import KVCache, Store, page_tokens  # noqa: E402

VOCAB, WIDTH, HEADS, KV_HEADS, DIM, LAYERS = 512, 256, 8, 2, 64, 2
BRANCH, DEPTH = 3, 3  # a drafted tree: BRANCH tries for the next token, each followed to DEPTH


class Model:
    def __init__(self, device, seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        r = lambda *s: torch.randn(*s, device=device, generator=g).mul_(s[0] ** -0.5).bfloat16()  # noqa: E731
        self.embed = torch.randn(VOCAB, WIDTH, device=device, generator=g).bfloat16()
        # a token's likeliest successor, unless what came before says otherwise
        self.follow = torch.randperm(VOCAB, device=device, generator=g)
        self.head = torch.empty_like(self.embed)
        self.head[self.follow] = self.embed
        self.layers = [dict(qkv=r(WIDTH, (HEADS + 2 * KV_HEADS) * DIM), out=r(HEADS * DIM, WIDTH),
                            norms=1 + 0.1 * torch.randn(2, DIM, device=device, generator=g)) for _ in range(LAYERS)]
        a = torch.arange(4096, device=device)[:, None] * 10000.0 ** (-torch.arange(DIM // 2, device=device) / (DIM // 2))
        self.cos, self.sin = a.cos(), a.sin()

    def __call__(self, cache, tokens, lens, starts, max_new, max_len, tree=None, positions=None):
        """Logits of packed new tokens; their keys and values go to the cache."""
        x = self.embed[tokens]
        how = dict(starts=starts, max_new=max_new)
        for i, w in enumerate(self.layers):
            q, k, v = (x @ w["qkv"]).split([HEADS * DIM, KV_HEADS * DIM, KV_HEADS * DIM], dim=1)
            n = len(x)
            q = cache.append(k.view(n, KV_HEADS, DIM), v.view(n, KV_HEADS, DIM), lens, q=q.view(n, HEADS, DIM), layer=i,
                             q_norm=w["norms"][0], k_norm=w["norms"][1], cos=self.cos, sin=self.sin, positions=positions, **how)
            if tree is None:
                y = cache.attend(q, lens, layer=i, max_len=max_len, **how)
            else:
                y = cache.attend_tree(q, lens, tree, layer=i, max_len=max_len, **how)
            x = torch.nn.functional.rms_norm(x + y.view(n, -1) @ w["out"], (WIDTH,))
        return x.float() @ self.head.float().T


def draft(model, last):
    """A tree behind token `last`: itself, then BRANCH chains by a bigram guess. Tokens, parents, ancestor words, depths."""
    follow = model.follow.tolist()
    tokens, parents = [last], [-1]
    for t in (model.embed[last].float() @ model.head.float().T).topk(BRANCH).indices.tolist():
        parent = 0
        for _ in range(DEPTH):
            tokens.append(t)
            parents.append(parent)
            parent, t = len(tokens) - 1, follow[t]
    words, depth = [], []
    for i, p in enumerate(parents):
        words.append((words[p] if p >= 0 else 0) | 1 << i)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return tokens, parents, words, depth


def decode(prompts, steps, device="cuda", seed=0):
    """Continues each prompt; returns the sequences and how many tokens each pass gave."""
    model = Model(device, seed)
    page = 1 << 16
    n = len(prompts)
    most = max(len(p) for p in prompts) + steps * (DEPTH + 1) + 64
    T = page_tokens(page, KV_HEADS, DIM, layers=LAYERS)
    store = Store(torch.empty(n * (-(-most // T) + 1) * page, dtype=torch.uint8, device=device), page)
    cache = KVCache(store, KV_HEADS, DIM, layers=LAYERS, max_seqs=n, max_tokens=most)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=device)  # noqa: E731

    # the prompts but for their last token, which begins the first draft
    new = [len(p) - 1 for p in prompts]
    cache.reserve([m + 64 for m in new])
    model(cache, torch.tensor(np.concatenate([p[:-1] for p in prompts]), device=device), ints(new),
          ints(np.cumsum([0] + new)), max(new), max(new))
    ctx, seqs, gained = list(new), [list(p) for p in prompts], []
    for _ in range(steps):
        trees = [draft(model, s[-1]) for s in seqs]
        m = len(trees[0][0])
        cache.reserve([c + m for c in ctx])
        lens = [c + m for c in ctx]
        logits = model(cache, torch.tensor(np.concatenate([t[0] for t in trees]), device=device), ints(lens),
                       ints(np.arange(n + 1) * m), m, max(lens), tree=torch.tensor(np.concatenate([t[2] for t in trees]), device=device),
                       positions=ints(np.concatenate([[c + d for d in t[3]] for c, t in zip(ctx, trees)])))
        choice = logits.argmax(-1).view(n, m).tolist()
        path = np.zeros((n, m), np.int32)
        counts = []
        for s, (tokens, parents, _, _) in enumerate(trees):
            node, kept = 0, [0]
            while True:  # follow what the model would have said
                child = [i for i in range(m) if parents[i] == node and tokens[i] == choice[s][node]]
                seqs[s].append(choice[s][node])
                if not child:
                    break
                node = child[0]
                kept.append(node)
            path[s, :len(kept)] = kept
            counts.append(len(kept))
        cache.commit(ints(ctx), torch.from_numpy(path).to(device), ints(counts))
        ctx = [c + k for c, k in zip(ctx, counts)]
        gained.append(counts)
    return seqs, gained


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=8)
    args = ap.parse_args()
    rng = np.random.default_rng(0)
    prompts = [rng.integers(0, VOCAB, k).tolist() for k in (17, 200, 65)]
    seqs, gained = decode(prompts, args.steps)
    for p, s in zip(prompts, seqs):
        print(f"{len(p)} tokens, then {s[len(p):]}")
    print("tokens kept a pass:", gained)


if __name__ == "__main__":
    main()
