"""Speculative decoding on sealed, paged KV: a prefill worker seals the KV of several users' prompts, a decode worker
opens it into its own paged cache and generates with trees of drafted tokens.

    python examples/speculative_decode.py

The model is a small decoder with random weights.  What the framework does here:

  prefill  gift.kv_tables     blocks and slots for the prompts
           gift.kv_append     their K and V, all layers, into the cache
           gift.seal_paged    each request under its user's key
  handoff  gift.open_paged    into other blocks of the decode worker's cache
  a step   gift.kv_tables     the owner check of the blocks that the step will read, nothing added yet
           gift.tree_attention  the drafted tree of every request over its cached tokens, layer by layer, under the
                              check's verdicts
           gift.kv_tables     blocks and slots for what was accepted, and the owner check once more
           gift.kv_append     the accepted rows, all layers
  at last  gift.seal_paged    the requests' blocks, to be swapped out

Drafts come from a table of the model's own favourite successors, so that some are accepted.  The result is checked
against the same model in 32 bits without a cache.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_25431_amd import gift  # noqa: E402

DEV = "cuda"
LAYERS, HEADS, KV_HEADS, DIM, VOCAB, BLOCK = 2, 8, 2, 64, 256, 16
HIDDEN = HEADS * DIM


class Model:
    """A decoder without MLPs: embeddings of token and position, then attention layers."""

    def __init__(self, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def w(*shape):
            return torch.randn(*shape, generator=g, device=DEV) / shape[0] ** 0.5

        self.token = torch.randn(VOCAB, HIDDEN, generator=g, device=DEV)
        self.place = 0.3 * torch.randn(4096, HIDDEN, generator=g, device=DEV)
        self.qkv = [w(HIDDEN, HIDDEN + 2 * KV_HEADS * DIM) for _ in range(LAYERS)]
        self.out = [w(HIDDEN, HIDDEN) for _ in range(LAYERS)]
        self.head = w(HIDDEN, VOCAB)

    def embed(self, tokens, places):
        return self.token[tokens] + self.place[places]

    def project(self, x, layer):
        y = (x / x.norm(dim=-1, keepdim=True) * HIDDEN ** 0.5) @ self.qkv[layer]
        q, k, v = y.split([HIDDEN, KV_HEADS * DIM, KV_HEADS * DIM], dim=-1)
        return q.view(-1, HEADS, DIM), k.view(-1, KV_HEADS, DIM), v.view(-1, KV_HEADS, DIM)

    def logits(self, tokens):
        """Of every position of one sequence, in 32 bits without a cache, and K and V of all layers."""
        n = len(tokens)
        x = self.embed(tokens, torch.arange(n, device=DEV))
        seen = torch.ones(n, n, dtype=torch.bool, device=DEV).tril()
        keys, values = [], []
        for i in range(LAYERS):
            q, k, v = self.project(x, i)
            keys.append(k)
            values.append(v)
            k, v = (t.repeat_interleave(HEADS // KV_HEADS, 1).transpose(0, 1).contiguous() for t in (k, v))
            s = torch.matmul(q.transpose(0, 1), k.transpose(1, 2)) * DIM ** -0.5
            o = torch.matmul(s.masked_fill(~seen, float("-inf")).softmax(-1), v)
            x = x + o.transpose(0, 1).reshape(n, HIDDEN) @ self.out[i]
        return x @ self.head, torch.stack(keys), torch.stack(values)


class Worker:
    """A paged cache, and the block tables of n requests in it."""

    def __init__(self, n, blocks, width, users, seed):
        plane = KV_HEADS * BLOCK * DIM
        self.cache = torch.zeros(LAYERS, blocks, 2, KV_HEADS, BLOCK, DIM, dtype=torch.bfloat16, device=DEV)
        self.kv = gift.paged_kv(self.cache, self.cache.nbytes, 4 * plane * blocks, 4 * plane, 4 * plane, 4 * plane, LAYERS, 1,
                                blocks)
        self.fmt = gift.kv_format(torch.bfloat16, KV_HEADS, DIM, BLOCK, 2 * DIM, 2 * BLOCK * DIM, 2 * plane)
        self.users = torch.tensor(users, dtype=torch.int32, device=DEV)
        self.free = torch.from_numpy(np.random.default_rng(seed).permutation(blocks).astype(np.int32)).to(DEV)
        self.tables = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
        self.labels = torch.full((blocks,), -1, dtype=torch.int32, device=DEV)  # gift.LABEL_UNOWNED
        self.lens = torch.zeros(n, dtype=torch.int32, device=DEV)

    def grow(self, new):
        """Blocks and slots for new tokens; returns (slots, verdicts)."""
        n, rows = len(new), int(sum(new))
        slots = torch.empty(rows, dtype=torch.int64, device=DEV)
        begin, lens, verdicts = (torch.empty(k, dtype=torch.int32, device=DEV) for k in (n + 1, n, n))
        taken = torch.empty(1, dtype=torch.int32, device=DEV)
        gift.kv_tables(self.users, self.lens, torch.tensor(new, dtype=torch.int32, device=DEV), BLOCK, self.free, self.tables,
                       self.labels, slots, begin, lens, taken, verdicts)
        self.free = self.free[int(taken):]
        self.lens = lens
        return slots, verdicts

    def blocks_of(self, b):
        return self.tables[b, :-(-int(self.lens[b]) // BLOCK)].cpu().numpy().astype(np.uint32)

    def requests(self, seq):
        users = self.users.tolist()
        return [(self.blocks_of(b), users[b], seq * len(users) + b) for b in range(len(users))]  # no IV twice


def handoff(prefill, decode, kt, nonces):
    """Seals every request out of one worker's cache and opens it into the other's."""
    reqs = prefill.requests(1)
    size = sum(len(r[0]) for r in reqs) * LAYERS * prefill.kv.chunk_bytes
    sealed = torch.empty(size, dtype=torch.uint8, device=DEV)
    tags = torch.empty(16 * len(reqs), dtype=torch.uint8, device=DEV)
    gift.seal_paged(prefill.kv, reqs, kt, nonces, sealed, tags, block_labels=prefill.labels)
    verdicts = torch.empty(len(reqs), dtype=torch.int32, device=DEV)
    gift.open_paged(decode.kv, [(decode.blocks_of(b), u, s) for b, (_, u, s) in enumerate(reqs)], kt, nonces, sealed, tags,
                    verdicts, block_labels=decode.labels)
    return verdicts.tolist()


def tree_of(root, likely, width, depth):
    """Tokens and parents of a draft tree: the root (the last accepted token) and its likely successors."""
    tokens, parents, level = [root], [-1], [0]
    for d in range(depth):
        after = []
        for node in level:
            for t in likely[tokens[node]][:max(1, width - d)]:
                tokens.append(int(t))
                parents.append(node)
                after.append(len(tokens) - 1)
        level = after
    return tokens, parents


def step(model, worker, work, trees, lens):
    """Logits of every tree's nodes, and K and V of all layers.  A request whose table names another user's block reads
    none of it: its attention is zeros."""
    _, verdicts = worker.grow([0] * len(trees))
    counts = [len(t) for t, _ in trees]
    begin = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV)
    mask, places = np.zeros((sum(counts), -(-max(counts) // 32) * 32), np.uint8), []
    row = 0
    for (tokens, parents), length in zip(trees, lens):
        deep = []
        for i, p in enumerate(parents):
            if p >= 0:
                mask[row + i] = mask[row + p]
            mask[row + i, i] = 1
            deep.append(0 if p < 0 else deep[p] + 1)
            places.append(length + deep[i])
        row += len(tokens)
    mask = torch.from_numpy(np.packbits(mask, axis=1, bitorder="little").view(np.int32)).to(DEV)
    tokens = torch.tensor([t for tree, _ in trees for t in tree], device=DEV)
    x = model.embed(tokens, torch.tensor(places, device=DEV))
    keys, values = [], []
    for layer in range(LAYERS):
        q, k, v = (t.to(torch.bfloat16) for t in model.project(x, layer))
        out = torch.empty_like(q)
        gift.tree_attention(work, worker.kv, worker.fmt, layer, q, k, v, begin, worker.lens, worker.tables, out, mask=mask,
                            verdicts=verdicts)
        keys.append(k)
        values.append(v)
        x = x + out.float().reshape(-1, HIDDEN) @ model.out[layer]
    return x @ model.head, torch.stack(keys), torch.stack(values)


def accepted(tokens, parents, best):
    """Nodes of the path that the model itself would have taken, and its token after the last of them."""
    path = [0]
    while True:
        want = best[path[-1]]
        child = [i for i, p in enumerate(parents) if p == path[-1] and tokens[i] == want]
        if not child:
            return path, want
        path.append(child[0])


def main(prompts=(37, 5, 64, 16), steps=12, seed=3, verbose=True):
    torch.backends.cuda.matmul.allow_tf32 = False
    model, n, users = Model(seed), len(prompts), [7, 2, 7, 5]
    r = np.random.default_rng(seed)
    keys, nonces = r.integers(0, 256, (8, 32), dtype=np.uint8), r.integers(0, 256, (8, 12), dtype=np.uint8)
    kt, work = gift.KeyTable(keys), gift.AttentionWork()
    texts = [r.integers(0, VOCAB, k).tolist() for k in prompts]
    likely = model.logits(torch.arange(VOCAB, device=DEV))[0].topk(3).indices.cpu().numpy()

    # prefill: K and V of all tokens but the last, which is the root of the first trees
    prefill, decode = (Worker(n, 64, 24, users[:n], s) for s in (1, 2))
    new = [len(t) - 1 for t in texts]
    kv = [model.logits(torch.tensor(t[:-1], device=DEV))[1:] for t in texts]
    k, v = (torch.cat([x[i] for x in kv], 1).to(torch.bfloat16) for i in (0, 1))
    slots, verdicts = prefill.grow(new)
    assert verdicts.tolist() == [gift.SEG_OK] * n
    gift.kv_append(prefill.kv, prefill.fmt, slots, k, v)
    _, verdicts = decode.grow(new)
    assert verdicts.tolist() == [gift.SEG_OK] * n
    assert handoff(prefill, decode, kt, nonces) == [gift.SEG_OK] * n

    made = 0
    for _ in range(steps):
        for t in texts:  # the favourites of a real context, as a drafting model would know them
            last = model.logits(torch.tensor(t, device=DEV))[0][-1]
            likely[t[-1]] = last.topk(3).indices.cpu().numpy()
        trees = [tree_of(t[-1], likely, 3, 3) for t in texts]
        logits, k, v = step(model, decode, work, trees, [len(t) - 1 for t in texts])
        best, row, index, new = logits.argmax(-1).tolist(), 0, [], []
        for t, (tokens, parents) in zip(texts, trees):
            path, after = accepted(tokens, parents, best[row:row + len(tokens)])
            t.extend([tokens[i] for i in path[1:]] + [after])
            index.extend(row + i for i in path)
            new.append(len(path))
            row += len(tokens)
            made += len(path)
        slots, verdicts = decode.grow(new)
        assert verdicts.tolist() == [gift.SEG_OK] * n
        gift.kv_append(decode.kv, decode.fmt, slots, k, v, index=torch.tensor(index, dtype=torch.int32, device=DEV))

    # every generated token is what the model prefers in 32 bits, up to what bfloat16 K, V and outputs change
    gap = 0.0
    for t, start in zip(texts, prompts):
        logits = model.logits(torch.tensor(t, device=DEV))[0]
        chosen = logits[torch.arange(start - 1, len(t) - 1), torch.tensor(t[start:], device=DEV)]
        gap = max(gap, float((logits[start - 1:-1].amax(-1) - chosen).max()) / float(logits.std()))

    # a table that names another user's block is found out: no slots, a verdict, and attention that gives zeros
    decode.tables[0, 0] = decode.tables[1, 0]
    _, verdicts = decode.grow([1] * n)
    seen = verdicts.tolist()
    q = torch.randn(n, HEADS, DIM, device=DEV).to(torch.bfloat16)
    out = torch.empty_like(q)
    gift.tree_attention(work, decode.kv, decode.fmt, 0, q, None, None, torch.arange(n + 1, dtype=torch.int32, device=DEV),
                        decode.lens, decode.tables, out, verdicts=verdicts)
    kept = bool((out[0] == 0).all()) and bool((out[1:].abs().amax((1, 2)) > 0).all())

    # the other requests leave the cache sealed
    reqs = decode.requests(2)[1:]
    sealed = torch.empty(sum(len(x[0]) for x in reqs) * LAYERS * decode.kv.chunk_bytes, dtype=torch.uint8, device=DEV)
    tags, ok = torch.empty(16 * len(reqs), dtype=torch.uint8, device=DEV), torch.empty(len(reqs), dtype=torch.int32, device=DEV)
    gift.seal_paged(decode.kv, reqs, kt, nonces, sealed, tags, block_labels=decode.labels, verdicts=ok)
    result = dict(tokens=made, per_step=made / (steps * n), gap=gap, verdicts=seen, zeroed=kept, sealed=ok.tolist())
    if verbose:
        print(f"{made} tokens in {steps} steps of {n} requests ({result['per_step']:.2f} a step and request); largest gap to the "
              f"preferred token {gap:.4f} of the logits' deviation; after a manipulated table: verdicts {seen}, "
              f"its rows zero and the others not: {kept}; sealed: {result['sealed']}")
    work.destroy()
    kt.destroy()
    return result


if __name__ == "__main__":
    main()
