"""The decode step of speculative serving on a paged KV cache, as cases that can be timed and compared.

Three operators, each reached through the public binding (paper_2608_25431_amd.gift):

  tables     block tables, slot maps and the owner check from request lengths (gift.kv_tables)
  append     rows of K and V of all layers into the slots of a paged cache (gift.kv_append)
  attention  attention of a tree of drafted tokens over a paged cache (gift.tree_attention)

A cache has blocks of `block` tokens; K and V of a (layer, block) lie in one chunk or in two planes (`parts`), head by
head or token by token (`order`).  Request lengths come from the case alone (its numbers seed them), contents from the seed.
The plain forms pad every request to the longest of the case and compute in 32 bits.
"""
import math
import random

import numpy as np
import torch

DEVICE = "cuda"
own = False
_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
_LABEL_UNOWNED = -1  # 0xFFFFFFFF as int32
_OK, _MIXED, _NO_SPACE = 0, 2, 3


def listed():
    return [
        # one user, one short prompt, a draft of four tokens: launches and latency decide
        dict(name="attention_tiny", kind="attention", reqs=1, lo=37, hi=37, dlo=4, dhi=4, heads=32, kv_heads=8, dim=128,
             block=16, order="head", parts=1, layers=2, dtype="bf16", tree="tree", rejected=0),
        # single-token decode of the Llama-3-8B handoff's 64 requests, 128-2048 tokens each: no draft, one row a request
        dict(name="attention_single", kind="attention", reqs=64, lo=128, hi=2048, dlo=1, dhi=1, heads=32, kv_heads=8,
             dim=128, block=16, order="token", parts=1, layers=2, dtype="bf16", tree="chain", rejected=0),
        # the same requests, each with a tree of 8 to 32 drafted tokens; one request's table names another user's block
        dict(name="attention_tree", kind="attention", reqs=64, lo=128, hi=2048, dlo=8, dhi=32, heads=32, kv_heads=8,
             dim=128, block=16, order="head", parts=1, layers=2, dtype="bf16", tree="tree", rejected=1),
        # Llama-3-70B handoff: 32 requests of 2048-8192 tokens, 64 query heads over 8, trees of 16 to 32 tokens
        dict(name="attention_wide", kind="attention", reqs=32, lo=2048, hi=8192, dlo=16, dhi=32, heads=64, kv_heads=8,
             dim=128, block=16, order="head", parts=1, layers=1, dtype="bf16", tree="tree", rejected=0),
        # one long document: few rows over a long axis
        dict(name="attention_long", kind="attention", reqs=1, lo=131072, hi=131072, dlo=5, dhi=5, heads=32, kv_heads=8,
             dim=128, block=64, order="token", parts=2, layers=1, dtype="f16", tree="tree", rejected=0),
        # a mixed batch: empty and odd contexts, requests without drafts, rows whose mask leaves nothing, one KV head
        # for each query head, odd head count
        dict(name="attention_ragged", kind="attention", reqs=37, lo=0, hi=513, dlo=0, dhi=63, heads=10, kv_heads=10,
             dim=64, block=32, order="token", parts=2, layers=3, dtype="f16", tree="holes", rejected=1),
        # a decode step's tables: 1024 requests that accepted 1-4 tokens each
        dict(name="tables_step", kind="tables", reqs=1024, lo=128, hi=2048, nlo=1, nhi=4, block=16, spare=0, mixed=3),
        # prompts coming in: nothing cached yet, every block is new
        dict(name="tables_prompts", kind="tables", reqs=64, lo=0, hi=0, nlo=128, nhi=2048, block=16, spare=0, mixed=0),
        # long documents: the owner check reads many blocks; the pool runs out before the last requests
        dict(name="tables_long", kind="tables", reqs=32, lo=32768, hi=131072, nlo=1, nhi=32, block=16, spare=-4, mixed=1),
        # one accepted token of one user
        dict(name="append_tiny", kind="append", reqs=1, nlo=1, nhi=1, drafted=4, layers=2, kv_heads=8, dim=128, block=16,
             order="head", parts=1, dtype="bf16"),
        # the accepted tokens of a speculative step, out of the drafted rows of all 32 layers
        dict(name="append_accepted", kind="append", reqs=64, nlo=1, nhi=4, drafted=16, layers=32, kv_heads=8, dim=128,
             block=16, order="head", parts=1, dtype="bf16"),
        # prompts of 16 requests, 32 layers: a large copy
        dict(name="append_prompts", kind="append", reqs=16, nlo=128, nhi=2048, drafted=0, layers=32, kv_heads=8, dim=128,
             block=16, order="token", parts=1, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "tables", "append"])
    block = rng.choice([1, 8, 16, 16, 32, 64, 128])
    if kind == "tables":
        reqs = _log_int(rng, 1, 1024)
        hi = _log_int(rng, 1, 131072 if reqs <= 32 else 4096)
        nhi = _log_int(rng, 1, 2048 if reqs <= 64 else 32)
        block = max(block, 8)
        return dict(kind="tables", reqs=reqs, lo=rng.randint(0, hi), hi=hi, nlo=rng.randint(0, nhi), nhi=nhi, block=block,
                    spare=rng.choice([-3, 0, 0, 7]), mixed=rng.choice([0, 1, 2]))
    order, parts, dtype = rng.choice(["head", "token"]), rng.choice([1, 2]), rng.choice(["bf16", "f16"])
    dim, kv_heads = rng.choice([64, 96, 128, 128, 256]), rng.choice([1, 2, 4, 5, 8, 10, 16])
    if kind == "append":
        reqs, layers = _log_int(rng, 1, 64), rng.choice([1, 2, 16, 28, 32])
        nhi = _log_int(rng, 1, max(1, min(2048, int(2 ** 32 / (2 * reqs * layers * kv_heads * dim * 4)))))
        return dict(kind="append", reqs=reqs, nlo=rng.randint(0, nhi), nhi=nhi, drafted=rng.choice([0, nhi, nhi + 5]),
                    layers=layers, kv_heads=kv_heads, dim=dim, block=block, order=order, parts=parts, dtype=dtype)
    reqs = _log_int(rng, 1, 256)
    group = rng.choice([1, 2, 4, 7, 8])
    dhi = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 2, 64)])
    room = 2 ** 26 // (reqs * kv_heads * dim) * 2  # cached tokens a request, so that the case costs no more than the listed ones
    room = min(room, 2 ** 31 // (reqs * kv_heads * group * dhi))
    hi = _log_int(rng, 1, max(2, min(131072, room)))
    return dict(kind="attention", reqs=reqs, lo=rng.randint(0, hi), hi=hi, dlo=rng.randint(0 if dhi > 1 else 1, dhi), dhi=dhi,
                heads=kv_heads * group, kv_heads=kv_heads, dim=dim, block=block, order=order, parts=parts,
                layers=rng.choice([1, 2]), dtype=dtype, tree="chain" if dhi == 1 else rng.choice(["tree", "holes", "chain"]),
                rejected=1 if reqs > 3 and rng.random() < 0.3 else 0)


def _lengths(case, lo, hi, what):
    r = random.Random(what + repr(sorted((k, v) for k, v in case.items() if k != "name")))
    return np.array([r.randint(case[lo], case[hi]) for _ in range(case["reqs"])], np.int64)


def _ceil(a, b):
    return -(-a // b)


def _geometry(case, blocks):
    """Strides, in elements, of a cache of `blocks` blocks: chunks are a power of two, as the paged calls have them."""
    heads, dim, block = case["kv_heads"], case["dim"], case["block"]
    plane = heads * block * dim
    token, head = (dim, block * dim) if case["order"] == "head" else (heads * dim, dim)
    chunk = 1 << (plane * (1 if case["parts"] == 2 else 2) - 1).bit_length()
    v_off = chunk if case["parts"] == 2 else plane
    block_stride = chunk * case["parts"]
    return dict(token=token, head=head, chunk=chunk, v_off=v_off, block=block_stride, layer=block_stride * blocks,
                size=block_stride * blocks * case["layers"])


def _cache(case, blocks, gen):
    g = _geometry(case, blocks)
    data = torch.empty(g["size"], dtype=_DTYPES[case["dtype"]], device=DEVICE).normal_(generator=gen)
    shape = (case["layers"], blocks, case["block"], case["kv_heads"], case["dim"])
    strides = (g["layer"], g["block"], g["token"], g["head"], 1)
    return data, g, torch.as_strided(data, shape, strides, 0), torch.as_strided(data, shape, strides, g["v_off"])


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.uint32).view(np.int32).copy()).to(DEVICE)


def _tables(lens, block, width, blocks, rs):
    """Every request's blocks at scattered places; entries past its last block are left over (-1)."""
    have = _ceil(lens, block)
    tab = np.full((len(lens), width), -1, np.int64)
    ids = rs.permutation(blocks)
    tab[np.arange(width)[None, :] < have[:, None]] = ids[:have.sum()]
    return tab, ids[have.sum():]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 32))
    n, block = case["reqs"], case["block"]
    users = rs.randint(0, max(2, n // 2), n)
    if case["kind"] == "tables":
        lens, new = _lengths(case, "lo", "hi", "l"), _lengths(case, "nlo", "nhi", "n")
        have, want = _ceil(lens, block), _ceil(lens + new, block)
        width = int(want.max()) + 3
        blocks = int(want.sum()) + 64
        tab, free = _tables(lens, block, width, blocks, rs)
        free = free[:max(0, int((want - have).sum()) + case["spare"])]
        labels = np.full(blocks, _LABEL_UNOWNED, np.int64)
        cached = np.arange(width)[None, :] < have[:, None]
        labels[tab[cached]] = np.broadcast_to(users[:, None], tab.shape)[cached]
        for b in rs.permutation(n)[:case["mixed"]]:  # tables that name a block of another user
            if have[b]:
                labels[tab[b, rs.randint(0, have[b])]] = users[b] + 1
        rows = int(new.sum())
        return dict(case=case, users=_i32(users), lens=_i32(lens), new=_i32(new), tables=_i32(tab), free=_i32(free),
                    labels=_i32(labels), slots=torch.zeros(rows, dtype=torch.int64, device=DEVICE),
                    row_begin=torch.zeros(n + 1, dtype=torch.int32, device=DEVICE),
                    lens_out=torch.zeros(n, dtype=torch.int32, device=DEVICE),
                    taken=torch.zeros(1, dtype=torch.int32, device=DEVICE),
                    verdicts=torch.zeros(n, dtype=torch.int32, device=DEVICE))
    if case["kind"] == "append":
        new = _lengths(case, "nlo", "nhi", "n")
        rows = int(new.sum())
        have = _ceil(new, block)
        blocks = max(1, int(have.sum()))
        data, geo, kview, vview = _cache(case, blocks, gen)
        tab, _ = _tables(new, block, max(1, int(have.max())), blocks, rs)
        pos = np.concatenate([np.arange(x) for x in new]) if rows else np.zeros(0, np.int64)
        req = np.repeat(np.arange(n), new)
        slots = tab[req, pos // block] * block + pos % block
        slots[rs.rand(rows) < 0.02] = -1  # rows of requests that were refused
        per = case["drafted"]
        src = n * per if per else rows
        index = None
        if per:  # the accepted path goes down the request's drafted rows
            index = _i32(req * per + (pos * max(1, per // max(1, int(new.max())))))
        shape = (case["layers"], src, case["kv_heads"], case["dim"])
        # K and V as a model has them after the projection: one buffer of [row][K heads, V heads]
        kv = torch.empty(case["layers"], src, 2 * case["kv_heads"], case["dim"], dtype=data.dtype, device=DEVICE)
        kv.normal_(generator=gen)
        k, v = kv[:, :, :case["kv_heads"]], kv[:, :, case["kv_heads"]:]
        assert k.shape == shape
        return dict(case=case, data=data, geo=geo, blocks=blocks, kview=kview, vview=vview, k=k, v=v, index=index,
                    slots=torch.from_numpy(slots).to(DEVICE))
    lens, drafts = _lengths(case, "lo", "hi", "l"), _lengths(case, "dlo", "dhi", "d")
    have = _ceil(lens, block)
    blocks = max(1, int(have.sum()) + int(have.sum()) // 20)
    width = max(1, int(have.max()))
    data, geo, kview, vview = _cache(case, blocks, gen)
    tab, _ = _tables(lens, block, width, blocks, rs)
    rows, words = int(drafts.sum()), max(1, _ceil(int(drafts.max()), 32))
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    qkv = torch.empty(rows, heads + 2 * kv_heads, dim, dtype=data.dtype, device=DEVICE).normal_(generator=gen)
    qkv[:, :heads] *= 1.5  # scores of a few units: some keys count far more than others
    mask = None
    if case["tree"] != "chain":
        bits = np.zeros((rows, 32 * words), np.uint8)
        row = 0
        for d in drafts:
            for i in range(d):  # a drafted token sees its parent's tokens and itself
                if i:
                    bits[row + i] = bits[row + rs.randint(max(0, i - 8), i)]
                bits[row + i, i] = 1
            row += d
        if case["tree"] == "holes":
            bits[rs.rand(rows) < 0.2] = 0
        mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32).copy()).to(DEVICE)
    verdicts = np.zeros(n, np.int64)
    verdicts[rs.permutation(n)[:case["rejected"]]] = _MIXED
    return dict(case=case, data=data, geo=geo, blocks=blocks, kview=kview, vview=vview, tables=_i32(tab), lens=_i32(lens),
                longest=int(lens.max()), most=int(drafts.max()), row_begin=_i32(np.concatenate([[0], np.cumsum(drafts)])),
                q=qkv[:, :heads], k=qkv[:, heads:heads + kv_heads], v=qkv[:, heads + kv_heads:], mask=mask,
                verdicts=_i32(verdicts), out=torch.empty(rows, heads, dim, dtype=data.dtype, device=DEVICE),
                lse=torch.empty(rows, heads, dtype=torch.float32, device=DEVICE), layer=case["layers"] - 1)


_kept = {}


def _attention_work():
    """The attention's workspace: a program makes it once for each stream and keeps it."""
    from paper_2608_25431_amd import gift
    if "work" not in _kept:
        _kept["work"] = gift.AttentionWork()
    return _kept["work"]


def _described(s):
    """The cache as the framework's calls take it."""
    from paper_2608_25431_amd import gift
    c, g = s["case"], s["geo"]
    kv = gift.paged_kv(s["data"], 2 * g["size"], 2 * g["layer"], 2 * g["block"], 2 * g["chunk"], 2 * g["chunk"], c["layers"],
                       c["parts"], s["blocks"])
    fmt = gift.kv_format(s["data"].dtype, c["kv_heads"], c["dim"], c["block"], token_stride=2 * g["token"],
                         head_stride=2 * g["head"], v_offset=2 * g["v_off"])
    return gift, kv, fmt


def run(state):
    s = state
    kind = s["case"]["kind"]
    if kind == "tables":
        if own:
            from paper_2608_25431_amd import gift
            gift.kv_tables(s["users"], s["lens"], s["new"], s["case"]["block"], s["free"], s["tables"], s["labels"],
                           s["slots"], s["row_begin"], s["lens_out"], s["taken"], s["verdicts"])
        else:
            _plain_tables(s)
        return {k: s[k] for k in ("tables", "labels", "slots", "row_begin", "lens_out", "taken", "verdicts")}
    if kind == "append":
        if own:
            gift, kv, fmt = _described(s)
            gift.kv_append(kv, fmt, s["slots"], s["k"], s["v"], index=s["index"])
        else:
            _plain_append(s)
        return s["data"]
    if own:
        gift, kv, fmt = _described(s)
        gift.tree_attention(_attention_work(), kv, fmt, s["layer"], s["q"], s["k"], s["v"], s["row_begin"], s["lens"],
                            s["tables"], s["out"], mask=s["mask"], verdicts=s["verdicts"], lse=s["lse"])
    else:
        _plain_attention(s)
    return {"out": s["out"], "lse": s["lse"]}


def _plain_tables(s):
    block, tab, labels = s["case"]["block"], s["tables"], s["labels"]
    n, width = tab.shape
    lens, new, users = s["lens"].long(), s["new"].long(), s["users"]
    have, want = (lens + block - 1) // block, (lens + new + block - 1) // block
    fits = want <= width
    need = torch.where(fits, want - have, 0)
    upto = need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= s["free"].numel()))
    col = torch.arange(width, device=tab.device)[None, :]
    cached = col < have[:, None]
    inside = (tab >= 0) & (tab < labels.numel())
    right = inside & (labels[torch.where(inside, tab, 0).long()] == users[:, None])
    mixed = (cached & ~right).any(1)
    added = (col >= have[:, None]) & (col < want[:, None]) & ok[:, None]
    at = (upto - need)[:, None] + col - have[:, None]
    if s["free"].numel():
        tab.copy_(torch.where(added, s["free"][at.clamp(0, s["free"].numel() - 1)], tab))
    labels[tab[added].long()] = users[:, None].expand(n, width)[added]
    verdict = torch.where(mixed, _MIXED, torch.where(ok, _OK, _NO_SPACE))
    s["verdicts"].copy_(verdict)
    s["lens_out"].copy_(torch.where(verdict == _OK, lens + new, lens))
    s["taken"].copy_(torch.where(ok, upto, 0).amax())
    s["row_begin"][1:] = new.cumsum(0)
    row = torch.arange(s["slots"].numel(), device=tab.device)
    req = torch.searchsorted(s["row_begin"][1:], row.int(), right=True).clamp(max=n - 1)
    pos = lens[req] + row - s["row_begin"][req]
    slot = tab[req, (pos // block).clamp(max=width - 1)].long() * block + pos % block
    s["slots"].copy_(torch.where(verdict[req] == _OK, slot, -1))


def _plain_append(s):
    slots, block, index = s["slots"], s["case"]["block"], s["index"]
    rows = torch.nonzero(slots >= 0)[:, 0]
    to = slots[rows]
    src = rows if index is None else index[rows].long()
    s["kview"][:, to // block, to % block] = s["k"][:, src]
    s["vview"][:, to // block, to % block] = s["v"][:, src]


def _plain_attention(s):
    c = s["case"]
    n, block, heads, kv_heads, dim = c["reqs"], c["block"], c["heads"], c["kv_heads"], c["dim"]
    group, longest, most = heads // kv_heads, s["longest"], s["most"]
    lens, first = s["lens"].long(), s["row_begin"].long()
    count = first[1:] - first[:-1]
    total = s["q"].shape[0]
    s["out"].zero_()
    s["lse"].fill_(-math.inf)
    if total == 0:
        return
    i = torch.arange(most, device=DEVICE)
    rows = (first[:-1, None] + i).clamp(max=total - 1)
    valid = i < count[:, None]
    ids = s["tables"][:, :_ceil(longest, block)].clamp(min=0).long()

    def keys(cached, drafted):
        a = cached[s["layer"]][ids].reshape(n, -1, kv_heads, dim)[:, :longest].float()
        a = torch.where((torch.arange(longest, device=DEVICE) < lens[:, None])[:, :, None, None], a, 0)
        b = torch.where(valid[:, :, None, None], drafted[rows].float(), 0)
        return torch.cat([a, b], 1).permute(0, 2, 1, 3)

    k, v = keys(s["kview"], s["k"]), keys(s["vview"], s["v"])
    q = s["q"][rows].float().reshape(n, most, kv_heads, group, dim).permute(0, 2, 1, 3, 4).reshape(n, kv_heads, -1, dim)
    scores = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(dim)
    if s["mask"] is None:
        among = (i[None, :] <= i[:, None])[None].expand(n, most, most)
    else:
        among = (s["mask"][rows][:, :, i // 32] >> (i % 32)) & 1 == 1
    among = among & valid[:, None, :]
    past = (torch.arange(longest, device=DEVICE) < lens[:, None])[:, None].expand(n, most, longest)
    allowed = torch.cat([past, among], 2)[:, None, :, None].expand(n, kv_heads, most, group, longest + most)
    scores = torch.where(allowed.reshape(scores.shape), scores, -math.inf)
    top = scores.amax(3, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0, top))
    total_p = p.sum(3, keepdim=True)
    out = torch.where(total_p > 0, torch.matmul(p, v) / total_p, 0)
    lse = top[..., 0] + torch.log(total_p[..., 0])
    good = valid & (s["verdicts"] == _OK)[:, None]
    out = out.reshape(n, kv_heads, most, group, dim).permute(0, 2, 1, 3, 4).reshape(n, most, heads, dim)
    lse = lse.reshape(n, kv_heads, most, group).permute(0, 2, 1, 3).reshape(n, most, heads)
    s["out"][rows[good]] = out[good].to(s["out"].dtype)
    s["lse"][rows[good]] = lse[good]


def work(case):
    c = case
    if c["kind"] == "tables":
        lens, new = _lengths(c, "lo", "hi", "l"), _lengths(c, "nlo", "nhi", "n")
        have, want = _ceil(lens, c["block"]), _ceil(lens + new, c["block"])
        return {"bytes": int(28 * c["reqs"] + 8 * have.sum() + 12 * (want - have).sum() + 8 * new.sum()), "flops": 0}
    if c["kind"] == "append":
        rows = int(_lengths(c, "nlo", "nhi", "n").sum())
        return {"bytes": max(1, 2 * rows * c["layers"] * c["kv_heads"] * c["dim"] * 2 * 2 + 12 * rows), "flops": 0}
    lens, drafts = _lengths(c, "lo", "hi", "l"), _lengths(c, "dlo", "dhi", "d")
    reads = np.where(drafts > 0, lens, 0)  # a request without rows reads nothing
    rows = int(drafts.sum())
    size = 2 * c["dim"] * (2 * c["kv_heads"] * int(reads.sum()) + rows * (2 * c["heads"] + 2 * c["kv_heads"]))
    return {"bytes": max(1, size + 4 * rows * c["heads"] + 4 * int(_ceil(reads, c["block"]).sum())),
            "flops": int(4 * c["dim"] * c["heads"] * (drafts * (lens + drafts)).sum())}


def exact(case, seed):
    if case["kind"] == "tables":
        return None
    s = prepare(case, seed)
    if case["kind"] == "append":
        # token rows of the cache, one after the other in a copy in 64 bits
        flat, g, slots = s["data"].double(), s["geo"], s["slots"].cpu().numpy()
        index = None if s["index"] is None else s["index"].cpu().numpy()
        live = np.nonzero(slots >= 0)[0]
        from_row = torch.from_numpy(np.asarray(live if index is None else index[live], np.int64)).to(DEVICE)
        b, t = slots[live] // case["block"], slots[live] % case["block"]
        start = torch.from_numpy(b * g["block"] + t * g["token"]).to(DEVICE)
        lane = torch.arange(case["dim"], device=DEVICE)
        for layer in range(case["layers"]):
            for h in range(case["kv_heads"]):
                at = start[:, None] + lane + (layer * g["layer"] + h * g["head"])
                flat[at] = s["k"][layer, from_row, h].double()
                flat[at + g["v_off"]] = s["v"][layer, from_row, h].double()
        return flat
    lens, first, tab = s["lens"].tolist(), s["row_begin"].tolist(), s["tables"].cpu().numpy()
    rejected, group, block = s["verdicts"].tolist(), case["heads"] // case["kv_heads"], case["block"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEVICE)
    for b in range(case["reqs"]):
        lo, hi, length = first[b], first[b + 1], lens[b]
        if lo == hi or rejected[b]:
            continue
        pos = np.arange(length)
        blk = torch.from_numpy(tab[b, pos // block].astype(np.int64)).to(DEVICE)
        off = torch.from_numpy(pos % block).to(DEVICE)
        drafted = np.tril(np.ones((hi - lo, hi - lo), bool))
        if s["mask"] is not None:
            words = np.ascontiguousarray(s["mask"][lo:hi].cpu().numpy()).view(np.uint8)
            drafted = np.unpackbits(words, axis=1, bitorder="little")[:, :hi - lo].astype(bool)
        seen = torch.from_numpy(np.concatenate([np.ones((hi - lo, length), bool), drafted], 1)).to(DEVICE)
        for h in range(case["kv_heads"]):
            k = torch.cat([s["kview"][s["layer"], blk, off, h], s["k"][lo:hi, h]]).double()
            v = torch.cat([s["vview"][s["layer"], blk, off, h], s["v"][lo:hi, h]]).double()
            for j in range(h * group, (h + 1) * group):
                z = (s["q"][lo:hi, j].double() @ k.T) * case["dim"] ** -0.5
                z = z.masked_fill(~seen, -math.inf)
                some = seen.any(1)
                lse[lo:hi, j] = torch.logsumexp(z, 1)
                weights = torch.softmax(z[some], 1)
                out[lo:hi, j][some] = weights @ v
    return {"out": out, "lse": lse}
