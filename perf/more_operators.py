"""Cases and plain forms of the operators of a decoding step over a paged KV pool.

append   new tokens' keys and values go to the pages of their sequences; queries and keys are normalised head by head
         and rotated by their positions (one or several axes) on the way
form     attention of the newest tokens over the paged pool in another form than plain causal: a mask among the newest
         tokens (drafted trees, documents, a prefix seen both ways), scores capped by a tanh, a bias by distance
accept   the accepted path of a drafted tree stays: its keys and values move, in every layer, to the place behind the
         tokens before the tree

With ``own`` false the operators run in their plain form (elementary torch operations in 32 bits, angles in 64); with
``own`` true ``run`` makes the calls that a user of the package makes.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK_MAJOR, LAYER_MAJOR = 0, 1     # [block][layer][K/V][token][head][dim], [layer][K/V][block][head][token][dim]

# new: newest tokens of a sequence at most; ragged: each sequence has its own number of them, from 1
_DEFAULTS = dict(op="form", layers=2, heads=8, group=4, dim=128, block=128, layout=LAYER_MAJOR, dtype="bf16", n=32, lens="fixed", lo=1, hi=2048,
                 len_seed=0, new=1, ragged=False, prefixes=0, prefix_len=0,
                 rotated=128, base=500000.0, adjacent=False, axes=1, norm=False, packed=False,
                 mask="causal", cap=0.0, slopes=False)


def _case(**kw):
    return {**_DEFAULTS, **kw}


def listed():
    return [
        # one decoding step of an 8B-shaped batch: 64 tokens
        _case(name="append-decode", op="append", n=64),
        # ragged prompts of an 8B-shaped batch, heads normalised, into the prefill side's blocks of 16 tokens
        _case(name="append-prompts", op="append", n=8, lens="uniform", lo=300, hi=4096, new=4096, packed=True, norm=True, block=16, layout=BLOCK_MAJOR, len_seed=21),
        # a few drafted tokens a sequence, heads that are not Llama-shaped and rotated in part, by adjacent pairs
        _case(name="append-odd", op="append", heads=5, group=3, dim=80, rotated=32, adjacent=True, base=10000.0, n=23, lens="uniform", lo=37, hi=1999, block=24,
              layout=BLOCK_MAJOR, dtype="fp16", new=4, ragged=True, packed=True, len_seed=23),
        # prompts with images: positions in time, height and width
        _case(name="append-images", op="append", heads=4, group=7, n=4, lens="uniform", lo=900, hi=1500, new=1300, packed=True, norm=True, axes=3, base=1000000.0, len_seed=25),
        # one short request on a small geometry, a tree of 8 drafted tokens: the latency of a call
        _case(name="tree-one-short", heads=4, group=2, dim=64, block=32, n=1, hi=300, new=8, mask="tree"),
        # trees of 64 drafted tokens over an 8B-shaped batch: 256 rows a KV head
        _case(name="tree-8b", n=16, hi=2048, new=64, mask="tree"),
        # ragged trees on a geometry that is not Llama-shaped
        _case(name="tree-odd-ragged", heads=5, group=3, dim=80, block=24, layout=BLOCK_MAJOR, dtype="fp16", n=23, lens="uniform", lo=37, hi=1999, new=7, ragged=True,
              mask="tree", len_seed=27),
        # decoding of the 8B-shaped uniform batch with capped scores
        _case(name="capped-8b-uniform", cap=50.0),
        # two long contexts, scores biased by distance
        _case(name="biased-long", n=2, lens="uniform", lo=90000, hi=131072, group=8, slopes=True, len_seed=3),
        # chunks of several documents behind a shared prefix, capped scores: the products and the tanh carry the call
        _case(name="capped-documents", n=4, lens="uniform", lo=700, hi=1500, new=256, ragged=True, mask="documents", cap=30.0, prefixes=1, prefix_len=2048, len_seed=29),
        # verification of an 8B-shaped batch done: accepted paths of trees of 32 tokens, all 32 layers
        _case(name="accept-8b", op="accept", layers=32, n=48, hi=60, lo=40, lens="uniform", new=32, ragged=True, block=16, len_seed=31),
        # a small batch on a geometry that is not Llama-shaped
        _case(name="accept-odd", op="accept", layers=5, heads=5, dim=80, block=24, layout=BLOCK_MAJOR, dtype="fp16", n=7, lens="uniform", lo=60, hi=400, new=13, ragged=True,
              len_seed=33),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case, of no more tokens, products and rows than the listed ones."""
    op = rng.choice(["append", "tree", "form", "form", "accept"])
    c = _case(op="form" if op == "tree" else op, layers=rng.choice([1, 2, 3]), heads=rng.choice([1, 2, 4, 5, 8]), group=rng.choice([1, 2, 3, 4, 7, 8]),
              dim=rng.choice([64, 80, 96, 128, 128, 128, 256]), block=rng.choice([16, 24, 32, 64, 100, 128, 256]), layout=rng.choice([BLOCK_MAJOR, LAYER_MAJOR]),
              dtype=rng.choice(["bf16", "fp16"]), len_seed=rng.randrange(1 << 20), lens=rng.choice(["fixed", "uniform", "uniform"]))
    if op == "append":
        c["rotated"] = rng.choice([0, 16, 20, 32, 64, c["dim"], c["dim"], c["dim"]])
        c["adjacent"] = rng.random() < 0.3
        c["axes"] = rng.choice([1, 1, 3]) if c["rotated"] else 1
        c["norm"] = rng.random() < 0.5
        c["base"] = rng.choice([10000.0, 500000.0])
        c["packed"] = rng.random() < 0.5
        c["n"] = _log_uniform(rng, 1, 256)
        rows = 8 * 2000 * 48 * 128 // ((c["group"] + 2) * c["heads"] * c["dim"])
        c["new"] = max(1, _log_uniform(rng, 1, max(2, min(8192, rows // c["n"]))))
        c["ragged"] = c["packed"] and rng.random() < 0.7
        c["hi"] = max(c["new"], min(8192, 2 * c["new"] + rng.randrange(512)))
    elif op == "accept":
        c["n"] = _log_uniform(rng, 1, 48)
        c["new"] = rng.choice([4, 13, 32, 64])
        c["layers"] = rng.choice([1, 4, 16, 32])
        c["ragged"] = rng.random() < 0.7
        c["hi"] = c["new"] + rng.randrange(64)
    else:
        c["mask"] = "tree" if op == "tree" else rng.choice(["causal", "causal", "documents", "prefix"])
        c["new"] = _log_uniform(rng, 2, 96) if c["mask"] != "causal" else rng.choice([1, 1, 1, 2, 5])
        c["ragged"] = c["mask"] != "causal" and rng.random() < 0.6
        if op == "form":
            c["cap"] = rng.choice([0.0, 20.0, 50.0])
            c["slopes"] = c["cap"] == 0.0 or rng.random() < 0.3
        c["n"] = _log_uniform(rng, 1, 64)
        if rng.random() < 0.3:
            c["prefixes"] = rng.choice([1, 1, 3])
            c["prefix_len"] = _log_uniform(rng, 33, 2048)
        cells = 32 * 2048 * 8 * 128                                                       # elements of K
        pairs = 4 * 8 * 1024 * 3000                                                       # logits of the plain form
        row = c["heads"] * c["group"] * c["new"]
        most = min(100000, cells // (c["heads"] * c["dim"] * c["n"]), pairs // (row * c["n"]) - c["prefix_len"] - 100)
        c["hi"] = _log_uniform(rng, 16, max(17, most))
        if most < 17:
            c["prefixes"] = c["prefix_len"] = 0
        c["hi"] = max(c["hi"], c["new"])
    c["lo"] = max(c["new"] if not c["packed"] else 1, 1 + rng.randrange(c["hi"]))
    c["lo"] = min(c["lo"], c["hi"])
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _rng(c, salt):
    return random.Random(c["len_seed"] * 7919 + salt)


def _lens(c):
    rng = _rng(c, 17)
    if c["lens"] == "fixed":
        return [c["hi"]] * c["n"]
    return [rng.randint(c["lo"], c["hi"]) for _ in range(c["n"])]


def _news(c):
    """Newest tokens of each sequence."""
    rng = _rng(c, 41)
    return [min(x, rng.randint(1, c["new"]) if c["ragged"] else c["new"]) for x in _lens(c)]


def _paths(c):
    """Accepted nodes of each tree.  The root stays where it is; further nodes come from behind the accepted places, so
    that a pass can be repeated on its own result."""
    rng = _rng(c, 43)
    out = []
    for m in _news(c):
        depth = max(1, min(rng.randint(1, 6), (m + 1) // 2))
        out.append([0] + sorted(rng.sample(range(depth, m), depth - 1)))
    return out


def _prefix_lens(c):
    return [c["prefix_len"] + 17 * i for i in range(c["prefixes"])]


def _torch_dtype(c):
    return {"bf16": torch.bfloat16, "fp16": torch.float16}[c["dtype"]]


def _shape(layout, layers, heads, dim, block, blocks):
    if layout == BLOCK_MAJOR:
        return (blocks, layers, 2, block, heads, dim)
    return (layers, 2, blocks, heads, block, dim)


def _tables(rng, counts, blocks):
    """Runs of a permutation of the pool's blocks, as CSR."""
    off = np.zeros(len(counts) + 1, np.int64)
    np.cumsum(np.asarray(counts, np.int64), out=off[1:])
    return off, rng.permutation(blocks)[:off[-1]].astype(np.int32)


def _trees(c, rng):
    """Visibility [sequence, node, node] and depth [sequence, node] of the newest tokens; nodes that are not there see nothing."""
    Q, news = c["new"], _news(c)
    see, depth = np.zeros((c["n"], Q, Q), bool), np.zeros((c["n"], Q), np.int32)
    for r, m in enumerate(news):
        if c["mask"] == "tree":
            for i in range(m):
                if i:
                    parent = int(rng.integers(max(0, i - 6), i))
                    see[r, i], depth[r, i] = see[r, parent], depth[r, parent] + 1
                see[r, i, i] = True
            continue
        depth[r, :m] = np.arange(m)
        at = np.arange(m)
        if c["mask"] == "causal":
            see[r, :m, :m] = at[:, None] >= at[None, :]
        elif c["mask"] == "documents":
            cuts = np.sort(rng.integers(0, m, 4))
            doc = (at[:, None] >= cuts[None, :]).sum(1)
            see[r, :m, :m] = (doc[:, None] == doc[None, :]) & (at[:, None] >= at[None, :])
        else:                                                       # the first part is seen both ways
            part = int(rng.integers(0, m))
            see[r, :m, :m] = (at[:, None] >= at[None, :]) | (at[None, :] < part)
    return see, depth


def _frequencies(c):
    pairs = c["rotated"] // 2
    return c["base"] ** (-np.arange(pairs, dtype=np.float64) / max(1, pairs))


def _axis_of_pair(c):
    pairs = c["rotated"] // 2
    return np.repeat(np.arange(3), [pairs - 2 * (3 * pairs // 8), 3 * pairs // 8, 3 * pairs // 8]) if c["axes"] == 3 else np.zeros(pairs, np.int64)


def _inputs(case, seed):
    c = {**_DEFAULTS, **case}
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt = _torch_dtype(c)
    lens, news, p_lens, B, H, G, D = _lens(c), _news(c), _prefix_lens(c), c["block"], c["heads"], c["group"], c["dim"]
    counts = [-(-n // B) for n in p_lens + lens]
    blocks = sum(counts) + max(1, sum(counts) // 16)
    off, tbl = _tables(rng, counts, blocks)
    P = c["prefixes"]
    s = {"case": c, "lens": lens, "news": news, "prefix_lens": p_lens, "member": [i % P if P else -1 for i in range(c["n"])],
         "prefix_off": off[:P + 1], "prefix_tbl": tbl[:off[P]], "off": off[P:] - off[P], "tbl": tbl[off[P]:], "layer": c["layers"] - 1, "blocks": blocks}
    s["pool"] = torch.empty(_shape(c["layout"], c["layers"], H, D, B, blocks), device="cuda", dtype=dt).normal_(generator=gen)
    if c["op"] == "append":
        rows = sum(news) if c["packed"] else c["n"] * c["new"]
        qkv = torch.randn(rows, (G + 2) * H * D, device="cuda", generator=gen).mul_(1.5).to(dt)      # what a fused projection leaves
        parts = [x.unflatten(1, (-1, D)) for x in qkv.split([G * H * D, H * D, H * D], 1)]
        s["q"], s["k"], s["v"] = parts if c["packed"] else [x.unflatten(0, (c["n"], c["new"])) for x in parts]
        s["starts"] = torch.tensor(np.cumsum([0] + news), dtype=torch.int32, device="cuda")
        if c["norm"]:
            s["q_norm"], s["k_norm"] = (1 + 0.2 * torch.randn(2, D, device="cuda", generator=gen)).unbind(0)
        if c["axes"] == 3:
            s["positions"] = torch.randint(0, 3000, (3, rows), device="cuda", generator=gen, dtype=torch.int32)
    elif c["op"] == "form":
        s["q"] = torch.randn(c["n"], c["new"], H * G, D, device="cuda", generator=gen).mul_(4 if c["cap"] else 2).to(dt)
        see, depth = _trees(c, rng)
        s["see"], s["depth"] = torch.from_numpy(see).cuda(), torch.from_numpy(depth).cuda()
        s["news_t"] = torch.tensor(news, dtype=torch.int32, device="cuda")
        if c["slopes"]:
            s["slopes"] = torch.pow(2.0, -8 * (1 + torch.arange(H * G, device="cuda")) / (H * G)).float()
    else:
        paths = _paths(c)
        width = max(len(p) for p in paths)
        s["paths"] = torch.tensor([p + [-1] * (width - len(p)) for p in paths], dtype=torch.int32, device="cuda")
        s["news_t"] = torch.tensor(news, dtype=torch.int32, device="cuda")
    return s


def _slots(lens, off, tbl, block):
    """[request, token]: block * block size + offset; 0 past a request's end."""
    pos = np.arange(max(lens))[None, :]
    at = np.minimum(off[:-1, None] + pos // block, len(tbl) - 1)
    slot = np.where(pos < np.asarray(lens)[:, None], tbl[at].astype(np.int64) * block + pos % block, 0)
    return torch.from_numpy(slot).cuda()


def prepare(case, seed):
    s = _inputs(case, seed)
    c, lens, news, B = s["case"], s["lens"], s["news"], s["case"]["block"]
    if own:
        from paper_2408_08147_b200.sequences import CacheSession, Rotary, Sequences, pack_mask
        from paper_2408_08147_b200.workloads import Geometry

        g = Geometry(c["layout"], c["layers"], c["heads"], c["dim"], 2, B, s["blocks"])
        seqs = Sequences(lens, s["off"], s["tbl"], s["prefix_lens"], s["prefix_off"], s["prefix_tbl"], s["member"])
        s["session"] = CacheSession(g, s["pool"], seqs, num_q_heads=c["heads"] * c["group"], q_tokens=1 if c["op"] == "append" else c["new"], dtype=_torch_dtype(c))
        if c["op"] == "append":
            s["rotary"] = Rotary(c["rotated"], frequencies=_frequencies(c), adjacent=c["adjacent"], axes=_axis_of_pair(c) if c["axes"] == 3 else None) if c["rotated"] else None
        elif c["op"] == "form":
            s["mask"] = pack_mask(s["see"]) if c["mask"] != "causal" else None
        return s
    # where each token lies (padded to the longest request): what a program without the operators keeps
    s["len_t"], s["slots"] = torch.tensor(lens, device="cuda"), _slots(lens, s["off"], s["tbl"], B)
    first = [n - m for n, m in zip(lens, news)]
    if c["op"] == "append":
        s["sequence"] = torch.from_numpy(np.repeat(np.arange(c["n"]), news)).cuda()
        s["place"] = torch.from_numpy(np.concatenate([f + np.arange(m) for f, m in zip(first, news)])).cuda()
        s["frequencies"], s["axis"] = torch.from_numpy(_frequencies(c)).cuda(), torch.from_numpy(_axis_of_pair(c)).cuda()
    elif c["op"] == "form":
        s["first"] = torch.tensor(first, device="cuda")
        if c["prefixes"]:
            s["prefix_len_t"] = torch.tensor(s["prefix_lens"], device="cuda")
            s["prefix_slots"] = _slots(s["prefix_lens"], s["prefix_off"], s["prefix_tbl"], B)
    else:
        s["first"] = torch.tensor(first, device="cuda")
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        session = state["session"]
        if c["op"] == "append":
            q = session.append(state["layer"], state["k"], state["v"], state["q"], rotary=state["rotary"], position_t=state.get("positions"), q_norm_t=state.get("q_norm"),
                               k_norm_t=state.get("k_norm"), row_begin_t=state["starts"] if c["packed"] else None)
            return {"q": q, "pool": state["pool"]}
        if c["op"] == "accept":
            return {"lens": session.accept(state["paths"], n_new_t=state["news_t"]), "pool": state["pool"]}
        out, lse = session.attend(state["layer"], state["q"], cap=c["cap"] or None, slopes_t=state.get("slopes"), mask_t=state["mask"],
                                  n_new_t=state["news_t"] if c["ragged"] else None, offset_t=state["depth"] if c["slopes"] and c["mask"] == "tree" else None)
        return {"out": out, "lse": lse}
    return {"append": _plain_append, "form": _plain_form, "accept": _plain_accept}[c["op"]](state)


def _plane(pool, layout, layer, kv):
    """One layer's keys or values as [block, token, head, dim]."""
    return pool[:, layer, kv] if layout == BLOCK_MAJOR else pool[layer, kv].transpose(1, 2)


def _rows(plane, slots, block):
    """[request, head, token, dim] in 32 bits of the given slots."""
    return plane[slots // block, slots % block].transpose(1, 2).float()


def _rotate(x, cos, sin, c):
    R = c["rotated"]
    if c["adjacent"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., R:]], -1)


def _plain_append(s):
    c = s["case"]
    q, k, v = (x if c["packed"] else x.flatten(0, 1) for x in (s["q"], s["k"], s["v"]))
    if c["axes"] == 3:
        position = s["positions"][s["axis"]].T.double()                          # [token, pair]
    else:
        position = s["place"].double()[:, None]
    angle = position * s["frequencies"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    q, k = q.float(), k.float()
    if c["norm"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + 1e-6) * s["q_norm"]
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + 1e-6) * s["k_norm"]
    q, k = _rotate(q, cos, sin, c).to(v.dtype), _rotate(k, cos, sin, c).to(v.dtype)
    at = s["slots"][s["sequence"], s["place"]]
    _plane(s["pool"], c["layout"], s["layer"], 0)[at // c["block"], at % c["block"]] = k
    _plane(s["pool"], c["layout"], s["layer"], 1)[at // c["block"], at % c["block"]] = v
    return {"q": q.view(s["q"].shape), "pool": s["pool"]}


def _plain_form(s):
    c = s["case"]
    n, H, G, D, Q, P = c["n"], c["heads"], c["group"], c["dim"], c["new"], c["prefixes"]
    k_all, v_all = (_plane(s["pool"], c["layout"], s["layer"], kv) for kv in (0, 1))
    q = s["q"].float().view(n, Q, H, G, D).permute(0, 2, 1, 3, 4).reshape(n, H, Q * G, D) / math.sqrt(D)
    W = s["slots"].shape[1]
    logits = torch.matmul(q, _rows(k_all, s["slots"], c["block"]).transpose(2, 3))            # [request, head, row, token]
    pos = torch.arange(W, device="cuda")
    newest = (pos[None, :] - s["first"][:, None]).clamp(0, Q - 1)                             # [request, token]
    old = pos[None, :] < s["first"][:, None]
    there = torch.arange(Q, device="cuda")[None, :] < s["news_t"][:, None]                    # [request, query]
    seen = old[:, None, :] | torch.gather(s["see"], 2, newest[:, None, :].expand(n, Q, W)) & (pos[None, :] < s["len_t"][:, None])[:, None, :]
    seen = (seen & there[:, :, None])[:, None, :, None, :]
    if P:
        # requests of one prefix side by side, so that its keys are multiplied once; request i has prefix i % P
        M = -(-n // P)
        grouped = torch.zeros(M * P, H, Q * G, D, device="cuda")
        grouped[:n] = q
        grouped = grouped.view(M, P, H, Q * G, D).permute(1, 2, 0, 3, 4).reshape(P, H, M * Q * G, D)
        over = torch.matmul(grouped, _rows(k_all, s["prefix_slots"], c["block"]).transpose(2, 3))
        wide = over.shape[-1]
        over = over.view(P, H, M, Q * G, wide).permute(2, 0, 1, 3, 4).reshape(M * P, H, Q * G, wide)[:n]
        logits = torch.cat([logits, over], -1)
        p_len = s["prefix_len_t"].repeat(M)[:n]
        p_pos = torch.arange(wide, device="cuda")
        p_seen = (p_pos[None, :] < p_len[:, None])[:, None, :] & there[:, :, None]
        seen = torch.cat([seen, p_seen[:, None, :, None, :]], -1)
    logits = logits.view(n, H, Q, G, -1)
    if c["cap"]:
        logits = c["cap"] * torch.tanh(logits / c["cap"])
    if c["slopes"]:
        key = torch.where(old, pos[None, :], s["first"][:, None] + torch.gather(s["depth"].long(), 1, newest))
        query = s["first"][:, None] + s["depth"]
        away = (key[:, None, :] - query[:, :, None]).float()
        if P:
            away = torch.cat([away, (p_pos[None, None, :] - (query + p_len[:, None])[:, :, None]).float()], -1)
        logits = logits + s["slopes"].view(1, H, 1, G, 1) * away[:, None, :, None, :]
    logits = logits.masked_fill(~seen, -math.inf).view(n, H, Q * G, -1)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - top.masked_fill(top == -math.inf, 0.0))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p[..., :W], _rows(v_all, s["slots"], c["block"]))
    if P:
        weights = torch.zeros(M * P, H, Q * G, wide, device="cuda")
        weights[:n] = p[..., W:]
        weights = weights.view(M, P, H, Q * G, wide).permute(1, 2, 0, 3, 4).reshape(P, H, M * Q * G, wide)
        op = torch.matmul(weights, _rows(v_all, s["prefix_slots"], c["block"]))
        o += op.view(P, H, M, Q * G, D).permute(2, 0, 1, 3, 4).reshape(M * P, H, Q * G, D)[:n]
    lse = (top + torch.log(total)).view(n, H, Q, G).permute(0, 2, 1, 3).reshape(n, Q, H * G)
    out = torch.where(total > 0, o / total, 0.0).view(n, H, Q, G, D).permute(0, 2, 1, 3, 4).reshape(n, Q, H * G, D).to(s["q"].dtype)
    return {"out": out, "lse": lse}


def _plain_accept(s):
    c = s["case"]
    held = s["paths"] >= 0
    r, j = held.nonzero(as_tuple=True)
    at = s["slots"][r, s["first"][r] + s["paths"][r, j]]
    to = s["slots"][r, s["first"][r] + j]
    B = c["block"]
    if c["layout"] == BLOCK_MAJOR:
        s["pool"][to // B, :, :, to % B] = s["pool"][at // B, :, :, at % B]
    else:
        s["pool"][:, :, to // B, :, to % B] = s["pool"][:, :, at // B, :, at % B]
    return {"lens": (s["first"] + held.sum(1)).int(), "pool": s["pool"]}


# ---------------------------------------------------------------------------
# the least a pass has to do, and what it has to give
# ---------------------------------------------------------------------------

def work(case):
    c = {**_DEFAULTS, **case}
    lens, news, p_lens = _lens(c), _news(c), _prefix_lens(c)
    H, G, D = c["heads"], c["group"], c["dim"]
    if c["op"] == "append":
        values = sum(news) * (G + 2) * H * D
        return {"bytes": 4 * values + 4 * c["axes"] * sum(news) * (c["axes"] > 1), "flops": 10 * values}
    if c["op"] == "accept":
        moved = sum(sum(x != j for j, x in enumerate(p)) for p in _paths(c))
        return {"bytes": 2 * 2 * 2 * c["layers"] * H * D * moved + 12 * c["n"], "flops": c["n"]}
    used = sum(p_lens[:c["n"]])
    size = 2 * 2 * H * D * (sum(lens) + used) + sum(news) * H * G * 2 * D + c["n"] * c["new"] * H * G * (2 * D + 4)
    if c["mask"] != "causal":
        size += sum(news) * -(-c["new"] // 32) * 4
    pairs = sum(m * (n + (p_lens[i % c["prefixes"]] if c["prefixes"] else 0)) for i, (m, n) in enumerate(zip(news, lens)))
    return {"bytes": size, "flops": 4 * D * H * G * pairs}


def exact(case, seed):
    s = _inputs(case, seed)
    return {"append": _exact_append, "form": _exact_form, "accept": _exact_accept}[s["case"]["op"]](s, s["case"])


def _where(c, off, tbl, r, tokens):
    """(block, offset) of the given tokens of one list."""
    t = torch.as_tensor(tbl[off[r]:off[r + 1]].astype(np.int64), device="cuda")
    return t[tokens // c["block"]], tokens % c["block"]


def _exact_append(s, c):
    H, G, D, R = c["heads"], c["group"], c["dim"], c["rotated"]
    pool = s["pool"].double()
    q_out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda").flatten(0, -3)
    q_in, k_in, v_in = (x.flatten(0, -3).double() for x in (s["q"], s["k"], s["v"]))
    freq = torch.tensor([c["base"] ** (-2.0 * i / R) for i in range(R // 2)], dtype=torch.float64, device="cuda")
    axis = torch.as_tensor(_axis_of_pair(c), device="cuda")

    def turned(x, w, position):                                     # x: [token, head, dim], position: [token, pair]
        if c["norm"]:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + 1e-6) * w.double()
        pairs = torch.arange(R // 2, device="cuda")
        a_at, b_at = (2 * pairs, 2 * pairs + 1) if c["adjacent"] else (pairs, pairs + R // 2)
        z = torch.polar(torch.ones_like(position), position * freq)[:, None] * torch.complex(x[..., a_at], x[..., b_at])
        y = x.clone()
        y[..., a_at], y[..., b_at] = z.real, z.imag
        return y

    row = 0
    for r, (n, m) in enumerate(zip(s["lens"], s["news"])):
        at = torch.arange(n - m, n, device="cuda")
        mine = slice(row, row + m)
        position = s["positions"][:, mine].double()[axis].T if c["axes"] == 3 else at.double()[:, None].expand(m, R // 2)
        q_out[mine] = turned(q_in[mine], s.get("q_norm"), position)
        k = turned(k_in[mine], s.get("k_norm"), position)
        blk, tt = _where(c, s["off"], s["tbl"], r, at)
        for kv, x in ((0, k), (1, v_in[mine])):
            if c["layout"] == BLOCK_MAJOR:
                pool[blk, s["layer"], kv, tt] = x
            else:
                pool[s["layer"], kv, blk, :, tt] = x
        row += m
    return {"q": q_out.view(s["q"].shape), "pool": pool}


def _token(pool, c, layer, kv, blk, tt):
    """[token, head, dim] of the tokens at (blk, tt), in 64 bits."""
    if c["layout"] == BLOCK_MAJOR:
        return pool[blk, layer, kv, tt].double()
    return pool[layer, kv, blk, :, tt].double()


def _exact_form(s, c):
    H, G, D, Q, n = c["heads"], c["group"], c["dim"], c["new"], c["n"]
    if n * H > 2000:
        return None
    out = torch.zeros(n, Q, H * G, D, dtype=torch.float64, device="cuda")
    lse = torch.full((n, Q, H * G), -math.inf, dtype=torch.float64, device="cuda")
    for r, (length, m) in enumerate(zip(s["lens"], s["news"])):
        P = s["prefix_lens"][s["member"][r]] if s["member"][r] >= 0 else 0
        parts = []
        if P:
            parts.append(_where(c, s["prefix_off"], s["prefix_tbl"], s["member"][r], torch.arange(P, device="cuda")))
        parts.append(_where(c, s["off"], s["tbl"], r, torch.arange(length, device="cuda")))
        k = torch.cat([_token(s["pool"], c, s["layer"], 0, *w) for w in parts])
        v = torch.cat([_token(s["pool"], c, s["layer"], 1, *w) for w in parts])
        before = P + length - m
        hidden = torch.zeros(m, P + length, dtype=torch.bool, device="cuda")
        hidden[:, before:] = ~s["see"][r, :m, :m]
        depth = s["depth"][r, :m].double()
        away = torch.cat([torch.arange(before, device="cuda").double(), before + depth])[None, :] - (before + depth)[:, None]
        for h in range(H):
            x = s["q"][r, :m, h * G:(h + 1) * G].double()                            # [query, g, dim]
            z = torch.einsum("igd,td->igt", x, k[:, h]) / math.sqrt(D)
            if c["cap"]:
                z = torch.tanh(z / c["cap"]) * c["cap"]
            if c["slopes"]:
                z = z + s["slopes"][h * G:(h + 1) * G].double()[None, :, None] * away[:, None, :]
            z = z.masked_fill(hidden[:, None, :], -math.inf)
            norm = torch.logsumexp(z, -1)
            w = torch.exp(z - norm[..., None]).nan_to_num(0.0)
            out[r, :m, h * G:(h + 1) * G] = torch.einsum("igt,td->igd", w, v[:, h])
            lse[r, :m, h * G:(h + 1) * G] = norm
    return {"out": out, "lse": lse}


def _exact_accept(s, c):
    pool = s["pool"].double()
    lens = []
    for r, (path, n, m) in enumerate(zip(_paths(c), s["lens"], s["news"])):
        first = n - m
        blk, tt = _where(c, s["off"], s["tbl"], r, first + torch.tensor(path, device="cuda"))
        b2, t2 = _where(c, s["off"], s["tbl"], r, first + torch.arange(len(path), device="cuda"))
        if c["layout"] == BLOCK_MAJOR:
            pool[b2, :, :, t2] = pool[blk, :, :, tt].clone()
        else:
            pool[:, :, b2, :, t2] = pool[:, :, blk, :, tt].clone()
        lens.append(first + len(path))
    return {"lens": torch.tensor(lens), "pool": pool}
