"""Cases and plain forms of the operators that read, weigh and shrink a paged KV pool.

attend   attention of the newest tokens of a batch over the paged pool; requests that share a
         long prompt prefix share the blocks that hold it
weigh    the same call, which also adds the attention weight that every cached token of a
         request receives to a running score per (request, KV head, token)
evict    keeps the heaviest tokens of every (layer, request, KV head) and moves their keys and
         values, in order, into the blocks of another pool; the scores move with them

With ``own`` false the operators run in their plain form (elementary torch operations in 32
bits); with ``own`` true ``run`` makes the calls that a user of the package makes.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK_MAJOR, LAYER_MAJOR = 0, 1     # [block][layer][K/V][token][head][dim], [layer][K/V][block][head][token][dim]

_DEFAULTS = dict(op="attend", layers=2, heads=8, group=4, dim=128, block=128, layout=LAYER_MAJOR, dtype="bf16", q_tokens=1,
                 n=32, lens="fixed", lo=1, hi=2048, len_seed=0, prefixes=0, prefix_len=0,
                 budget=0, sink=0, recent=0, dst_block=128, dst_layout=LAYER_MAJOR)


def _case(**kw):
    return {**_DEFAULTS, **kw}


def listed():
    return [
        # one short request on a small geometry: the latency of a call
        _case(name="attend-one-short", op="attend", heads=4, group=2, dim=64, n=1, lens="fixed", hi=300, block=32),
        # 8B-shaped batch of the uniform benchmark, 32 x 2048 tokens
        _case(name="attend-8b-uniform", op="attend", n=32, lens="fixed", hi=2048),
        # 8B-shaped batch with lognormal prompt lengths, read where prefill left it: 16-token block-major blocks
        _case(name="attend-8b-lognormal", op="attend", n=64, lens="lognormal", lo=16, hi=8192, block=16, layout=BLOCK_MAJOR, dtype="fp16"),
        # two long contexts with 70B-shaped heads: few rows, the work lies along the tokens
        _case(name="attend-long", op="attend", n=2, lens="uniform", lo=90000, hi=131072, group=8, len_seed=3),
        # verification of four drafted tokens on a geometry that is not Llama-shaped
        _case(name="attend-odd-verify", op="attend", heads=5, group=3, dim=80, n=23, lens="uniform", lo=37, hi=1999, block=24, layout=BLOCK_MAJOR, q_tokens=4, len_seed=5),
        # many small requests behind one system prompt
        _case(name="prefix-small-requests", op="attend", n=256, lens="uniform", lo=64, hi=512, prefixes=1, prefix_len=2048, len_seed=7),
        # 70B-shaped heads, 64 requests over one document: the products over the prefix carry the call
        _case(name="prefix-document", op="attend", n=64, lens="uniform", lo=16, hi=300, group=8, block=64, layout=BLOCK_MAJOR, prefixes=1, prefix_len=16001, len_seed=9),
        # several prompts, a few requests on each (parallel samples of one prompt)
        _case(name="prefix-samples", op="attend", n=64, lens="uniform", lo=1, hi=700, prefixes=16, prefix_len=1024, dtype="fp16", len_seed=11),
        # scores kept while decoding the uniform batch
        _case(name="weigh-8b-uniform", op="weigh", n=32, lens="fixed", hi=2048),
        # scores of the prompt's last 16 tokens, behind a shared prefix, ragged lengths
        _case(name="weigh-window", op="weigh", n=12, lens="uniform", lo=300, hi=4096, q_tokens=16, prefixes=2, prefix_len=513, len_seed=13),
        # lognormal batch cut to 1024 tokens a head on its way from the prefill to the decode pool
        _case(name="evict-8b-lognormal", op="evict", layers=4, n=64, lens="lognormal", lo=16, hi=8192, block=16, layout=BLOCK_MAJOR, budget=1024, sink=4, recent=256),
        # one long context cut to an odd budget
        _case(name="evict-long", op="evict", layers=2, n=1, lens="fixed", hi=100003, budget=4999, sink=1, recent=64, block=128, dst_block=64, dtype="fp16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case.  The tokens of a case are bounded by those of the listed long and uniform ones."""
    op = rng.choice(["attend", "attend", "prefix", "prefix", "weigh", "evict"])
    c = _case(op="attend" if op == "prefix" else op, layers=rng.choice([1, 2, 3]),
              heads=rng.choice([1, 2, 4, 5, 8]), group=rng.choice([1, 2, 3, 4, 7, 8, 16]), dim=rng.choice([64, 80, 96, 128, 128, 128, 256]),
              block=rng.choice([16, 24, 32, 64, 100, 128, 256]), layout=rng.choice([BLOCK_MAJOR, LAYER_MAJOR]), dtype=rng.choice(["bf16", "fp16"]),
              q_tokens=rng.choice([1, 1, 1, 2, 4, 7]), len_seed=rng.randrange(1 << 20))
    cells = 32 * 2048 * 8 * 128               # elements of K of the uniform batch
    tokens = cells // (c["heads"] * c["dim"])
    c["n"] = _log_uniform(rng, 1, 128)
    top = max(32, min(100000, tokens // c["n"]))
    c["hi"] = max(c["q_tokens"], _log_uniform(rng, 16, top))
    c["lens"] = rng.choice(["fixed", "uniform", "uniform"])
    c["lo"] = max(c["q_tokens"], 1 + rng.randrange(c["hi"]))
    c["lo"] = min(c["lo"], c["hi"])
    if op == "prefix":
        c["prefixes"] = rng.choice([1, 1, 2, 5])
        # products over the prefix: never more than those of the listed document case
        rows = c["n"] * c["q_tokens"] * c["group"] * c["heads"] * c["dim"]
        c["prefix_len"] = _log_uniform(rng, 33, max(64, min(30000, 64 * 8 * 8 * 128 * 16001 // rows)))
    if op == "evict":
        c.update(q_tokens=1, dst_block=rng.choice([16, 48, 64, 128]), dst_layout=rng.choice([BLOCK_MAJOR, LAYER_MAJOR]))
        c["layers"] = 1 if c["n"] * c["hi"] * c["heads"] * c["dim"] > cells // 2 else c["layers"]
        c["recent"] = rng.randrange(1 + c["hi"] // 8)
        c["sink"] = rng.choice([0, 1, 4])
        c["budget"] = c["recent"] + c["sink"] + max(1, _log_uniform(rng, 1, c["hi"]))
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _lens(c):
    rng = random.Random(c["len_seed"] * 7919 + 17)
    if c["lens"] == "fixed":
        return [c["hi"]] * c["n"]
    if c["lens"] == "uniform":
        return [rng.randint(c["lo"], c["hi"]) for _ in range(c["n"])]
    return [max(c["lo"], min(c["hi"], round(math.exp(math.log(1024) + 0.8 * rng.gauss(0, 1))))) for _ in range(c["n"])]


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


def _members(c):
    """Prefix of each request (-1: none); requests are dealt to the prefixes in turn."""
    return [i % c["prefixes"] if c["prefixes"] else -1 for i in range(c["n"])]


def _inputs(case, seed):
    c = {**_DEFAULTS, **case}
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt = _torch_dtype(c)
    lens = _lens(c)
    B = c["block"]
    p_lens = [c["prefix_len"] + 17 * i for i in range(c["prefixes"])]
    counts = [-(-n // B) for n in p_lens + lens]
    blocks = sum(counts) + max(1, sum(counts) // 16)
    off, tbl = _tables(rng, counts, blocks)
    np_ = c["prefixes"]
    s = {"case": c, "lens": lens, "prefix_lens": p_lens, "member": _members(c),
         "prefix_off": off[:np_ + 1], "prefix_tbl": tbl[:off[np_]], "off": off[np_:] - off[np_], "tbl": tbl[off[np_]:],
         "layer": c["layers"] - 1, "blocks": blocks}
    s["pool"] = torch.empty(_shape(c["layout"], c["layers"], c["heads"], c["dim"], B, blocks), device="cuda", dtype=dt).normal_(generator=gen)
    width = max(lens)
    if c["op"] == "evict":
        D = c["dst_block"]
        d_counts = [-(-min(n, c["budget"]) // D) for n in lens]
        d_blocks = max(1, sum(d_counts))
        s["dst_off"], s["dst_tbl"] = _tables(rng, d_counts, d_blocks)
        s["dst_blocks"] = d_blocks
        s["dst_pool"] = torch.zeros(_shape(c["dst_layout"], c["layers"], c["heads"], c["dim"], D, d_blocks), device="cuda", dtype=dt)
        # accumulated weights: a few tokens hold most of it, some were never looked at
        w = torch.randn(c["layers"], c["n"], c["heads"], width, device="cuda", generator=gen).mul_(2).exp_()
        s["scores"] = w.mul_(torch.rand(w.shape, device="cuda", generator=gen) > 0.1)
    else:
        s["q"] = torch.randn(c["n"], c["q_tokens"], c["heads"] * c["group"], c["dim"], device="cuda", generator=gen).mul_(2).to(dt)
        if c["op"] == "weigh":
            s["scores"] = torch.rand(c["n"], c["heads"], width, device="cuda", generator=gen)
            s["scores_out"] = torch.zeros_like(s["scores"])
    return s


def _slots(lens, off, tbl, block):
    """[request, token]: block * block size + offset; 0 past a request's end."""
    pos = np.arange(max(lens))[None, :]
    at = np.minimum(off[:-1, None] + pos // block, len(tbl) - 1)
    slot = np.where(pos < np.asarray(lens)[:, None], tbl[at].astype(np.int64) * block + pos % block, 0)
    return torch.from_numpy(slot).cuda()


def prepare(case, seed):
    s = _inputs(case, seed)
    c, lens, p_lens, B = s["case"], s["lens"], s["prefix_lens"], case.get("block", _DEFAULTS["block"])

    if own:
        from paper_2408_08147_b200.sequences import CacheSession, Sequences
        from paper_2408_08147_b200.workloads import Geometry

        dt = _torch_dtype(c)
        g = Geometry(c["layout"], c["layers"], c["heads"], c["dim"], 2, B, s["blocks"])
        seqs = Sequences(lens, s["off"], s["tbl"], p_lens, s["prefix_off"], s["prefix_tbl"], s["member"])
        if c["op"] == "evict":
            s["session"] = CacheSession(g, s["pool"], seqs)
            g2 = Geometry(c["dst_layout"], c["layers"], c["heads"], c["dim"], 2, c["dst_block"], s["dst_blocks"])
            s["dst_session"] = CacheSession(g2, s["dst_pool"], Sequences([min(n, c["budget"]) for n in lens], s["dst_off"], s["dst_tbl"]))
        else:
            s["session"] = CacheSession(g, s["pool"], seqs, num_q_heads=c["heads"] * c["group"], q_tokens=c["q_tokens"], dtype=dt)
    else:
        # where each token lies (padded to the longest request): what a program without the operators keeps
        s["len_t"] = torch.tensor(lens, device="cuda")
        s["slots"] = _slots(lens, s["off"], s["tbl"], B)
        if p_lens:
            s["prefix_len_t"] = torch.tensor(p_lens, device="cuda")
            s["prefix_slots"] = _slots(p_lens, s["prefix_off"], s["prefix_tbl"], B)
        if c["op"] == "evict":
            s["dst_slots"] = _slots([min(n, c["budget"]) for n in lens], s["dst_off"], s["dst_tbl"], c["dst_block"])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        if c["op"] == "evict":
            kept, kept_scores, new_len = state["session"].evict(state["dst_session"], state["scores"], c["budget"], sink=c["sink"], recent=c["recent"])
            return {"kept": kept, "scores": kept_scores, "lens": new_len, "pool": state["dst_pool"]}
        if c["op"] == "weigh":
            out, lse = state["session"].attend(state["layer"], state["q"], scores_in_t=state["scores"], scores_t=state["scores_out"])
            return {"out": out, "lse": lse, "scores": state["scores_out"]}
        out, lse = state["session"].attend(state["layer"], state["q"])
        return {"out": out, "lse": lse}
    return _plain_evict(state) if c["op"] == "evict" else _plain_attend(state)


def _plane(pool, layout, layer, kv):
    """One layer's keys or values as [block, token, head, dim]."""
    return pool[:, layer, kv] if layout == BLOCK_MAJOR else pool[layer, kv].transpose(1, 2)


def _rows(plane, slots, block):
    """[request, head, token, dim] in 32 bits of the given slots."""
    return plane[slots // block, slots % block].transpose(1, 2).float()


def _plain_attend(s):
    c = s["case"]
    n, H, G, D, Q, P = c["n"], c["heads"], c["group"], c["dim"], c["q_tokens"], c["prefixes"]
    k_all, v_all = (_plane(s["pool"], c["layout"], s["layer"], kv) for kv in (0, 1))
    q = s["q"].float().view(n, Q, H, G, D).permute(0, 2, 1, 3, 4).reshape(n, H, Q * G, D) / math.sqrt(D)
    W = s["slots"].shape[1]
    logits = torch.matmul(q, _rows(k_all, s["slots"], c["block"]).transpose(2, 3))            # [request, head, row, token]
    pos = torch.arange(W, device="cuda")
    hidden = (Q - 1) - torch.arange(Q, device="cuda").repeat_interleave(G)                    # newest tokens a row does not see
    seen = pos[None, None, :] < (s["len_t"][:, None] - hidden[None, :])[:, :, None]
    logits.masked_fill_(~seen[:, None], -math.inf)
    if P:
        # requests of one prefix side by side, so that its keys are multiplied once; request i has prefix i % P
        M = -(-n // P)
        grouped = torch.zeros(M * P, H, Q * G, D, device="cuda")
        grouped[:n] = q
        grouped = grouped.view(M, P, H, Q * G, D).permute(1, 2, 0, 3, 4).reshape(P, H, M * Q * G, D)
        over = torch.matmul(grouped, _rows(k_all, s["prefix_slots"], c["block"]).transpose(2, 3))
        wide = over.shape[-1]
        over.masked_fill_((torch.arange(wide, device="cuda")[None, :] >= s["prefix_len_t"][:, None])[:, None, None, :], -math.inf)
        over = over.view(P, H, M, Q * G, wide).permute(2, 0, 1, 3, 4).reshape(M * P, H, Q * G, wide)[:n]
        logits = torch.cat([logits, over], -1)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p[..., :W], _rows(v_all, s["slots"], c["block"]))
    if P:
        weights = torch.zeros(M * P, H, Q * G, wide, device="cuda")
        weights[:n] = p[..., W:]
        weights = weights.view(M, P, H, Q * G, wide).permute(1, 2, 0, 3, 4).reshape(P, H, M * Q * G, wide)
        op = torch.matmul(weights, _rows(v_all, s["prefix_slots"], c["block"]))
        o += op.view(P, H, M, Q * G, D).permute(2, 0, 1, 3, 4).reshape(M * P, H, Q * G, D)[:n]
    lse = (top + torch.log(total)).view(n, H, Q, G).permute(0, 2, 1, 3).reshape(n, Q, H * G)
    out = (o / total).view(n, H, Q, G, D).permute(0, 2, 1, 3, 4).reshape(n, Q, H * G, D).to(s["q"].dtype)
    if c["op"] != "weigh":
        return {"out": out, "lse": lse}
    torch.add(s["scores"], (p[..., :W] / total).sum(2), out=s["scores_out"])
    return {"out": out, "lse": lse, "scores": s["scores_out"]}


def _plain_evict(s):
    c = s["case"]
    L, H, K, n = c["layers"], c["heads"], c["budget"], c["n"]
    W = s["slots"].shape[1]
    pos, length = torch.arange(W, device="cuda"), s["len_t"][:, None]
    weight = s["scores"].masked_fill((pos[None] >= length)[None, :, None], -math.inf)
    always = (pos[None] < c["sink"]) | ((pos[None] >= length - c["recent"]) & (pos[None] < length))
    weight = weight.masked_fill(always[None, :, None], math.inf)
    idx = torch.sort(weight, dim=-1, descending=True, stable=True)[1][..., :K]
    idx = torch.where(idx < length[None, :, None], idx, W).sort(-1)[0]                        # in order, W: nothing
    wide = idx.shape[-1]
    held = idx < W
    kept = torch.full((L, n, H, K), -1, dtype=torch.int32, device="cuda")
    kept[..., :wide] = torch.where(held, idx, -1)
    kept_scores = torch.zeros(L, n, H, K, device="cuda")
    kept_scores[..., :wide] = torch.gather(s["scores"], 3, idx.clamp(max=W - 1)).masked_fill(~held, 0.0)
    l, r, h, j = held.nonzero(as_tuple=True)
    at, to = s["slots"][r, idx[l, r, h, j]], s["dst_slots"][r, j]
    for kv in (0, 1):
        if c["layout"] == BLOCK_MAJOR:
            rows = s["pool"][at // c["block"], l, kv, at % c["block"], h]
        else:
            rows = s["pool"][l, kv, at // c["block"], h, at % c["block"]]
        if c["dst_layout"] == BLOCK_MAJOR:
            s["dst_pool"][to // c["dst_block"], l, kv, to % c["dst_block"], h] = rows
        else:
            s["dst_pool"][l, kv, to // c["dst_block"], h, to % c["dst_block"]] = rows
    return {"kept": kept, "scores": kept_scores, "lens": s["len_t"].clamp(max=K).int(), "pool": s["dst_pool"]}


# ---------------------------------------------------------------------------
# the least a pass has to do, and what it has to give
# ---------------------------------------------------------------------------

def work(case):
    c = {**_DEFAULTS, **case}
    lens = _lens(c)
    H, G, D, Q = c["heads"], c["group"], c["dim"], c["q_tokens"]
    if c["op"] == "evict":
        kept = sum(min(n, c["budget"]) for n in lens)
        rows = c["layers"] * H
        return {"bytes": rows * (4 * sum(lens) + 4 * 2 * kept + 2 * 2 * 2 * D * kept), "flops": rows * sum(lens)}
    member = _members(c)
    p_lens = [c["prefix_len"] + 17 * i for i in range(c["prefixes"])]
    used = sum(p_lens[i] for i in set(member) if i >= 0)
    row = Q * H * G
    size = 2 * 2 * H * D * (sum(lens) + used) + c["n"] * row * (2 * 2 * D + 4)
    if c["op"] == "weigh":
        size += 2 * 4 * H * sum(lens)
    pairs = sum(lens) + sum(p_lens[i] for i in member if i >= 0)
    return {"bytes": size, "flops": 4 * D * row * pairs}


def _token(pool, c, layer, kv, blk, tt):
    """[token, head, dim] of the tokens at (blk, tt), in 64 bits."""
    if c["layout"] == BLOCK_MAJOR:
        return pool[blk, layer, kv, tt].double()
    return pool[layer, kv, blk, :, tt].double()


def exact(case, seed):
    s = _inputs(case, seed)
    c = s["case"]
    return _exact_evict(s, c) if c["op"] == "evict" else _exact_attend(s, c)


def _exact_attend(s, c):
    H, G, D, Q, n = c["heads"], c["group"], c["dim"], c["q_tokens"], c["n"]
    out = torch.zeros(n, Q, H * G, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(n, Q, H * G, dtype=torch.float64, device="cuda")
    scores = s["scores"].double() if c["op"] == "weigh" else None
    if c["op"] == "weigh":
        scores_out = torch.zeros_like(scores) + scores

    def where(off, tbl, r, length):
        pos = torch.arange(length, device="cuda")
        t = torch.as_tensor(tbl[off[r]:off[r + 1]].astype(np.int64), device="cuda")
        return t[pos // c["block"]], pos % c["block"]

    for r in range(n):
        parts = []
        if s["member"][r] >= 0:
            g = s["member"][r]
            parts.append(where(s["prefix_off"], s["prefix_tbl"], g, s["prefix_lens"][g]))
        parts.append(where(s["off"], s["tbl"], r, s["lens"][r]))
        k = torch.cat([_token(s["pool"], c, s["layer"], 0, *w) for w in parts])
        v = torch.cat([_token(s["pool"], c, s["layer"], 1, *w) for w in parts])
        total = k.shape[0]
        for h in range(H):
            for j in range(Q):
                sees = total - (Q - 1 - j)
                qs = s["q"][r, j, h * G:(h + 1) * G].double()
                z = qs @ k[:sees, h].T / math.sqrt(D)
                norm = torch.logsumexp(z, -1)
                w = torch.exp(z - norm[:, None])
                out[r, j, h * G:(h + 1) * G] = w @ v[:sees, h]
                lse[r, j, h * G:(h + 1) * G] = norm
                if scores is not None:
                    own_from = total - s["lens"][r]
                    scores_out[r, h, :sees - own_from] += w[:, own_from:].sum(0)
    return {"out": out, "lse": lse, "scores": scores_out} if scores is not None else {"out": out, "lse": lse}


def _exact_evict(s, c):
    L, H, K, n = c["layers"], c["heads"], c["budget"], c["n"]
    sc = s["scores"].cpu().numpy().astype(np.float64)
    if sc.size > 4_000_000:
        return None
    kept = np.full((L, n, H, K), -1, np.int64)
    ks = np.zeros((L, n, H, K))
    pool = torch.zeros(s["dst_pool"].shape, dtype=torch.float64, device="cuda")
    for r, length in enumerate(s["lens"]):
        m = min(length, K)
        o = s["off"][r]
        for l in range(L):
            for h in range(H):
                row = sc[l, r, h, :length]
                if length <= K:
                    ids = np.arange(length)
                else:
                    rank = -row.copy()
                    rank[:c["sink"]] = -math.inf
                    rank[length - c["recent"]:] = -math.inf
                    ids = np.sort(np.lexsort((np.arange(length), rank))[:K])
                kept[l, r, h, :m] = ids
                ks[l, r, h, :m] = row[ids]
                blk = torch.as_tensor(s["tbl"][o + ids // c["block"]].astype(np.int64), device="cuda")
                tt = torch.as_tensor(ids % c["block"], device="cuda")
                to = np.arange(m)
                d_blk = torch.as_tensor(s["dst_tbl"][s["dst_off"][r] + to // c["dst_block"]].astype(np.int64), device="cuda")
                d_tt = torch.as_tensor(to % c["dst_block"], device="cuda")
                for kv in (0, 1):
                    got = _token(s["pool"], c, l, kv, blk, tt)[:, h]
                    if c["dst_layout"] == BLOCK_MAJOR:
                        pool[d_blk, l, kv, d_tt, h] = got
                    else:
                        pool[l, kv, d_blk, h, d_tt] = got
    return {"kept": torch.from_numpy(kept), "scores": torch.from_numpy(ks),
            "lens": torch.tensor([min(x, K) for x in s["lens"]]), "pool": pool}
