"""What the constrained beam-search operators are measured on.

Four operators, each in a plain form (elementary torch operations in 32 bits) and through the
library's own calls:

  select     one selection step of beam search over beams x vocabulary under packed token masks
  blocks     block tables and slot maps from request lengths: a step is drafted (its tokens get
             cache slots, new blocks are taken) and rolled back (the blocks are given back)
  reorder    the cache follows the selection: block tables move to the parents', full blocks are
             shared, a partly filled last block is copied for every further child
  backtrack  the hypotheses of a finished search read back from the per-step parents

``own`` chooses the side; everything a call casts, unpacks or lays out is done inside ``run``.
"""
import math

import numpy as np
import torch

own = False

NORM_ALLOWED, NORM_FULL, NORM_NONE = 0, 1, 2
NEG_INF = float("-inf")
MOST_LOGITS = 128 * 8 * 128256      # the largest selection that is listed


# ---------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------
def listed():
    return [
        # one interactive request with 4 beams inside a template: the call is all latency
        {"name": "select_html_1x4", "op": "select", "R": 1, "K": 4, "V": 32000, "pad": 0, "dtype": "fp32",
         "mask": "literal", "norm": NORM_ALLOWED, "n_out": 4},
        # a small serving batch that fills in JSON: a few allowed tokens per row, two candidates
        # kept per beam
        {"name": "select_json_8x4", "op": "select", "R": 8, "K": 4, "V": 128256, "pad": 0, "dtype": "bf16",
         "mask": "literal", "norm": NORM_ALLOWED, "n_out": 8},
        # free-text slots: nearly every token is allowed, so every logit is read
        {"name": "select_text_16x5", "op": "select", "R": 16, "K": 5, "V": 128256, "pad": 0, "dtype": "bf16",
         "mask": "text", "norm": NORM_ALLOWED, "n_out": 5},
        # scores by the model's own distribution (the whole vocabulary in the denominator), masked
        # afterwards; odd vocabulary in rows that are not padded
        {"name": "select_model_64x8_odd", "op": "select", "R": 64, "K": 8, "V": 151937, "pad": 0, "dtype": "bf16",
         "mask": "mixed", "norm": NORM_FULL, "n_out": 16},
        # a large vocabulary with fp32 logits, some rows in literals and some in free text
        {"name": "select_snippets_32x4", "op": "select", "R": 32, "K": 4, "V": 256000, "pad": 0, "dtype": "fp32",
         "mask": "mixed", "norm": NORM_ALLOWED, "n_out": 8},
        # offline batch at full width, rows padded to whole lines
        {"name": "select_wide_128x8", "op": "select", "R": 128, "K": 8, "V": 128256, "pad": 64, "dtype": "bf16",
         "mask": "text", "norm": NORM_ALLOWED, "n_out": 8},
        # one decode step of 1024 sequences: a token each, one block in sixteen is new
        {"name": "blocks_decode_1024", "op": "blocks", "S": 1024, "new": 1, "ctx": 2048, "block": 16,
         "n_blocks": 163840, "short": False},
        # prompts of very different lengths enter together
        {"name": "blocks_prefill_64", "op": "blocks", "S": 64, "new": 8192, "ctx": 64, "block": 16,
         "n_blocks": 65536, "short": False},
        # a small batch of beams over a few layers
        {"name": "reorder_4x4", "op": "reorder", "R": 4, "K": 4, "prompt": 256, "gen": 40, "block": 16,
         "planes": 8, "token_elems": 512},
        # a full batch of wide beams with long prompts
        {"name": "reorder_64x8", "op": "reorder", "R": 64, "K": 8, "prompt": 500, "gen": 64, "block": 16,
         "planes": 16, "token_elems": 1024},
        # a short answer read back, and the longest
        {"name": "backtrack_256_8x4", "op": "backtrack", "T": 256, "R": 8, "K": 4},
        {"name": "backtrack_4096_128x8", "op": "backtrack", "T": 4096, "R": 128, "K": 8},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["select", "select", "select", "blocks", "reorder", "backtrack"])
    if op == "select":
        K = rng.choice([1, 2, 3, 4, 5, 8, 12, 16])
        V = _log_int(rng, 1000, 256000)
        R = _log_int(rng, 1, 128)
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        limit = MOST_LOGITS if dtype == "bf16" else MOST_LOGITS // 2
        R = max(1, min(R, limit // (K * V)))
        return {"op": op, "R": R, "K": K, "V": V, "pad": rng.choice([0, 1, 64]), "dtype": dtype,
                "mask": rng.choice(["literal", "text", "mixed", "none"]),
                "norm": rng.choice([NORM_ALLOWED, NORM_FULL, NORM_NONE]),
                "n_out": rng.choice([K, 2 * K, K + 1])}
    if op == "blocks":
        S, block = _log_int(rng, 1, 2048), rng.choice([8, 16, 32, 64])
        new = _log_int(rng, 1, max(1, min(16384, 262144 // S)))
        ctx = _log_int(rng, 1, 4096)
        need = S * (-(-(new + ctx) // block) + 1)
        return {"op": op, "S": S, "new": new, "ctx": ctx, "block": block,
                "n_blocks": need + rng.randrange(1, 20000), "short": rng.random() < 0.25}
    if op == "reorder":
        R, K, block = _log_int(rng, 1, 64), rng.choice([2, 3, 4, 5, 8, 12]), rng.choice([8, 16, 32])
        R = max(1, min(R, 512 // K))
        return {"op": op, "R": R, "K": K, "prompt": _log_int(rng, 1, 600), "gen": _log_int(rng, 1, 100),
                "block": block, "planes": rng.choice([2, 4, 6, 12]), "token_elems": rng.choice([64, 128, 320, 512])}
    return {"op": op, "T": _log_int(rng, 1, 4096), "R": _log_int(rng, 1, 128), "K": rng.choice([1, 2, 3, 4, 5, 8])}


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _masks(case, g, N, V):
    """Packed masks: literal states allow a handful of tokens, free-text slots nearly all; one
    row in 32 allows nothing (its hypothesis cannot go on)."""
    W = (V + 31) // 32
    if case["mask"] == "none":
        return None
    bits = torch.zeros((N, W * 32), dtype=torch.bool, device="cuda")
    rows = torch.arange(N, device="cuda")
    text = {"literal": rows < 0, "text": rows >= 0, "mixed": rows % 4 == 0}[case["mask"]]
    for a in range(0, N, 64):
        b = min(N, a + 64)
        wide = torch.rand((b - a, V), device="cuda", generator=g) < 0.93
        bits[a:b, :V] = wide & text[a:b, None]
    few = torch.randint(0, V, (N, 48), device="cuda", generator=g)
    take = torch.rand((N, 1), device="cuda", generator=g) * 48 >= torch.arange(48, device="cuda")[None, :]
    small = torch.zeros((N, W * 32), dtype=torch.int32, device="cuda")
    small.scatter_add_(1, few, take.to(torch.int32))
    bits |= (small > 0) & ~text[:, None]
    bits &= (torch.rand((N, 1), device="cuda", generator=g) >= 1 / 32)
    out = torch.empty((N, W), dtype=torch.int32, device="cuda")
    weights = (torch.ones(32, dtype=torch.int64, device="cuda") << torch.arange(32, device="cuda"))
    for a in range(0, N, 64):
        words = (bits[a:a + 64].view(-1, W, 32).to(torch.int64) * weights).sum(2)
        out[a:a + 64] = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
    return out


def _unpack(bitmask, V):
    bit = torch.arange(32, device=bitmask.device, dtype=torch.int32)
    return ((bitmask[:, :, None] >> bit) & 1).bool().reshape(bitmask.shape[0], -1)[:, :V]


def _top64(s, scores, keep):
    """The best `keep` candidates of every request in 64 bits: (score, beam, logit), best first."""
    V, K = s["V"], s["K"]
    R = s["logits"].shape[0] // K
    per = min(keep, V)
    best, logit = [], []
    for i in range(0, R * K, 64):
        j = min(R * K, i + 64)
        x = s["logits"][i:j].double()
        m = _unpack(s["bitmask"][i:j], V) if s["bitmask"] is not None else torch.ones_like(x, dtype=torch.bool)
        inside = torch.where(m, x, NEG_INF)
        if s["norm"] == NORM_NONE:
            lse = torch.zeros((j - i, 1), dtype=torch.float64, device="cuda")
        else:
            lse = torch.logsumexp(inside if s["norm"] == NORM_ALLOWED else x, 1, keepdim=True)
        top = torch.topk(inside, per, dim=1).values
        value = torch.where(torch.isfinite(top), top - lse, NEG_INF)
        done = s["finished"][i:j, None] != 0
        first = torch.arange(per, device="cuda")[None, :] == 0
        value = torch.where(done, torch.where(first, 0.0, NEG_INF), value)
        best.append(value)
        logit.append(torch.where(done, 0.0, top))
    return torch.cat(best).view(R, K, per), torch.cat(logit).view(R, K, per)


def _apart(s, g):
    """Scores of running hypotheses for which the order of the kept candidates does not hang on
    the last bits of a logarithm: where two candidates of different beams are within 1e-4, the
    request's scores are drawn again.  (Equal logits of one row stay equal, and stay in.)"""
    R, K = s["R"], s["K"]
    draw_scores = lambda: -12.0 * torch.rand((R, K), device="cuda", generator=g)  # noqa: E731
    scores = draw_scores()
    gone = torch.rand((R, K), device="cuda", generator=g) < 1 / 16   # hypotheses that were given up
    keep = s["n_out"] + 1
    value, logit = _top64(s, scores, keep)
    beam = torch.arange(K, device="cuda")[None, :, None].expand_as(value)
    n = min(keep, value.shape[1] * value.shape[2])
    for _ in range(8):
        scores = torch.where(gone, NEG_INF, scores)
        total = (scores.double()[:, :, None] + value).reshape(R, -1)
        top, at = torch.topk(total, n, dim=1)
        b, x = beam.reshape(R, -1).gather(1, at), logit.reshape(R, -1).gather(1, at)
        gap = top[:, :-1] - top[:, 1:]
        same = (b[:, :-1] == b[:, 1:]) & (x[:, :-1] == x[:, 1:])
        bad = ((gap < 1e-4) & ~same & torch.isfinite(top[:, 1:])).any(1)
        scores = torch.where(bad[:, None], draw_scores(), scores)
    return torch.where(gone, NEG_INF, scores).reshape(-1).contiguous()


def _prepare_select(case, seed):
    g = _generator(seed)
    R, K, V = case["R"], case["K"], case["V"]
    N = R * K
    stride = V if not case["pad"] else -(-V // case["pad"]) * case["pad"] + (case["pad"] if case["pad"] == 1 else 0)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    whole = torch.empty((N, stride), dtype=dtype, device="cuda")
    for a in range(0, N, 64):
        x = torch.randn((min(64, N - a), stride), device="cuda", generator=g) * 2.0
        # fp32 logits carry the 10 fraction bits of a reduced-precision output head
        whole[a:a + 64] = x if dtype == torch.bfloat16 else torch.round(x * 1024.0) / 1024.0
    s = {"op": "select", "R": R, "K": K, "V": V, "norm": case["norm"], "n_out": case["n_out"],
         "logits": whole[:, :V], "eos": 2, "bitmask": _masks(case, g, N, V),
         "finished": (torch.rand(N, device="cuda", generator=g) < 1 / 8).to(torch.int32)}
    s["score"] = _apart(s, g)
    s["score_out"] = torch.empty((R, case["n_out"]), dtype=torch.float32, device="cuda")
    s["parent_out"] = torch.empty((R, case["n_out"]), dtype=torch.int32, device="cuda")
    s["token_out"] = torch.empty((R, case["n_out"]), dtype=torch.int32, device="cuda")
    if own:
        import paper_2507_16768_b200 as wg
        s["beam"] = wg.Beam(V, max_requests=R, max_beams=K, max_out=case["n_out"])
        s["plan"] = wg.BeamPlan(s["beam"], K, s["score"], s["score_out"], s["parent_out"], s["token_out"],
                                bitmask=s["bitmask"], finished=s["finished"], eos_id=s["eos"], norm=case["norm"])
    return s


def _pool(s, n_blocks, block, rows, ref):
    """The library's handles for a cache whose reference counts are `ref`."""
    import paper_2507_16768_b200 as wg
    s["pool"] = wg.KvPool(n_blocks, block, max_seqs=rows)
    s["pool"].load(ref)
    s["tables"] = wg.KvTables(s["pool"], s["table"], s["len"], s["status"])


def _step_tokens(case):
    mean = 1.0 if case["new"] == 1 else (case["new"] - 1) / math.log(case["new"])
    return int(case["S"] * mean * 1.125) + 8


def _prepare_blocks(case, seed):
    g = _generator(seed)
    S, block, n_blocks = case["S"], case["block"], case["n_blocks"]
    ctx = torch.randint(0, case["ctx"] + 1, (S,), device="cuda", generator=g, dtype=torch.int32)
    if case["new"] == 1:
        new = torch.ones(S, dtype=torch.int32, device="cuda")
    else:  # lengths over their logarithm, as prompts come; one request in 16 brings nothing
        u = torch.rand(S, device="cuda", generator=g)
        new = torch.exp(u * math.log(case["new"])).round().to(torch.int32)
        new = torch.where(torch.rand(S, device="cuda", generator=g) < 1 / 16, 0, new).to(torch.int32)
    # the step has room for so many tokens; requests that do not fit in wait
    T = _step_tokens(case)
    new = torch.where(torch.cumsum(new, 0) <= T, new, 0).to(torch.int32)
    M = -(-(case["ctx"] + case["new"]) // block)
    held = (ctx + block - 1) // block
    ids = torch.randperm(n_blocks, device="cuda", generator=g, dtype=torch.int64)
    if case["short"]:   # other requests hold so much that not everybody gets the blocks wanted
        total, need = int(held.sum()), int((((ctx + new + block - 1) // block) - held).sum())
        taken = min(n_blocks, max(total, n_blocks - need * 3 // 4))
    else:
        total = taken = int(held.sum())
    col = torch.arange(M, device="cuda")
    at = (torch.cumsum(held, 0) - held)[:, None] + col[None, :]
    table = torch.where(col[None, :] < held[:, None], ids[at.clamp(max=n_blocks - 1)], -1).to(torch.int32)
    ref = torch.zeros(n_blocks, dtype=torch.int32, device="cuda")
    ref[ids[:taken]] = 1
    s = {"op": "blocks", "block": block, "n_blocks": n_blocks, "T": T, "table": table.contiguous(),
         "len": ctx.clone(), "keep": ctx.clone(), "new": new, "ref": ref,
         "status": torch.zeros(S, dtype=torch.int32, device="cuda")}
    if own:
        import paper_2507_16768_b200 as wg
        _pool(s, n_blocks, block, S, ref)
        s["slots"] = wg.SlotMap(S, T)
    return s


def _prepare_reorder(case, seed):
    g = _generator(seed)
    R, K, block = case["R"], case["K"], case["block"]
    N = R * K
    prompt = torch.randint((case["prompt"] + 1) // 2, case["prompt"] + 1, (R,), device="cuda", generator=g)
    gen = torch.randint((case["gen"] + 1) // 2, case["gen"] + 1, (R,), device="cuda", generator=g)
    lens = (prompt + gen)[:, None].expand(R, K).clone()
    ended = torch.rand((R, K), device="cuda", generator=g) < 1 / 8     # hypotheses that ended earlier
    lens = torch.where(ended, prompt[:, None] + (gen[:, None] * torch.rand((R, K), device="cuda", generator=g)).long(), lens)
    shared = prompt // block
    held = (lens + block - 1) // block
    M = -(-(case["prompt"] + case["gen"]) // block) + 1
    private = held - shared[:, None]
    n_blocks = R * (case["prompt"] // block) + N * (-(-case["gen"] // block) + 2)
    ids = torch.randperm(n_blocks, device="cuda", generator=g, dtype=torch.int64)
    col = torch.arange(M, device="cuda")[None, None, :]
    of_prompt = (torch.cumsum(shared, 0) - shared)[:, None, None] + col
    flat = private.reshape(-1)
    of_beam = int(shared.sum()) + (torch.cumsum(flat, 0) - flat).view(R, K, 1) + col - shared[:, None, None]
    at = torch.where(col < shared[:, None, None], of_prompt, of_beam).clamp(0, n_blocks - 1)
    table = torch.where(col < held[:, :, None], ids[at], -1).to(torch.int32).view(N, M).contiguous()
    ref = torch.zeros(n_blocks, dtype=torch.int32, device="cuda")
    ref.index_add_(0, table.reshape(-1).long().clamp(min=0), (table.reshape(-1) >= 0).to(torch.int32))
    parent = torch.randint(0, K, (R, K), device="cuda", generator=g, dtype=torch.int32)
    planes = torch.empty((case["planes"], n_blocks, block, case["token_elems"]), dtype=torch.bfloat16, device="cuda")
    for p in range(case["planes"]):
        planes[p] = torch.randn(planes.shape[1:], device="cuda", generator=g, dtype=torch.bfloat16)
    s = {"op": "reorder", "R": R, "K": K, "block": block, "n_blocks": n_blocks, "table": table,
         "len": lens.to(torch.int32).reshape(-1).contiguous(), "ref": ref, "parent": parent, "planes": planes,
         "status": torch.zeros(N, dtype=torch.int32, device="cuda")}
    if own:
        import paper_2507_16768_b200 as wg
        _pool(s, n_blocks, block, N, ref)
        s["kv"] = wg.KvPlanes(list(planes.unbind(0)), block)
    return s


def _prepare_backtrack(case, seed):
    g = _generator(seed)
    T, R, K = case["T"], case["R"], case["K"]
    token = torch.randint(0, 128256, (T, R, K), device="cuda", generator=g, dtype=torch.int32)
    # most beams go on from the few best of the step before; some are given up
    u = torch.rand((T, R, K), device="cuda", generator=g)
    parent = (u * u * K).to(torch.int32).clamp(max=K - 1)
    lost = torch.rand((T, R, K), device="cuda", generator=g) < 0.1 / T
    parent = torch.where(lost, -1, parent).to(torch.int32)
    return {"op": "backtrack", "token": token, "parent": parent,
            "out": torch.empty((R, K, T), dtype=torch.int32, device="cuda")}


def prepare(case, seed):
    return {"select": _prepare_select, "blocks": _prepare_blocks, "reorder": _prepare_reorder,
            "backtrack": _prepare_backtrack}[case["op"]](case, seed)


# ---------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------
def _plain_select(s):
    R, K, V, n_out = s["R"], s["K"], s["V"], s["n_out"]
    x = s["logits"].float()
    inside = x if s["bitmask"] is None else torch.where(_unpack(s["bitmask"], V), x, NEG_INF)
    if s["norm"] == NORM_NONE:
        lp = inside
    else:
        y = inside if s["norm"] == NORM_ALLOWED else x
        top = y.amax(1, keepdim=True)
        top = torch.where(torch.isfinite(top), top, 0.0)
        lse = top + torch.log(torch.exp(y - top).sum(1, keepdim=True))
        lp = torch.where(inside == NEG_INF, NEG_INF, inside - lse)
    score = s["score"][:, None]
    total = score + lp
    only = torch.where(torch.arange(V, device=x.device)[None, :] == s["eos"], score, NEG_INF)
    total = torch.where(s["finished"][:, None] != 0, only, total) + 0.0   # (-0.0 counts as 0.0)
    total = torch.where(torch.isnan(total), NEG_INF, total).view(R, K * V)
    # one whole number per candidate, unlike any other: the score's order, then the lower index
    bits = total.view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).to(torch.int64)
    key = order * (1 << 32) + ((1 << 32) - 1 - torch.arange(K * V, device=x.device))
    at = torch.topk(key, min(n_out, K * V), dim=1).indices
    best = total.gather(1, at)
    ok = best > NEG_INF
    s["score_out"].copy_(best)
    s["parent_out"].copy_(torch.where(ok, at // V, -1))
    s["token_out"].copy_(torch.where(ok, at % V, -1))
    return {"score": s["score_out"], "parent": s["parent_out"], "token": s["token_out"]}


def _free_ids(ref, n):
    """The first n free blocks in ascending order (entries past the last free one are not used)."""
    free = ref == 0
    at = torch.cumsum(free, 0) - 1
    ids = torch.zeros(max(n, 1) + 1, dtype=torch.int64, device=ref.device)
    ids.scatter_(0, torch.where(free, at, n + 1).clamp(max=max(n, 1)), torch.arange(ref.numel(), device=ref.device))
    return ids, free.sum()


def _plain_blocks(s):
    block, table, lens, new, ref = s["block"], s["table"], s["len"], s["new"], s["ref"]
    S, M = table.shape
    dev = table.device
    # draft: slots for the new tokens
    before, after = (lens + block - 1) // block, (lens + new + block - 1) // block
    need = after - before
    upto = torch.cumsum(need, 0)
    ids, n_free = _free_ids(ref, s["n_blocks"])
    granted = (need == 0) | (upto <= n_free)
    col = torch.arange(M, device=dev)[None, :]
    fresh = (col >= before[:, None]) & (col < after[:, None]) & granted[:, None]
    rank = (upto - need)[:, None] + col - before[:, None]
    got = ids[rank.clamp(0, s["n_blocks"])]
    table.copy_(torch.where(fresh, got, table))
    ref.index_add_(0, torch.where(fresh, got, 0).reshape(-1), fresh.reshape(-1).to(torch.int32))
    cu = torch.zeros(S + 1, dtype=torch.int32, device=dev)
    cu[1:] = torch.cumsum(new, 0)
    t = torch.arange(s["T"], device=dev, dtype=torch.int32)
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=S - 1)
    valid = t < cu[-1]
    pos = lens[seq] + t - cu[seq]
    slot = table[seq, (pos // block).clamp(0, M - 1).long()].long() * block + pos % block
    slot = torch.where(valid & granted[seq], slot, -1)
    pos = torch.where(valid, pos, -1)
    seq = torch.where(valid, seq, -1).to(torch.int32)
    status = torch.where(granted, 0, -3).to(torch.int32)
    lens.copy_(torch.where(granted, lens + new, lens))
    # roll back: what was taken is free again
    gone = (col >= ((s["keep"] + block - 1) // block)[:, None]) & (col < ((lens + block - 1) // block)[:, None])
    ref.index_add_(0, torch.where(gone, table, 0).reshape(-1).long(), -gone.reshape(-1).to(torch.int32))
    table.copy_(torch.where(gone, -1, table))
    lens.copy_(s["keep"])
    return {"cu": cu, "slot": slot, "pos": pos, "seq": seq, "status": status, "table": table,
            "len": lens, "ref": ref}


def _plain_reorder(s):
    R, K, block, table, lens, ref = s["R"], s["K"], s["block"], s["table"], s["len"], s["ref"]
    N, M = table.shape
    dev = table.device
    parent = s["parent"].long()
    row = (torch.arange(R, device=dev)[:, None] * K + parent.clamp(min=0)).reshape(-1)
    alive = parent.reshape(-1) >= 0
    new_len = torch.where(alive, lens[row], 0)
    col = torch.arange(M, device=dev)[None, :]
    moved = torch.where(col < ((new_len + block - 1) // block)[:, None], table[row], -1)
    # a child shares its parent's partly filled block only if no earlier sibling does
    earlier = (parent[:, None, :] == parent[:, :, None]) & \
        (torch.arange(K, device=dev)[None, :] < torch.arange(K, device=dev)[:, None])[None]
    further = earlier.any(2).reshape(-1) & alive & (new_len % block != 0)
    last = (new_len // block).long()
    is_last = (col == last[:, None]) & further[:, None]
    source = torch.where(further, moved.gather(1, last.clamp(max=M - 1)[:, None])[:, 0], -1)
    held = table >= 0
    ref.index_add_(0, torch.where(held, table, 0).reshape(-1).long(), -held.reshape(-1).to(torch.int32))
    stays = (moved >= 0) & ~is_last
    ref.index_add_(0, torch.where(stays, moved, 0).reshape(-1).long(), stays.reshape(-1).to(torch.int32))
    ids, n_free = _free_ids(ref, N)
    rank = torch.cumsum(further, 0) - 1
    granted = further & (rank < n_free)
    target = torch.where(granted, ids[rank.clamp(min=0)], -1)
    table.copy_(torch.where(is_last, target[:, None], moved))
    ref.index_add_(0, target.clamp(min=0), granted.to(torch.int32))
    lens.copy_(torch.where(further & ~granted, last * block, new_len))
    # the filled tokens of every copied block, in all planes at once
    who = granted.nonzero()[:, 0]
    at = torch.arange(block, device=dev)[None, :]
    child, token = (at < (new_len[who] % block)[:, None]).nonzero(as_tuple=True)
    s["planes"][:, target[who[child]], token] = s["planes"][:, source[who[child]].long(), token]
    s["status"].copy_(torch.where(further & ~granted, -3, 0))
    return {"table": table, "len": lens, "ref": ref, "status": s["status"], "planes": s["planes"]}


def _plain_backtrack(s):
    token, parent, out = s["token"], s["parent"], s["out"]
    T, R, K = token.shape
    # the way back in doubling strides: where[t] = the beam at step t that the final beams came by
    hop = parent.long()
    dead = hop < 0
    # suffix composition: after round k, `hop[t]` leads from step t + 2^k - 1 down to step t - 1
    where = torch.arange(K, device=token.device).expand(T, R, K).clone()   # step t's beam of each final beam
    lost = torch.zeros((T, R, K), dtype=torch.bool, device=token.device)
    jump = torch.cat([hop[1:], torch.arange(K, device=token.device).expand(1, R, K)])   # jump[t]: step t+1 -> t
    gone = torch.cat([dead[1:], torch.zeros((1, R, K), dtype=torch.bool, device=token.device)])
    span = 1
    while span < 2 * T:
        # beams of step min(t + 2 * span, T - 1) to step t: first to t + span, then on to t
        far = torch.arange(T, device=token.device) + span
        there = far.clamp(max=T - 1)
        reach = (far <= T - 1)[:, None, None]
        mid = torch.where(reach, jump[there], torch.arange(K, device=token.device))
        mid_gone = torch.where(reach, gone[there], False)
        mid = mid.clamp(min=0)
        gone = mid_gone | gone.gather(2, mid)
        jump = jump.gather(2, mid)
        span *= 2
    where, lost = jump.clamp(min=0), gone | dead.gather(2, jump.clamp(min=0))
    lost = lost.any(0, keepdim=True).expand(T, R, K)
    out.copy_(torch.where(lost, -1, token.gather(2, where)).permute(1, 2, 0))
    return {"out": out}


# ---------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------
def _own_select(s):
    s["plan"](s["logits"])
    return {"score": s["score_out"], "parent": s["parent_out"], "token": s["token_out"]}


def _own_blocks(s):
    m = s["slots"]
    s["tables"].extend(s["new"], m)
    s["tables"].shrink(s["keep"])
    return {"cu": m.cu, "slot": m.slot, "pos": m.pos, "seq": m.seq, "status": s["status"], "table": s["table"],
            "len": s["len"], "ref": s["pool"].ref}


def _own_reorder(s):
    s["tables"].reorder(s["parent"], s["kv"])
    return {"table": s["table"], "len": s["len"], "ref": s["pool"].ref, "status": s["status"], "planes": s["planes"]}


def _own_backtrack(s):
    import paper_2507_16768_b200 as wg
    wg.wg_beam_backtrack(s["token"], s["parent"], s["out"])
    return {"out": s["out"]}


def run(state):
    side = (_own_select, _own_blocks, _own_reorder, _own_backtrack) if own else \
        (_plain_select, _plain_blocks, _plain_reorder, _plain_backtrack)
    return dict(zip(("select", "blocks", "reorder", "backtrack"), side))[state["op"]](state)


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "select":
        N, V = case["R"] * case["K"], case["V"]
        size = 2 if case["dtype"] == "bf16" else 4
        dense = {"literal": 0.0, "text": 1.0, "mixed": 0.25, "none": 1.0}[case["mask"]]
        live = 7 / 8 * 15 / 16       # rows that are neither finished nor given up
        read = N * live * (1.0 if case["norm"] == NORM_FULL else dense)
        few = N * live - read        # rows of which a few scattered 32-byte sectors are read
        nbytes = read * V * size + few * 24 * 32 + case["R"] * case["n_out"] * 12 + N * 8
        if case["mask"] != "none":
            nbytes += N * live * (V + 31) // 32 * 4
        return {"bytes": nbytes, "flops": 4.0 * read * V}
    if case["op"] == "blocks":
        tokens = _step_tokens(case)
        fresh = tokens / case["block"] + (case["S"] if case["new"] > 1 else 0) / 2
        # slots, positions, owners; new entries twice; lengths; the counts of the taken blocks twice
        return {"bytes": tokens * 16 + fresh * 16 + case["S"] * 28 + case["n_blocks"] / 8, "flops": 0.0}
    if case["op"] == "reorder":
        N, K, block = case["R"] * case["K"], case["K"], case["block"]
        held = (0.75 * (case["prompt"] + case["gen"])) / block
        copies = case["R"] * K * (1 - 1 / K) ** K * (block - 1) / block
        return {"bytes": N * held * 4 + copies * case["planes"] * (block / 2) * case["token_elems"] * 2 * 2 + N * 20,
                "flops": 0.0}
    return {"bytes": 12.0 * case["T"] * case["R"] * case["K"], "flops": 0.0}


# ---------------------------------------------------------------------------------------
# 64-bit values
# ---------------------------------------------------------------------------------------
def exact(case, seed):
    """Selection scores from the definition in 64 bits, row by row.  The other operators' outputs
    are whole numbers and moved data: they have no such value."""
    if case["op"] != "select":
        return None
    s = prepare(case, seed)
    R, K, V, n_out = case["R"], case["K"], case["V"], case["n_out"]
    score = s["score"].double().cpu().numpy()
    finished = s["finished"].cpu().numpy()
    best = np.full((R, n_out), -np.inf)
    for r in range(R):
        found = []
        for b in range(K):
            i = r * K + b
            if not score[i] > -np.inf:
                continue
            if finished[i]:
                found.append(np.array([score[i]]))
                continue
            x = s["logits"][i].double()
            if s["bitmask"] is None:
                chosen = x
            else:
                words = np.ascontiguousarray(s["bitmask"][i].cpu().numpy()).view(np.uint8)
                bits = np.unpackbits(words, bitorder="little")[:V]
                chosen = x[torch.from_numpy(np.flatnonzero(bits)).cuda()]
            if not chosen.numel():
                continue
            top = torch.sort(chosen, descending=True).values[:n_out].cpu().numpy()
            if case["norm"] != NORM_NONE:
                y = chosen if case["norm"] == NORM_ALLOWED else x
                high = y.max()
                top = top - float(high + torch.log(torch.exp(y - high).sum()))
            found.append(score[i] + top)
        if found:
            line = np.sort(np.concatenate(found))[::-1][:n_out]
            best[r, :len(line)] = line
    return {"score": torch.from_numpy(best), "parent": None, "token": None}
