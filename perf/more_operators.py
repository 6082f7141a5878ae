"""What the operators on a paged cache's contents are measured on.

Three operators, each in a plain form (elementary torch operations in 32 bits) and through the library's
own calls:

  write   a step's keys, values and queries: queries and keys are rotated by their positions, keys and
          values go to their cache slots, quantised where the cache holds 8 bits
  read    whole sequences read back out of the cache, dense and in 16 bits
  attend  attention of new tokens over their sequences' keys and values, through the block tables

``own`` chooses the side; everything a call casts, gathers or lays out is done inside ``run``.
"""
import math

import torch

own = False

NEG_INF = float("-inf")
LARGEST = {"bf16": 0.0, "fp16": 0.0, "e4m3": 448.0, "int8": 127.0}
HELD = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
MODEL = {"bf16": torch.bfloat16, "fp16": torch.float16}
MOST_VISITED = 64 * 16384 * 8 * 128     # tokens x heads x head size that a case's rows see: the largest listed


# ---------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------
def listed():
    return [
        # a step of four sequences: one launch, all latency
        {"name": "write_step_4", "op": "write", "T": 4, "S": 4, "base": 2000, "Hq": 32, "H": 8, "D": 128, "block": 16,
         "model": "bf16", "held": "bf16", "rot": 128, "inter": False, "factor": 1.0},
        # a step of a full batch at far positions, neighbouring dimensions rotated, 8-bit cache
        {"name": "write_step_512_far", "op": "write", "T": 512, "S": 512, "base": 120000, "Hq": 28, "H": 4, "D": 128,
         "block": 32, "model": "bf16", "held": "e4m3", "rot": 128, "inter": True, "factor": 8.0},
        # prompts of several requests in one go, 8-bit cache
        {"name": "write_prompts_12001", "op": "write", "T": 12001, "S": 7, "base": 0, "Hq": 32, "H": 8, "D": 128,
         "block": 16, "model": "bf16", "held": "e4m3", "rot": 128, "inter": False, "factor": 1.0},
        # as many key heads as query heads, a head size that is no power of two, of which a part is rotated
        {"name": "write_prompts_part", "op": "write", "T": 5000, "S": 3, "base": 500, "Hq": 16, "H": 16, "D": 80,
         "block": 8, "model": "fp16", "held": "fp16", "rot": 32, "inter": False, "factor": 1.0},
        # one request's cache handed to another attention, which takes dense keys and values
        {"name": "read_one", "op": "read", "S": 1, "L": 700, "lens": "even", "H": 8, "D": 128, "block": 16, "model": "bf16",
         "held": "e4m3"},
        # a batch of very different lengths moved out of the cache
        {"name": "read_ragged", "op": "read", "S": 40, "L": 16384, "lens": "ragged", "H": 8, "D": 128, "block": 16,
         "model": "bf16", "held": "int8"},
        # one interactive request
        {"name": "attend_1", "op": "attend", "S": 1, "L": 1000, "lens": "even", "Hq": 32, "H": 8, "D": 128, "block": 16,
         "model": "bf16", "held": "bf16", "window": 0, "new": 1, "beams": 1},
        # a serving batch, one token each
        {"name": "attend_32", "op": "attend", "S": 32, "L": 4096, "lens": "even", "Hq": 32, "H": 8, "D": 128, "block": 16,
         "model": "bf16", "held": "bf16", "window": 0, "new": 1, "beams": 1},
        # long contexts, 8-bit cache: the largest
        {"name": "attend_64_long", "op": "attend", "S": 64, "L": 16384, "lens": "even", "Hq": 32, "H": 8, "D": 128,
         "block": 32, "model": "bf16", "held": "e4m3", "window": 0, "new": 1, "beams": 1},
        # a beam search: the hypotheses of a request share their prompt's blocks
        {"name": "attend_beams_32x8", "op": "attend", "S": 256, "L": 1800, "lens": "even", "Hq": 32, "H": 8, "D": 128,
         "block": 16, "model": "bf16", "held": "bf16", "window": 0, "new": 1, "beams": 8},
        # four drafted tokens a sequence are looked at together, lengths from a few tokens on
        {"name": "attend_drafts_24x4", "op": "attend", "S": 24, "L": 9000, "lens": "ragged", "Hq": 28, "H": 4, "D": 128,
         "block": 64, "model": "bf16", "held": "int8", "window": 0, "new": 4, "beams": 1},
        # a layer that looks back over a window, as many key heads as query heads
        {"name": "attend_window_48", "op": "attend", "S": 48, "L": 8000, "lens": "ragged", "Hq": 16, "H": 16, "D": 64,
         "block": 16, "model": "fp16", "held": "fp16", "window": 1024, "new": 1, "beams": 1},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["write", "read", "attend", "attend", "attend"])
    model = rng.choice(["bf16", "bf16", "fp16"])
    held = rng.choice([model, "e4m3"] if op == "write" else [model, "e4m3", "int8"])
    H = rng.choice([1, 2, 4, 8, 16])
    D = rng.choice([64, 80, 96, 128, 128, 256])
    case = {"op": op, "H": H, "D": D, "block": rng.choice([1, 8, 16, 16, 32, 64, 100]), "model": model, "held": held}
    if op == "write":
        T = _log_int(rng, 1, max(2, 12001 * 8 * 128 // (max(H, 8) * max(D, 128))))
        S = T if rng.random() < 0.4 else _log_int(rng, 1, min(T, 32))
        Hq = H * rng.choice([q for q in (1, 2, 4, 7, 8) if H * q <= 32])
        return dict(case, T=T, S=S, base=_log_int(rng, 1, 120000), Hq=Hq, rot=rng.choice([D, D, D // 32 * 16, 0]),
                    inter=rng.random() < 0.5, factor=rng.choice([1.0, 4.0, 8.0]))
    L = _log_int(rng, 1, 16384)
    lens = rng.choice(["even", "ragged"])
    if op == "read":
        L = max(1, min(L, 40 * 1536 * 8 * 128 // (H * D)))
        return dict(case, S=_log_int(rng, 1, max(1, min(64, 40 * 512 * 8 * 128 // (L * H * D)))), L=L, lens=lens)
    new, beams = rng.choice([(1, 1), (1, 1), (2, 1), (5, 1), (1, 2), (1, 4), (1, 5), (1, 12)])
    rows = max(1, min(300, MOST_VISITED // (L * H * D * 2)))
    S = max(1, _log_int(rng, 1, rows) // (new * beams)) * beams
    Hq = H * rng.choice([q for q in (1, 2, 4, 7, 8, 16, 24) if H * q <= 48])
    return dict(case, S=S, L=L, lens=lens, Hq=Hq, window=rng.choice([0, 0, 0, 1, 300, 4096]), new=new, beams=beams)


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _lengths(case):
    """The lengths of a case's sequences (of its requests, where beams share a prompt); one in sixteen has ended."""
    n, L = case["S"] // case.get("beams", 1), case["L"]
    even = case["lens"] == "even"
    part = [(i + 0.5) / n for i in range(n)]
    lens = [max(1, round(L * (0.75 + 0.25 * u) if even else L ** u)) for u in part]
    lens[-1] = L
    return [0 if i % 16 == 7 else x for i, x in enumerate(lens)]


def _quantise(x, held):
    """(codes, scale) of vectors along the last axis: scale = largest magnitude / the largest code, in fp32."""
    if not LARGEST[held]:
        return x.to(HELD[held]), None
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    small = top < 2.0 ** -100
    codes = x * torch.where(small, 0.0, LARGEST[held] / torch.where(small, 1.0, top))
    codes = codes.to(HELD[held]) if held == "e4m3" else torch.round(codes).to(torch.int8)
    return codes, torch.where(small, 1.0, top / LARGEST[held])[..., 0]


def _cache(case, g, n_blocks):
    """A cache that holds something in every slot: keys with a few strong dimensions, values of changing size."""
    shape = (n_blocks, case["block"], case["H"], case["D"])
    strong = torch.exp(0.5 * torch.randn(shape[2:], device="cuda", generator=g))
    planes = {}
    for what in ("keys", "values"):
        data = torch.empty(shape, dtype=HELD[case["held"]], device="cuda")
        scale = torch.empty(shape[:3], dtype=torch.float32, device="cuda") if LARGEST[case["held"]] else None
        step = max(1, (1 << 26) // (shape[1] * shape[2] * shape[3]))
        for a in range(0, n_blocks, step):
            b = min(n_blocks, a + step)
            x = torch.randn((b - a,) + shape[1:], device="cuda", generator=g)
            if what == "keys":
                x = x * strong
            else:
                x = x * torch.exp(0.7 * torch.randn(x.shape[:3] + (1,), device="cuda", generator=g))
            codes, s = _quantise(x, case["held"])
            data[a:b] = codes
            if scale is not None:
                scale[a:b] = s
        planes[what], planes[what + "_scale"] = data, scale
    return planes


def _tables(case, g):
    """(lens, table, n_blocks): sequences on blocks in no order; the beams of a request share whole blocks of the
    first 15/16 of it, which were its prompt."""
    beams, block = case.get("beams", 1), case["block"]
    lens = torch.tensor(_lengths(case), device="cuda")
    lens = lens[torch.randperm(lens.numel(), device="cuda", generator=g)]
    n = lens.numel()
    shared = lens * 15 // 16 // block if beams > 1 else torch.zeros_like(lens)
    held = (lens + block - 1) // block
    private = held - shared
    M = max(1, -(-case["L"] // block)) + 1
    col = torch.arange(M, device="cuda")
    total = int(shared.sum() + private.sum() * beams)
    n_blocks = total + max(4, total // 50)
    ids = torch.randperm(n_blocks, device="cuda", generator=g)
    of_prompt = (torch.cumsum(shared, 0) - shared)[:, None, None] + col
    flat = private[:, None].expand(n, beams).reshape(-1)
    of_beam = int(shared.sum()) + (torch.cumsum(flat, 0) - flat).view(n, beams, 1) + col - shared[:, None, None]
    at = torch.where(col < shared[:, None, None], of_prompt, of_beam).clamp(0, n_blocks - 1)
    table = torch.where(col < held[:, None, None], ids[at], -1).to(torch.int32).view(n * beams, M).contiguous()
    return lens[:, None].expand(n, beams).reshape(-1).to(torch.int32).contiguous(), table, n_blocks


def _frequencies(case):
    """Rotations per position in 64 bits.  With a factor, dimensions that turn less than once over 8192 positions are
    slowed down by it, those that turn more than four times are not, and the ones between in part."""
    j = torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda")
    f = 10000.0 ** (-2.0 * j / max(1, case["rot"]))
    if case["factor"] != 1.0:
        keep = ((8192.0 * f / (2.0 * math.pi) - 1.0) / 3.0).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / case["factor"])
    return f


def _prepare_write(case, seed):
    g = _generator(seed)
    T, S, Hq, H, D, block = (case[k] for k in ("T", "S", "Hq", "H", "D", "block"))
    # the sequences' new tokens one after the other, as slot maps have them
    begin = torch.arange(S + 1, device="cuda") * T // S
    t = torch.arange(T, device="cuda")
    seq = torch.searchsorted(begin[1:].contiguous(), t, right=True)
    start = torch.randint(0, case["base"] + 1, (S,), device="cuda", generator=g)
    pos = (start[seq] + t - begin[seq]).to(torch.int32)
    n_blocks = T // block + 3
    slot = torch.randperm(n_blocks * block, device="cuda", generator=g)[:T]
    # a token in 32 has no slot: its sequence was refused
    slot = torch.where(torch.rand(T, device="cuda", generator=g) < 1 / 32, -1, slot)
    whole = torch.randn((T, (Hq + 2 * H) * D), device="cuda", generator=g)       # one projection's output
    whole = (whole * torch.exp(0.5 * torch.randn(whole.shape[1], device="cuda", generator=g))).to(MODEL[case["model"]])
    q, k, v = (x.view(T, -1, D) for x in whole.split([Hq * D, H * D, H * D], 1))
    s = dict(_cache(case, g, n_blocks), op="write", q=q, k=k, v=v, slot=slot, pos=pos, held=case["held"], rot=case["rot"],
             inter=case["inter"], q_out=torch.zeros((T, Hq, D), dtype=q.dtype, device="cuda"))
    n_pos = case["base"] + T // S + 2
    if own:
        import paper_2507_16768_b200 as wg
        s["cache"] = wg.KvCache(s["keys"], s["values"], s["keys_scale"], s["values_scale"])
        s["slots"] = wg.SlotMap(S, T)
        for to, x in ((s["slots"].cu, begin), (s["slots"].slot, slot), (s["slots"].pos, pos), (s["slots"].seq, seq)):
            to.copy_(x)
        how = {} if case["factor"] == 1.0 else {"factor": case["factor"], "low": 1.0, "high": 4.0, "original": 8192}
        s["rope"] = wg.Rope(n_pos, case["rot"], interleaved=case["inter"], **how) if case["rot"] else None
    else:
        angle = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * _frequencies(case)
        s["cos"], s["sin"] = torch.cos(angle).float(), torch.sin(angle).float()
    return s


def _prepare_read(case, seed):
    g = _generator(seed)
    lens, table, n_blocks = _tables(case, g)
    cu = torch.zeros(case["S"] + 1, dtype=torch.int32, device="cuda")
    cu[1:] = torch.cumsum(lens, 0)
    rows = sum(_lengths(case)) + 3
    out = [torch.zeros((rows, case["H"], case["D"]), dtype=MODEL[case["model"]], device="cuda") for _ in range(2)]
    s = dict(_cache(case, g, n_blocks), op="read", lens=lens, table=table, cu=cu, k_out=out[0], v_out=out[1])
    if own:
        import paper_2507_16768_b200 as wg
        s["cache"] = wg.KvCache(s["keys"], s["values"], s["keys_scale"], s["values_scale"])
        s["pool"] = wg.KvPool(n_blocks, case["block"], case["S"])
        s["tables"] = wg.KvTables(s["pool"], table, lens)
    return s


def _prepare_attend(case, seed):
    g = _generator(seed)
    S, new = case["S"], case["new"]
    lens, table, n_blocks = _tables(case, g)
    T = S * new
    seq = torch.arange(T, device="cuda", dtype=torch.int32) // new
    pos = lens[seq] - new + torch.arange(T, device="cuda", dtype=torch.int32) % new
    pos = torch.where(pos < 0, -1, pos).to(torch.int32)        # (a sequence of fewer tokens than were drafted)
    q = torch.randn((T, case["Hq"], case["D"]), device="cuda", generator=g) * 1.5
    s = dict(_cache(case, g, n_blocks), op="attend", q=q.to(MODEL[case["model"]]), lens=lens, table=table, seq=seq, pos=pos,
             window=case["window"], new=new, group=max(new, case["beams"]))
    if own:
        import paper_2507_16768_b200 as wg
        s["cache"] = wg.KvCache(s["keys"], s["values"], s["keys_scale"], s["values_scale"])
        s["pool"] = wg.KvPool(n_blocks, case["block"], S)
        s["tables"] = wg.KvTables(s["pool"], table, lens)
        s["attend"] = wg.Attend(T, case["Hq"], case["H"], case["D"])
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((T, case["Hq"]), dtype=torch.float32, device="cuda")
        s["slots"] = None
        if new > 1:
            s["slots"] = wg.SlotMap(S, T)
            slot = table[seq.long(), (pos // case["block"]).clamp(min=0).long()].long() * case["block"] + pos % case["block"]
            for to, x in ((s["slots"].cu, torch.arange(S + 1, device="cuda") * new), (s["slots"].seq, seq),
                          (s["slots"].pos, pos), (s["slots"].slot, torch.where(pos < 0, -1, slot))):
                to.copy_(x)
    return s


def prepare(case, seed):
    return {"write": _prepare_write, "read": _prepare_read, "attend": _prepare_attend}[case["op"]](case, seed)


# ---------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------
def _rotated(x, cos, sin, rot, inter):
    """x in 32 bits with its first `rot` dimensions turned in pairs: (i, i + rot/2), or (2i, 2i + 1)."""
    x = x.float()
    if not rot:
        return x
    part = x[..., :rot]
    a, b = (part[..., 0::2], part[..., 1::2]) if inter else (part[..., :rot // 2], part[..., rot // 2:])
    turned = (a * cos - b * sin, b * cos + a * sin)
    turned = torch.stack(turned, -1).flatten(-2) if inter else torch.cat(turned, -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_write(s):
    at = s["pos"].long()
    cos, sin = s["cos"][at][:, None], s["sin"][at][:, None]
    ok = s["slot"] >= 0
    q = _rotated(s["q"], cos, sin, s["rot"], s["inter"]).to(s["q"].dtype)
    s["q_out"].copy_(torch.where(ok[:, None, None], q, s["q_out"]))
    slot = s["slot"][ok]
    for what, x in (("keys", _rotated(s["k"], cos, sin, s["rot"], s["inter"])), ("values", s["v"])):
        codes, scale = _quantise(x[ok], s["held"])
        _slots(s[what])[slot] = _slots(codes, 0)
        if scale is not None:
            s[what + "_scale"].view(-1, scale.shape[-1])[slot] = scale
    return _written(s)


def _slots(x, dims=1):
    """The slots of a plane one after the other; 8-bit floats, which torch does not index, as bytes."""
    x = x.flatten(0, dims)
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _written(s):
    return {"q": s["q_out"], "keys": s["keys"], "values": s["values"], "keys_scale": s["keys_scale"],
            "values_scale": s["values_scale"]}


def _gathered(s, what, slot):
    """Keys or values of the slots, in 32 bits."""
    x = _slots(s[what])[slot].view(s[what].dtype).float()
    if s[what + "_scale"] is not None:
        x.mul_(s[what + "_scale"].view(-1, x.shape[-2])[slot][..., None])
    return x


def _plain_read(s):
    rows = torch.arange(s["k_out"].shape[0], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["cu"][1:].contiguous(), rows, right=True).clamp(max=s["lens"].numel() - 1)
    p, block = (rows - s["cu"][seq]).long(), s["keys"].shape[1]
    inside = rows < s["cu"][-1]
    slot = s["table"][seq, (p // block).clamp(max=s["table"].shape[1] - 1)].long() * block + p % block
    for what, out in (("keys", s["k_out"]), ("values", s["v_out"])):
        x = _gathered(s, what, torch.where(inside, slot, 0)).to(out.dtype)
        out.copy_(torch.where(inside[:, None, None], x, out))
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain_attend(s):
    T, Hq, D = s["q"].shape
    block, H = s["keys"].shape[1], s["keys"].shape[2]
    L = max(1, int(s["lens"].max()))
    p = torch.arange(L, device="cuda")
    entry = s["table"][:, p // block][s["seq"].long()].long()
    seen = (p[None, :] <= s["pos"][:, None]) & (entry >= 0)
    if s["window"]:
        seen = seen & (p[None, :] > s["pos"][:, None] - s["window"])
    slot = torch.where(entry < 0, 0, entry) * block + p % block
    k = _gathered(s, "keys", slot).permute(0, 2, 3, 1)                       # [T, H, D, L]
    q = s["q"].float().view(T, H, Hq // H, D)
    x = torch.matmul(q, k) / math.sqrt(D)
    del k
    x = torch.where(seen[:, None, None, :], x, NEG_INF)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top > NEG_INF, top, 0.0)
    w = torch.exp(x - top)
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w, _gathered(s, "values", slot).permute(0, 2, 1, 3))
    out = torch.where(total > 0, out / total, 0.0)
    return {"out": out.reshape(T, Hq, D).to(s["q"].dtype), "lse": (top + torch.log(total)).reshape(T, Hq)}


# ---------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------
def _own_write(s):
    s["cache"].write(s["k"], s["v"], s["slots"], rope=s["rope"], q=s["q"], q_out=s["q_out"])
    return _written(s)


def _own_read(s):
    s["cache"].read(s["tables"], s["cu"], s["k_out"], s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_attend(s):
    s["attend"](s["q"], s["cache"], s["tables"], s["out"], slots=s["slots"], window=s["window"], group=s["group"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    side = (_own_write, _own_read, _own_attend) if own else (_plain_write, _plain_read, _plain_attend)
    return dict(zip(("write", "read", "attend"), side))[state["op"]](state)


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    H, D = case["H"], case["D"]
    wide = bool(LARGEST[case["held"]])
    token = 2 * H * (D + 4 if wide else 2 * D)         # bytes of a token's keys and values in the cache
    if case["op"] == "write":
        T, Hq = case["T"], case["Hq"]
        angles = min(T, case["base"] + T // case["S"]) * case["rot"] * 4
        return {"bytes": T * 31 / 32 * (4.0 * Hq * D + 4.0 * H * D + token) + 12.0 * T + angles,
                "flops": T * (3.0 * case["rot"] * (Hq + H) + (4.0 * H * D if wide else 0.0))}
    lens = _lengths(case)
    if case["op"] == "read":
        return {"bytes": sum(lens) * (token + 4.0 * H * D + 4.0 / case["block"]), "flops": 2.0 * H * D * sum(lens) if wide else 0.0}
    beams, new, window = case["beams"], case["new"], case["window"] or 1 << 40
    read = seen = 0.0
    for n in lens:
        far = min(n, window + new - 1)
        shared = min(far, max(0, n * 15 // 16 // case["block"] * case["block"] - (n - far))) if beams > 1 else 0
        read += shared + beams * (far - shared)
        seen += beams * sum(min(max(0, n - i), window) for i in range(new))
    T = case["S"] * new
    return {"bytes": read * (token + 4.0 / case["block"]) + T * case["Hq"] * (4.0 * D + 4.0) + 8.0 * T,
            "flops": 4.0 * seen * case["Hq"] * D}


# ---------------------------------------------------------------------------------------
# 64-bit values
# ---------------------------------------------------------------------------------------
def _rounded_e4m3(y):
    """The nearest of the format's values to y (64 bits): three fraction bits down to 2^-6, steps of 2^-9 below."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(y / step) * step


def _exact_write(case, s):
    T, D, rot, held = case["T"], case["D"], case["rot"], case["held"]
    pos = s["pos"].double()
    result = {"q": s["q_out"].double(), "keys": s["keys"].double(), "values": s["values"].double()}
    for what in ("keys", "values"):
        result[what + "_scale"] = None if s[what + "_scale"] is None else s[what + "_scale"].double()
    ok = torch.nonzero(s["slot"] >= 0)[:, 0]
    block, offset = s["slot"][ok] // case["block"], s["slot"][ok] % case["block"]
    f = _frequencies(case)
    for what, x in (("q", s["q"]), ("keys", s["k"]), ("values", s["v"])):
        y = x[ok].double().clone()
        if what != "values":
            for j in range(rot // 2):
                a, b = (2 * j, 2 * j + 1) if case["inter"] else (j, j + rot // 2)
                z = torch.polar(torch.ones_like(pos[ok]), pos[ok] * f[j])[:, None] * torch.complex(y[..., a], y[..., b])
                y[..., a], y[..., b] = z.real, z.imag
        if what == "q":
            result["q"][ok] = y
            continue
        if LARGEST[held]:
            scale = torch.linalg.vector_norm(y, float("inf"), -1) / LARGEST[held]
            result[what + "_scale"][block, offset] = scale
            y = _rounded_e4m3(y / scale[..., None])
        result[what][block, offset] = y
    return result


def _sequence64(case, s, what, row, first, last):
    """Keys or values of positions first .. last - 1 of a sequence: [H, n, D] in 64 bits."""
    p = torch.arange(first, last, device="cuda")
    b = s["table"][row].long()[p // case["block"]]
    x = s[what].view(torch.uint8)[b, p % case["block"]].view(s[what].dtype).double()
    if s[what + "_scale"] is not None:
        x = x * s[what + "_scale"][b, p % case["block"]].double().unsqueeze(-1)
    return x.transpose(0, 1)


def _exact_read(case, s):
    out = {"k": s["k_out"].double(), "v": s["v_out"].double()}
    at = 0
    for row, n in enumerate(s["lens"].tolist()):
        for key, what in (("k", "keys"), ("v", "values")):
            out[key][at:at + n] = _sequence64(case, s, what, row, 0, n).transpose(0, 1)
        at += n
    return out


def _exact_attend(case, s):
    T, Hq, D = s["q"].shape
    H = case["H"]
    out = torch.zeros((T, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hq), NEG_INF, dtype=torch.float64, device="cuda")
    for t, (row, p) in enumerate(zip(s["seq"].tolist(), s["pos"].tolist())):
        if p < 0:
            continue
        first = max(0, p - case["window"] + 1) if case["window"] else 0
        k, v = (_sequence64(case, s, what, row, first, p + 1) for what in ("keys", "values"))
        x = torch.bmm(k, s["q"][t].double().view(H, Hq // H, D).transpose(1, 2)).transpose(1, 2) * D ** -0.5
        lse[t] = torch.logsumexp(x, -1).view(-1)
        out[t] = torch.bmm(torch.softmax(x, -1), v).view(Hq, D)
    return {"out": out, "lse": lse}


def exact(case, seed):
    """The definitions in 64 bits, token by token and dimension by dimension; e4m3 codes as the values they are."""
    return {"write": _exact_write, "read": _exact_read, "attend": _exact_attend}[case["op"]](case, prepare(case, seed))
