"""Attention with a sliding window and sinks over the paged cache, and the cache's pages: what a streaming server calls.

Every case has a plain form in elementary torch operations (``own`` false) and the calls of this library (``own`` true).
The cache, the block table and the pool are kept from call to call; a pass is one call, or the few calls that belong
together, with what the program has in hand.  Caches are in the library's granule layout (``include/coopt.h``).

Kinds of pass:
  decode    window_decode: one query token per sequence, with ``append`` its K/V written first
  prefill   window_prefill: runs of query tokens behind cached ones, or whole prompts
  copy      pages_copy: whole blocks of all layers copied inside their caches
  branch    pages_release of the old branches, pages_fork of new ones, pages_reserve of room for their next tokens
  compact   pages_compact: the blocks in use moved to the front of the pool, table and counts renumbered
"""
import math
import random

import torch

own = False

BLOCK = 16
FORMATS = {"e4m3": 0, "bf16": 1, "e5m2": 2}
FP8 = {"e4m3": (torch.float8_e4m3fn, 448.0), "e5m2": (torch.float8_e5m2, 57344.0)}


def _attention(name, kind, batch, lo, hi, hq, hkv, dim, window, sinks, **more):
    """``lo`` .. ``hi``: context lengths after the call, spread over the sequences (drawn from ``mix``); ``new``: query
    tokens of a sequence (0: the whole prompt)."""
    c = {"name": name, "kind": kind, "batch": batch, "lo": lo, "hi": hi, "hq": hq, "hkv": hkv, "dim": dim, "window": window,
         "sinks": sinks, "format": "e4m3", "new": 1, "append": False, "mix": 1}
    c.update(more)
    return c


def _pages(name, kind, layers, hkv, dim, blocks, rows, **more):
    c = {"name": name, "kind": kind, "layers": layers, "hkv": hkv, "dim": dim, "blocks": blocks, "rows": rows, "format": "e4m3", "mix": 1}
    c.update(more)
    return c


def listed():
    return [
        # one user's stream, far past its window: nothing to fill the GPU with, all latency
        _attention("stream_one", "decode", 1, 20011, 20011, 40, 8, 128, 1024, 4, mix=3),
        # a full batch of long streams, each with its new token: the step that a streaming server makes per layer
        _attention("stream_step_32", "decode", 32, 2500, 90000, 40, 8, 128, 2048, 4, append=True, mix=5),
        # a small model, no quantisation, contexts on both sides of an odd window, more sinks than a block holds
        _attention("stream_bf16_dim64", "decode", 70, 3, 6000, 16, 4, 64, 1500, 19, format="bf16", mix=7),
        # chunks of prompts behind a long stream
        _attention("chunks_behind_stream", "prefill", 8, 5000, 40000, 40, 8, 128, 1024, 4, new=512, mix=9),
        # whole prompts of a small model, ragged, several windows long
        _attention("prompts_dim64", "prefill", 4, 900, 2900, 32, 8, 64, 500, 8, new=0, mix=11),
        # a few drafted tokens of each request to be verified, the other FP8 format
        _attention("drafts_e5m2", "prefill", 24, 100, 9000, 16, 2, 128, 777, 33, format="e5m2", new=5, mix=13),
        # two blocks of a beam moved, of four layers: the smallest call
        _pages("copy_few", "copy", 4, 8, 128, 300, 1, pairs=2, mix=15),
        # the blocks of a preempted group moved, of sixteen layers
        _pages("copy_many", "copy", 16, 8, 128, 1500, 1, pairs=700, mix=17),
        # a few parents branched in four, the branches of the turn before dropped
        _pages("branch_few", "branch", 8, 8, 128, 700, 24, children=8, lo=40, hi=900, grow=17, mix=19),
        # best-of-n over a large batch and pool, small heads
        _pages("branch_many", "branch", 12, 4, 64, 20000, 192, children=128, lo=100, hi=2600, grow=40, mix=21),
        # a pool that a day of traffic has left in holes
        _pages("compact_large", "compact", 12, 8, 128, 2500, 96, lo=1, hi=500, holes=0.4, mix=23),
        # a small pool of many short requests
        _pages("compact_small", "compact", 2, 2, 64, 900, 64, lo=1, hi=150, holes=0.15, mix=25),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: any kind, format, group size 1 to 8 and head dim, windows and sinks of odd sizes."""
    while True:
        kind = rng.choice(["decode", "decode", "prefill", "prefill", "copy", "branch", "compact"])
        dim, hkv = rng.choice([128, 128, 64]), rng.choice([1, 2, 4, 8])
        mix = rng.randrange(1, 100000)
        fmt = rng.choice(["e4m3", "e4m3", "e5m2", "bf16"])
        if kind in ("decode", "prefill"):
            hi = _log(rng, 20, 100000 if kind == "decode" else 40000)
            c = _attention("", kind, _log(rng, 1, 96 if kind == "decode" else 24), rng.choice([hi, max(1, hi // 2), max(1, hi // 30)]), hi,
                           hkv * rng.choice([1, 2, 4, 5, 7, 8]), hkv, dim, _log(rng, 1, 4096), rng.choice([0, 1, 4, _log(rng, 5, 200)]), format=fmt, mix=mix)
            if kind == "decode":
                c["append"] = rng.random() < 0.5
                dear = work(c)["bytes"] > 1.6e8
            else:
                c["format"] = rng.choice(["e4m3", "e5m2"])
                c["new"] = rng.choice([0, _log(rng, 2, 1024), _log(rng, 2, 1024)])
                lens, new = _lens(c), _new(c)
                span = max(min(L, n + c["window"] + c["sinks"] + 48) for L, n in zip(lens, new))
                dear = work(c)["flops"] > 9e10 or c["batch"] * c["hq"] * max(new) * span > 6e8
        else:
            c = _pages("", kind, rng.choice([1, 2, 5, 8, 16, 24]), hkv, dim, _log(rng, 60, 30000), _log(rng, 4, 200), format=fmt, mix=mix)
            if kind == "copy":
                c["pairs"] = _log(rng, 1, max(2, c["blocks"] // 2))
            else:
                hi = _log(rng, 2, max(8, c["blocks"] * BLOCK // c["rows"]))
                c.update(lo=max(1, hi // rng.choice([2, 10, 50])), hi=hi)
            if kind == "branch":
                c.update(children=max(1, c["rows"] // rng.choice([2, 3])), grow=_log(rng, 1, 100))
            if kind == "compact":
                c["holes"] = round(rng.uniform(0.02, 0.6), 2)
            dear = c["layers"] * c["blocks"] * c["hkv"] * _granule(c) > 2.2e9 or work(c)["bytes"] > 7e8
            if kind == "branch":                                      # (a pool with room for its branches)
                dear = dear or c["children"] * (c["grow"] // BLOCK + 3) > 0.3 * c["blocks"]
        del c["name"]
        if not dear:
            return c


# ---- sizes -------------------------------------------------------------------------------------------------------

def _granule(c):
    return 2 * BLOCK * c["dim"] * 2 if c["format"] == "bf16" else 2 * BLOCK * c["dim"] + 128


def _used(c):
    """Bytes of a granule that hold anything."""
    return _granule(c) if c["format"] == "bf16" else 2 * BLOCK * c["dim"] + 32


def _lens(c):
    rng = random.Random(c["mix"])
    return [rng.randint(c["lo"], c["hi"]) for _ in range(c["batch"])]


def _new(c):
    """Query tokens of each sequence."""
    if c["kind"] == "decode":
        return [1] * c["batch"]
    rng = random.Random(c["mix"] + 1)
    return [L if c["new"] == 0 else min(L, rng.randint(max(1, c["new"] // 3), c["new"])) for L in _lens(c)]


def _held(c, L, n):
    """Block positions of a sequence that the call may look at: those with sinks, and those from the first window on."""
    sinks, first, end = -(-c["sinks"] // BLOCK), max(0, L - n + 1 - c["window"]) // BLOCK, -(-L // BLOCK)
    return list(range(min(sinks, first, end))) + list(range(min(first, end), end)) if first > sinks else list(range(end))


def _rows(c):
    """Lengths of the rows of a pool, and the number of rows that hold something: the last ``children`` rows are the branches."""
    rng = random.Random(c["mix"])
    n = c["rows"] - c.get("children", 0)
    room = int(c["blocks"] * (1 - c.get("holes", 0.3)))          # blocks that may be in use at most
    lens = []
    for _ in range(n):
        L = rng.randint(c["lo"], c["hi"])
        need = -(-L // BLOCK)
        lens.append(L if need <= room else 0)
        room -= need if need <= room else 0
    return lens


def _branches(c):
    """(parent row, its length) of every branch; a branch needs room for a copied block and for ``grow`` more tokens."""
    rng = random.Random(c["mix"] + 1)
    lens = _rows(c)
    return [(p, lens[p]) for p in (rng.randrange(len(lens)) for _ in range(c["children"]))]


def _moves(c):
    """Blocks that a compaction moves: as many as there are holes below the count of used blocks."""
    used = sum(-(-L // BLOCK) for L in _rows(c))
    place = random.Random(c["mix"] + 2).sample(range(c["blocks"]), used)
    return sum(1 for x in place if x >= used)


def work(case):
    c, kind = case, case["kind"]
    if kind in ("decode", "prefill"):
        lens, new, hkv, hq, d = _lens(c), _new(c), c["hkv"], c["hq"], c["dim"]
        token = 2 * hkv * d * (2 if c["format"] == "bf16" else 1)
        scale = 0 if c["format"] == "bf16" else 8 * hkv
        read = pairs = 0
        for L, n in zip(lens, new):
            t = L - n                                                 # position of the first query
            first = max(0, t + 1 - c["window"])                       # .. and of its window
            read += (min(c["sinks"], first) + L - first) * token + len(_held(c, L, n)) * (scale + 4) + 4
            # the visible keys of positions t .. L - 1: min(p + 1, window) in the window, min(sinks, p + 1 - window) before it
            W, S = c["window"], c["sinks"]
            tri = lambda x: x * (x + 1) // 2 if x > 0 else 0          # noqa: E731
            upto = lambda e, cap: tri(min(e, cap)) + max(0, e - cap) * cap     # sum over x = 1 .. e of min(x, cap)    # noqa: E731
            pairs += upto(L, W) - upto(t, W) + upto(max(0, L - W), S) - upto(max(0, t - W), S)
        io = sum(new) * 2 * hq * d * 2 + (c["batch"] * (2 * hkv * d * 2 + 8 + token + scale) if c["append"] else 0)
        return {"bytes": read + io, "flops": 4 * d * hq * pairs}
    block = c["layers"] * c["hkv"] * _used(c)
    if kind == "copy":
        return {"bytes": c["pairs"] * (2 * block + 8), "flops": 0}
    width = _width(c)
    if kind == "branch":
        tails = sum(1 for _, L in _branches(c) if L % BLOCK)
        shared = sum(L // BLOCK for _, L in _branches(c))
        # the copied blocks; the counts looked through once; the branches' rows dropped and written; the counts of shared blocks
        return {"bytes": tails * 2 * block + c["blocks"] * 4 + c["children"] * (3 * width * 4 + 24) + shared * 16, "flops": 0}
    return {"bytes": _moves(c) * 2 * block + 2 * c["blocks"] * 4 + 2 * c["rows"] * width * 4, "flops": 0}


def _width(c):
    return -(-(c["hi"] + c.get("grow", 0)) // BLOCK) + 1


# ---- the cache's layout ------------------------------------------------------------------------------------------

def _unpack(g, c):
    """Granules uint8 [..., granule] -> (codes or values [..., 2, 16, D] in the cache's own type, scales fp32 [..., 2] or None)."""
    d, lead = c["dim"], g.shape[:-1]
    if c["format"] == "bf16":
        x = g.contiguous().view(torch.bfloat16)
        k, v = x[..., :BLOCK * d], x[..., BLOCK * d:]
        n = len(lead)
        at = lambda *i: tuple(range(n)) + tuple(n + j for j in i)     # noqa: E731
        # K: [token / 8][dim / 32][token % 8][dim % 8 / 2][dim / 16 % 2][dim / 8 % 2][dim % 2]
        k = k.reshape(*lead, 2, d // 32, 8, 4, 2, 2, 2).permute(at(0, 2, 1, 4, 5, 3, 6)).reshape(*lead, BLOCK, d)
        # V: [dim / 16][dim % 8][token % 8 / 2][dim / 8 % 2][token / 8][token % 2]
        v = v.reshape(*lead, d // 16, 8, 4, 2, 2, 2).permute(at(4, 2, 5, 0, 3, 1)).reshape(*lead, BLOCK, d)
        return torch.stack([k, v], dim=-3), None
    k = g[..., :BLOCK * d].reshape(*lead, 2, d // 16, 8, 16).transpose(-3, -2).reshape(*lead, BLOCK, d)
    v = g[..., BLOCK * d:2 * BLOCK * d].reshape(*lead, d, BLOCK).transpose(-2, -1)
    scales = g[..., 2 * BLOCK * d:2 * BLOCK * d + 8].contiguous().view(torch.float32)
    return torch.stack([k, v], dim=-3).contiguous().view(FP8[c["format"]][0]), scales


def _pack(x, scales, c):
    """The reverse: granules without their padding, uint8 [..., used bytes]."""
    d, lead = c["dim"], x.shape[:-3]
    k, v = x[..., 0, :, :], x[..., 1, :, :]
    if c["format"] == "bf16":
        n = len(lead)
        at = lambda *i: tuple(range(n)) + tuple(n + j for j in i)     # noqa: E731
        k = k.reshape(*lead, 2, 8, d // 32, 2, 2, 4, 2).permute(at(0, 2, 1, 5, 3, 4, 6)).reshape(*lead, BLOCK * d)
        v = v.reshape(*lead, 2, 4, 2, d // 16, 2, 8).permute(at(3, 5, 1, 4, 0, 2)).reshape(*lead, BLOCK * d)
        return torch.cat([k, v], dim=-1).contiguous().view(torch.uint8)
    k, v = k.view(torch.uint8), v.view(torch.uint8)
    k = k.reshape(*lead, 2, 8, d // 16, 16).transpose(-3, -2).reshape(*lead, BLOCK * d)
    v = v.transpose(-2, -1).reshape(*lead, BLOCK * d)
    head = torch.zeros(*lead, 32, dtype=torch.uint8, device=x.device)
    head[..., :8] = scales.contiguous().view(torch.uint8)
    return torch.cat([k, v, head], dim=-1)


# ---- inputs ------------------------------------------------------------------------------------------------------

def _values(gen, rows, heads, dim, loud):
    """N(0, 1) in bf16; K and V of earnest models have a few loud channels, which is what block scales are for."""
    x = torch.randn(rows, heads, dim, generator=gen, device="cuda")
    if loud:
        at = torch.rand(heads, dim, generator=gen, device="cuda").topk(2, dim=1).indices
        x = x * torch.ones(heads, dim, device="cuda").scatter_(1, at, 20.0)
    return x.to(torch.bfloat16)


def _filled_cache(gen, blocks, c):
    """A cache whose every block holds sixteen tokens."""
    hkv, d = c["hkv"], c["dim"]
    cache = torch.zeros(blocks, hkv, _granule(c), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (hkv * d * 2 * BLOCK))
    loud = torch.ones(2, hkv, d, device="cuda").scatter_(2, torch.rand(2, hkv, d, generator=gen, device="cuda").topk(2, dim=2).indices, 20.0)
    for b in range(0, blocks, step):
        n = min(step, blocks - b)
        x = torch.randn(n, hkv, 2, BLOCK, d, generator=gen, device="cuda") * loud.transpose(0, 1)[None, :, :, None, :]
        x = x.to(torch.bfloat16)
        if c["format"] == "bf16":
            cache[b:b + n] = _pack(x, None, c)
        else:
            kind, most = FP8[c["format"]]
            scale = x.float().abs().amax(dim=(-2, -1)) / most
            cache[b:b + n, :, :_used(c)] = _pack((x.float() / scale[..., None, None]).to(kind), scale, c)
    return cache


def prepare(case, seed):
    c, gen = case, torch.Generator(device="cuda").manual_seed(seed)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")     # noqa: E731
    if c["kind"] in ("decode", "prefill"):
        lens, new = _lens(c), _new(c)
        held = [_held(c, L, n) for L, n in zip(lens, new)]
        need = sum(len(h) for h in held)
        blocks = need + max(1, need // 10)
        place = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32).cpu()
        table = torch.full((c["batch"], max(-(-L // BLOCK) for L in lens)), -1, dtype=torch.int32)
        at = 0
        for b, h in enumerate(held):
            table[b, torch.tensor(h, dtype=torch.long)] = place[at:at + len(h)]
            at += len(h)
        s = {"case": c, "cache": _filled_cache(gen, blocks, c), "blocks": blocks, "table": table.cuda(), "lens": ints(lens), "scale": 1.0 / math.sqrt(c["dim"]),
             "q": _values(gen, sum(new), c["hq"], c["dim"], False)}
        s["out"] = torch.empty_like(s["q"])
        if c["kind"] == "prefill":
            s["cu"] = torch.cat([ints([0]), ints(new).cumsum(0).to(torch.int32)])
            s["longest"] = max(new)
        if c["append"]:
            s["k"], s["v"] = _values(gen, c["batch"], c["hkv"], c["dim"], True), _values(gen, c["batch"], c["hkv"], c["dim"], True)
            pos = s["lens"].long() - 1
            s["slots"] = s["table"].gather(1, (pos // BLOCK)[:, None])[:, 0].long() * BLOCK + pos % BLOCK
        return s
    blocks = c["blocks"]
    s = {"case": c, "blocks": blocks, "caches": torch.randint(0, 256, (c["layers"], blocks, c["hkv"], _granule(c)), dtype=torch.uint8, generator=gen, device="cuda")}
    if c["kind"] == "copy":
        place = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32)
        s["src"], s["dst"] = place[:c["pairs"]].contiguous(), place[c["pairs"]:2 * c["pairs"]].contiguous()
        return s
    lens = _rows(c)
    need = [-(-L // BLOCK) for L in lens]
    # (where the blocks lie: for a compaction by the case, so that its work is known; their order by the seed)
    place = torch.tensor(random.Random(c["mix"] + 2).sample(range(blocks), sum(need)), dtype=torch.int32)
    if c["kind"] == "branch":
        place = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32).cpu()[:sum(need)]
    place = place[torch.randperm(sum(need), generator=gen, device="cuda").cpu()]
    table = torch.full((c["rows"], _width(c)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = place[at:at + n]
        at += n
    s["table"], s["lens"] = table.cuda(), ints(lens + [0] * (c["rows"] - len(lens)))
    # (a prefix store may hold a block beside its row)
    s["refs"] = torch.zeros(blocks, dtype=torch.int32, device="cuda")
    s["refs"][place.long().cuda()] = torch.randint(1, 4, (sum(need),), dtype=torch.int32, generator=gen, device="cuda")
    if c["kind"] == "branch":
        pairs = _branches(c)
        s["parents"], s["children"] = ints([p for p, _ in pairs]), ints(list(range(len(lens), c["rows"])))
        s["grown"] = ints([L + c["grow"] for _, L in pairs])
    else:
        s["table_out"], s["refs_out"] = torch.empty_like(s["table"]), torch.empty_like(s["refs"])
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------

def _append(s):
    """The new token of every sequence into its block: the block's scale may grow, and what it holds follows."""
    c = s["case"]
    blk, off = s["slots"] // BLOCK, s["slots"] % BLOCK
    x, old = _unpack(s["cache"][blk], c)
    new = torch.stack([s["k"], s["v"]], dim=2)                       # [B, H, 2, D]
    here = (torch.arange(BLOCK, device="cuda") == off[:, None])[:, None, None, :, None]
    if c["format"] == "bf16":
        s["cache"][blk] = _pack(torch.where(here, new[..., None, :], x), None, c)
        return
    kind, most = FP8[c["format"]]
    fresh = (off == 0)[:, None, None]
    old = torch.where(fresh, 0.0, old)
    scale = torch.maximum(old, new.float().abs().amax(-1) / most)
    kept = torch.where(fresh[..., None, None], torch.zeros((), device="cuda"), x.float())
    moved = ((kept * old[..., None, None]) / scale[..., None, None]).to(kind)
    grown = ((scale > old) & (old > 0))[..., None, None]
    kept = torch.where(grown, moved.view(torch.uint8), torch.where(fresh[..., None, None], torch.zeros((), dtype=torch.uint8, device="cuda"), x.view(torch.uint8)))
    codes = (new.float() / scale[..., None]).to(kind).view(torch.uint8)
    s["cache"][blk, :, :_used(c)] = _pack(torch.where(here, codes[..., None, :], kept).view(kind), scale, c)


def _keys(s, first):
    """What the sequences' blocks with sinks and from position ``first`` on hold: K, V fp32 [B, H, keys, D], positions [B, keys]."""
    c = s["case"]
    sinks = -(-c["sinks"] // BLOCK)
    gap = (first // BLOCK - sinks).clamp(min=0)                      # blocks passed over between the two
    end = (s["lens"].long() + BLOCK - 1) // BLOCK
    v = torch.arange(s["most"], device="cuda")[None]
    real = torch.where(v < sinks, v, v + gap[:, None])
    there = real < end[:, None]
    ids = torch.where(there, s["table"].gather(1, real.clamp(max=s["table"].shape[1] - 1)), 0).long()
    x, scales = _unpack(s["cache"][ids], c)                          # [B, blocks, H, 2, 16, D]
    x = x.float() if scales is None else x.float() * scales[..., None, None]
    x = x.permute(0, 2, 3, 1, 4, 5).flatten(3, 4)                    # [B, H, 2, keys, D]
    pos = (torch.where(there, real, 1 << 40)[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")).flatten(1)
    return x[:, :, 0], x[:, :, 1], pos


def _plain_attention(s):
    c = s["case"]
    B, G, H, D = c["batch"], c["hq"] // c["hkv"], c["hkv"], c["dim"]
    lens = s["lens"].long()
    if c["kind"] == "decode":
        n, cu, longest = torch.ones_like(lens), torch.arange(B, device="cuda"), 1
    else:
        cu = s["cu"].long()
        n, cu, longest = cu[1:] - cu[:-1], cu[:-1], s["longest"]
    if "most" not in s:
        s["most"] = max(len(_held(c, L, k)) for L, k in zip(_lens(c), _new(c)))
    i = torch.arange(longest, device="cuda")
    at = lens[:, None] - n[:, None] + i                              # positions of the queries
    k, v, pos = _keys(s, (lens - n + 1 - c["window"]).clamp(min=0))
    rows = cu[:, None] + i
    real = i < n[:, None]
    q = s["q"][torch.where(real, rows, 0)].float().view(B, longest, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * longest, D)
    score = (q @ k.transpose(-1, -2)).mul_(s["scale"]).view(B, H, G, longest, -1)
    p, t = pos[:, None, :], at[:, :, None]
    seen = (p <= t) & ((p < c["sinks"]) | (p > t - c["window"]))     # [B, queries, keys]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = score.sum(-1, keepdim=True)
    v = torch.where((pos < lens[:, None])[:, None, :, None], v, 0.0)
    o = (score.view(B, H, G * longest, -1) @ v).view(B, H, G, longest, D) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, longest, H * G, D)
    s["out"].copy_(o[real] if c["kind"] == "prefill" else o[:, 0])
    return s["out"]


def _copy_blocks(s, src, dst):
    c = s["case"]
    s["caches"][:, dst, :, :_used(c)] = s["caches"][:, src, :, :_used(c)]


def _lowest_free(refs, n):
    """The n free blocks of lowest number, n as a length."""
    return torch.nonzero(refs == 0)[:n, 0]


def _plain_branch(s):
    table, refs, lens, kids, parents = s["table"], s["refs"], s["lens"], s["children"].long(), s["parents"].long()
    # the branches of the turn before go
    had = table[kids]
    refs.index_add_(0, had[had >= 0].long(), torch.full_like(had[had >= 0], -1))
    table[kids], lens[kids] = -1, 0
    # new ones: full blocks shared, the last one copied if it is partly filled
    L = lens[parents].long()
    col = torch.arange(table.shape[1], device="cuda")[None]
    shared = torch.where(col < (L // BLOCK)[:, None], table[parents], -1)
    refs.index_add_(0, shared[shared >= 0].long(), torch.ones_like(shared[shared >= 0]))
    part = torch.nonzero(L % BLOCK)[:, 0]
    tail = table[parents[part], L[part] // BLOCK].long()
    fresh = _lowest_free(refs, len(part))
    refs[fresh] = 1
    shared[part, L[part] // BLOCK] = fresh.int()
    _copy_blocks(s, tail, fresh)
    # room for what they will say
    new = s["grown"].long()
    want = (col >= ((L + BLOCK - 1) // BLOCK)[:, None]) & (col < ((new + BLOCK - 1) // BLOCK)[:, None])
    fresh = _lowest_free(refs, int(want.sum()))
    refs[fresh] = 1
    shared[want] = fresh.int()
    table[kids], lens[kids] = shared, s["grown"]
    return {"table": table, "refs": refs, "lens": lens, "caches": s["caches"]}


def _plain_compact(s):
    used = s["refs"] > 0
    n = used.sum()
    ids = torch.arange(s["blocks"], device="cuda")
    movers, holes = torch.nonzero(used & (ids >= n))[:, 0], torch.nonzero(~used & (ids < n))[:, 0]
    to = ids.clone()
    to[movers] = holes
    s["table_out"].copy_(torch.where(s["table"] >= 0, to[s["table"].clamp(min=0).long()], -1))
    s["refs_out"].copy_(s["refs"])
    s["refs_out"][holes], s["refs_out"][movers] = s["refs"][movers], 0
    _copy_blocks(s, movers, holes)
    return {"table": s["table_out"], "refs": s["refs_out"], "used": n.int().view(1), "caches": s["caches"]}


# ---- one pass ----------------------------------------------------------------------------------------------------

def _handles(s):
    """What a program makes once and keeps: descriptors of its caches, a workspace."""
    if "ws" not in s:
        from paper_2602_09323_b200 import binding
        c = s["case"]
        s["lib"] = binding
        wrap = lambda data: binding.Cache(s["blocks"], c["hkv"], c["dim"], FORMATS[c["format"]], data=data)     # noqa: E731
        if c["kind"] in ("decode", "prefill"):
            s["handle"] = wrap(s["cache"].view(-1))
            s["ws"] = binding.new_workspace(c["batch"], c["hq"], c["hkv"], c["dim"], s["table"].shape[1], 0, s["q"].shape[0])
        else:
            s["set"] = binding.CacheSet([wrap(x.view(-1)) for x in s["caches"]])
            s["ws"] = binding.new_pages_workspace(s["blocks"], c["rows"])
            if c["kind"] != "copy":
                s["pages"] = binding.Pages(s["refs"], s["table"], s["lens"])
    return s["lib"]


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if own:
        lib = _handles(s)
        if kind == "decode":
            new = (s["k"], s["v"], s["slots"]) if c["append"] else (None, None, None)
            lib.window_decode(s["handle"], s["q"], s["table"], s["lens"], c["window"], c["sinks"], s["scale"], s["ws"], *new, out=s["out"])
            return [s["out"], s["cache"]] if c["append"] else [s["out"]]
        if kind == "prefill":
            return [lib.window_prefill(s["handle"], s["q"], s["cu"], s["table"], s["lens"], c["window"], c["sinks"], s["scale"], s["ws"], out=s["out"])]
        if kind == "copy":
            lib.pages_copy(s["set"], s["src"], s["dst"])
            return s["caches"]
        if kind == "branch":
            lib.pages_release(s["pages"], s["children"], s["ws"])
            lib.pages_fork(s["set"], s["pages"], s["parents"], s["children"], s["ws"])
            lib.pages_reserve(s["pages"], s["children"], s["grown"], s["ws"])
            return {"table": s["table"], "refs": s["refs"], "lens": s["lens"], "caches": s["caches"]}
        used = lib.pages_compact(s["set"], s["pages"], s["ws"], table_out=s["table_out"], refs_out=s["refs_out"])
        return {"table": s["table_out"], "refs": s["refs_out"], "used": used, "caches": s["caches"]}
    if kind == "decode":
        if c["append"]:
            _append(s)
            return [_plain_attention(s), s["cache"]]
        return [_plain_attention(s)]
    if kind == "prefill":
        return [_plain_attention(s)]
    if kind == "copy":
        _copy_blocks(s, s["src"].long(), s["dst"].long())
        return s["caches"]
    return _plain_branch(s) if kind == "branch" else _plain_compact(s)


# ---- the definition, in 64 bits ----------------------------------------------------------------------------------

def _code_values(fmt):
    """The values of an 8-bit format's 256 codes, from its definition (sign, exponent, mantissa)."""
    e_bits, bias = (4, 7) if fmt == "e4m3" else (5, 15)
    m_bits = 7 - e_bits
    got = []
    for code in range(256):
        e, m = (code >> m_bits) & ((1 << e_bits) - 1), code & ((1 << m_bits) - 1)
        x = math.ldexp(m, 1 - bias - m_bits) if e == 0 else math.ldexp((1 << m_bits) + m, e - bias - m_bits)
        got.append(-x if code & 128 else x)
    return torch.tensor(got, dtype=torch.float64, device="cuda")


def _encode(x, fmt):
    """The nearest value of the format, ties to the even code, by search."""
    top = 127 if fmt == "e4m3" else 124
    grid = _code_values(fmt)[:top]                                   # the finite values that are not negative, in order
    mag = x.abs()
    hi = torch.searchsorted(grid, mag).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    a, b = mag - grid[lo], grid[hi] - mag
    up = (b < a) | ((b == a) & (hi % 2 == 0))
    return torch.where(up, grid[hi], grid[lo]) * torch.where(x < 0, -1.0, 1.0)


def _logical(granule, c):
    """One sequence's K, V [blocks, 16, D] in 64 bits, element by element of the documented layout."""
    d = c["dim"]
    t = torch.arange(BLOCK, device="cuda")[:, None]
    e = torch.arange(d, device="cuda")[None]
    if c["format"] == "bf16":
        x = granule.contiguous().view(torch.bfloat16)
        k_at = (((t // 8) * (d // 32) + e // 32) * 32 + 4 * (t % 8) + (e % 8) // 2) * 8 + (e // 16 % 2) * 4 + (e // 8 % 2) * 2 + e % 2
        v_at = ((e // 16) * 32 + 4 * (e % 8) + (t % 8) // 2) * 8 + (e // 8 % 2) * 4 + (t // 8) * 2 + t % 2
        return x[:, k_at].double(), x[:, BLOCK * d + v_at].double()
    k_at = (t // 8) * 8 * d + (e // 16) * 128 + (t % 8) * 16 + e % 16
    v_at = (e // 8) * 128 + (e % 8) * 16 + t
    scale = granule[:, 2 * BLOCK * d:2 * BLOCK * d + 8].contiguous().view(torch.float32).double()
    value = _code_values(c["format"])
    return value[granule[:, k_at].long()] * scale[:, 0, None, None], value[granule[:, BLOCK * d + v_at].long()] * scale[:, 1, None, None]


def exact(case, seed):
    c = case
    if c["kind"] not in ("decode", "prefill") or work(c)["flops"] > 3e11:
        return None
    s = prepare(c, seed)
    G, lens, new = c["hq"] // c["hkv"], _lens(c), _new(c)
    out = torch.zeros(sum(new), c["hq"], c["dim"], dtype=torch.float64, device="cuda")
    at = 0
    for b, (L, n) in enumerate(zip(lens, new)):
        cols = torch.tensor(_held(c, L, n), device="cuda")
        ids = s["table"][b, cols].long()
        j = (cols[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")).flatten()
        t = torch.arange(L - n, L, device="cuda")[:, None]
        hidden = (j > t) | ((j >= c["sinks"]) & (j + c["window"] <= t))
        for h in range(c["hkv"]):
            k, v = _logical(s["cache"][ids, h], c)
            if c["append"]:
                for which, (kv, new_rows) in enumerate(((k, s["k"]), (v, s["v"]))):
                    x, off = new_rows[b, h], (L - 1) % BLOCK
                    if c["format"] == "bf16":
                        kv[-1, off] = x.double()
                        continue
                    d = c["dim"]
                    old = torch.zeros((), device="cuda") if off == 0 else s["cache"][ids[-1], h, 2 * BLOCK * d + 4 * which:2 * BLOCK * d + 4 * which + 4].view(torch.float32)[0]
                    scale = torch.maximum(old, x.float().abs().max() / FP8[c["format"]][1])
                    if bool(scale > old) and bool(old > 0):
                        kv[-1] = _encode((kv[-1].float() / scale).double(), c["format"]) * scale.double()
                    kv[-1, off] = _encode((x.float() / scale).double(), c["format"]) * scale.double()
            k, v = k.flatten(0, 1), v.flatten(0, 1)
            q = s["q"][at:at + n, h * G:(h + 1) * G].double()
            z = torch.einsum("ngd,kd->gnk", q, k) * s["scale"]
            z = torch.where(hidden, -math.inf, z)
            out[at:at + n, h * G:(h + 1) * G] = torch.einsum("gnk,kd->ngd", torch.softmax(z, -1), torch.where((j < L)[:, None], v, 0.0))
        at += n
    return [out, None] if c["append"] else [out]
