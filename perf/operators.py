"""Performance cases of the paged KV cache held in 8 bits: its block tables
and slot maps, the write of new tokens, the read of stored tokens and the
attention over it, each in a plain form and through the library.

kind    one pass
tables  a serving step's bookkeeping: the pages of finished requests go back
        to the free list (ss_block_release, where requests finish), then the
        step's tokens get their pages, slots and positions (ss_block_tables)
write   a step's new K and V written into 8-bit block records, with a scale
        for each block and head and the filled blocks' metadata, and the rows
        of blocks that stay open kept in bf16 (ss_write_kv8)
read    the stored tokens of some requests as bf16 rows, as the attention of
        a prompt's next chunk reads them (ss_read_kv8)
attend  a decode step's attention over the records: blocks selected for each
        head from a shared pool, all blocks of each request with its open
        block, or the slots of an HBM block cache (ss_sparse_attention_kv8)

Record of blk tokens of one KV head, d = 128 channels: blk*d bytes of K
codes, blk*d bytes of V codes, then 128 bytes that begin with the fp32 scales
of K and V, the rest zero.  Codes stand in subtiles s of T = min(blk, 16)
tokens; token t of a subtile and channel c:
  K: s*T*d + (c/16)*T*16 + t*16 + c%16
  V: s*T*d + (c%8/4)*T*64 + (t/4)*256 + (c/8)*16 + (c%4)*4 + t%4
A value is its code (e4m3 or int8) times the scale: with the largest
magnitude m = max(|x|, 2^-100) of the tile and Q = 448 or 127, the scale is
m/Q and the code x*(Q/m), rounded to nearest even.

Values are synthetic: K, V ~ N(0,1) times a scale U[0.5, 2] per channel,
queries ~ N(0,1), as in synth/.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
Q_MAX = {"e4m3": 448.0, "int8": 127.0}
TINY = 2.0 ** -100
MOST_TOKENS = 131072 * 8  # tokens times KV heads of the largest write
MOST_ATTEND = 16 * 8 * 36000  # and of the largest attention


def listed():
    return [
        # the smallest call: one more token for each of 64 running requests
        {"name": "tables-decode-b64", "kind": "tables", "B": 64, "blk": 16, "ctx": 32768, "join": 0.0, "short": False},
        # a busy server's step: 1 in 32 of 512 requests has finished and a prompt takes its place, the others decode
        {"name": "tables-turn-b512", "kind": "tables", "B": 512, "blk": 16, "ctx": 16384, "join": 0.03125,
         "short": False},
        # one token for each of 64 requests; every 16th block fills (a decode step's append)
        {"name": "write-decode-b64", "kind": "write", "B": 64, "Hkv": 8, "blk": 16, "tokens": 64, "prompts": 0,
         "fmt": "e4m3", "meta": "cuboid"},
        # a mixed step of a GQA-7 model: three prompt chunks of odd length beside 21 decoding requests
        {"name": "write-mixed-gqa7", "kind": "write", "B": 24, "Hkv": 4, "blk": 8, "tokens": 8191, "prompts": 3,
         "fmt": "int8", "meta": "mean"},
        # the largest: one layer of a 128k-token prompt
        {"name": "write-prompt-128k", "kind": "write", "B": 1, "Hkv": 8, "blk": 16, "tokens": 131072, "prompts": 1,
         "fmt": "e4m3", "meta": "cuboid"},
        # the history that one more chunk of a long prompt attends to
        {"name": "read-b1-64k", "kind": "read", "B": 1, "Hkv": 8, "blk": 16, "ctx": 65521, "fmt": "e4m3"},
        # ragged short histories, blocks of 32
        {"name": "read-ragged-int8", "kind": "read", "B": 7, "Hkv": 2, "blk": 32, "ctx": 5000, "fmt": "int8"},
        # two short requests of a small model, selected blocks of a shared pool; launches and latency
        {"name": "attend-tiny", "kind": "attend", "mode": "sparse", "B": 2, "Hq": 8, "Hkv": 2, "blk": 16, "k": 16,
         "ctx": 4096, "fmt": "e4m3"},
        # the 128k-context batch over its HBM block cache (1024 slots for each head)
        {"name": "attend-b64-cache", "kind": "attend", "mode": "slots", "B": 64, "Hq": 32, "Hkv": 8, "blk": 16,
         "k": 128, "ctx": 16384, "fmt": "e4m3"},
        # a ragged batch of the GQA-7 model, 512 selected blocks of 8 tokens from a shared pool
        {"name": "attend-gqa7-sparse", "kind": "attend", "mode": "sparse", "B": 11, "Hq": 28, "Hkv": 4, "blk": 8,
         "k": 512, "ctx": 20000, "fmt": "int8"},
        # one request over all of a 128k context
        {"name": "attend-b1-128k-dense", "kind": "attend", "mode": "dense", "B": 1, "Hq": 32, "Hkv": 8, "blk": 32,
         "k": 4096, "ctx": 131071, "fmt": "int8"},
        # the largest: a ragged batch of 8k to 64k tokens, all blocks
        {"name": "attend-b16-dense", "kind": "attend", "mode": "dense", "B": 16, "Hq": 32, "Hkv": 8, "blk": 16,
         "k": 4096, "ctx": 65536, "fmt": "e4m3"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tables", "write", "write", "read", "attend", "attend", "attend"])
    blk, fmt, hkv = rng.choice([8, 16, 16, 32]), rng.choice(["e4m3", "int8"]), rng.choice([1, 2, 4, 8])
    if kind == "tables":
        B = _log(rng, 1, 512)
        return {"kind": kind, "B": B, "blk": blk, "ctx": _log(rng, 64, 16384),
                "join": rng.choice([0.0, 0.01, 0.02, 0.03]), "short": rng.random() < 0.25}
    if kind == "write":
        prompts = rng.choice([0, 1, 4])
        B = _log(rng, max(1, prompts), 16 if prompts else 256)
        tokens = _log(rng, B + 1, 131072) if prompts else B
        return {"kind": kind, "B": B, "Hkv": hkv, "blk": blk, "tokens": tokens, "prompts": prompts, "fmt": fmt,
                "meta": rng.choice(["none", "cuboid", "mean"])}
    if kind == "read":
        B = _log(rng, 1, 32)
        return {"kind": kind, "B": B, "Hkv": hkv, "blk": blk,
                "ctx": _log(rng, 16, min(65536, MOST_TOKENS // 2 // (B * hkv))), "fmt": fmt}
    B, mode = _log(rng, 1, 64), rng.choice(["sparse", "slots", "dense"])
    ctx = _log(rng, 64, min(131072, MOST_ATTEND // (B * hkv)))
    k = ctx // blk + 1 if mode == "dense" else _log(rng, 1, max(1, min(4096, ctx) // blk))
    return {"kind": "attend", "mode": mode, "B": B, "Hq": hkv * rng.choice([1, 2, 4, 5, 7, 8, 16]), "Hkv": hkv,
            "blk": blk, "k": k, "ctx": ctx, "fmt": fmt}


# ------------------------------------------------------------------- inputs
def _rand(c, seed=None):
    """A generator of the case's own properties, or of an input's."""
    return random.Random("%s %s %s" % (sorted((k, v) for k, v in c.items() if k != "name"), seed, "cases"))


def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + tag) & ((1 << 62) - 1))
    return g


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def _normal(shape, scales, g):
    """bf16 N(0,1) times a scale per channel (the last axis)."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    return (x.mul_(scales)).to(torch.bfloat16)


def _channel_scales(hkv, g):
    return 0.5 + 1.5 * torch.rand((hkv, 2, D), generator=g, device="cuda")


def _lens(c):
    """Lengths of the sequences: one of ctx tokens, the others down to an eighth of it; a property of the case."""
    r = _rand(c)
    n = [r.randint(max(1, c["ctx"] // 8), c["ctx"]) for _ in range(c["B"])]
    n[r.randrange(c["B"])] = c["ctx"]
    return np.asarray(n, np.int64)


def _held(n, blk):
    return (n + blk - 1) // blk


def _prepare_tables(c, seed):
    rng = np.random.RandomState(seed % (1 << 31))
    B, blk, ctx = c["B"], c["blk"], c["ctx"]
    n_join = math.ceil(B * c["join"])
    done = np.zeros(B, np.int64)
    done[rng.permutation(B)[:n_join]] = 1
    length = rng.randint(1, ctx + 1, B)
    n_new = np.ones(B, np.int64)
    if B >= 8:
        n_new[rng.permutation(B)[:B // 16]] = 0  # rows of a padded batch
    n_new[done > 0] = rng.randint(ctx // 2, ctx + 1, n_join)
    max_blocks = (ctx + blk) // blk + 1
    n_pages = B * max_blocks + 5
    held = _held(length, blk)
    pages = rng.permutation(n_pages)
    table = np.full((B, max_blocks), -1, np.int64)
    at = np.cumsum(held) - held
    for b in range(B):
        table[b, :held[b]] = pages[at[b]:at[b] + held[b]]
    left = pages[held.sum():]
    free = np.full(n_pages, -1, np.int64)
    n_free = len(left)
    if c["short"]:  # the pool runs out within the step
        base = np.where(done > 0, 0, length)
        need = int((_held(base + n_new, blk) - _held(base, blk)).sum())
        n_free = max(0, min(n_free, need // 2 - int(held[done > 0].sum())))
    free[:n_free] = left[:n_free]
    cap = B + n_join * ctx
    s = {"case": c, "len": _i32(length), "n_new": _i32(n_new), "done": _i32(done), "n_free": _i32([n_free]),
         "free": _i32(free), "tables": _i32(table), "cap": cap, "max_blocks": max_blocks, "n_pages": n_pages}
    new = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    s.update(len_mid=new(B), nblk_mid=new(B), n_free_mid=new(1), len_out=new(B), nblk=new(B), n_free_out=new(1),
             tok_begin=new(B + 1), slots=new(cap), positions=new(cap), taken=new(B + 1), status=new(B))
    return s


def _prepare_write(c, seed):
    rng = np.random.RandomState(seed % (1 << 31))
    B, hkv, blk, cap = c["B"], c["Hkv"], c["blk"], c["tokens"]
    n_new = np.ones(B, np.int64)
    if c["prompts"]:
        left = cap - (B - c["prompts"])
        who = rng.permutation(B)[:c["prompts"]]
        cut = np.sort(rng.randint(0, left + 1, c["prompts"] - 1))
        n_new[who] = np.diff(np.concatenate([[0], cut, [left]]))
    # a prompt alone begins its sequence; in a mixed step every row holds some tokens already
    length = np.zeros(B, np.int64) if B == 1 and c["prompts"] else rng.randint(0, 8 * blk, B)
    if not c["prompts"]:
        length = length // blk * blk + (np.arange(B) + int(rng.randint(blk))) % blk  # steady state: 1 in blk fills
    begin = np.concatenate([[0], np.cumsum(n_new)])
    seq = np.repeat(np.arange(B), n_new)
    pos = np.arange(cap) - begin[seq] + length[seq]
    held = _held(length + n_new, blk)
    n_pages = 10 * B + cap // blk + 3
    page0 = np.cumsum(held) - held
    pages = rng.permutation(n_pages)
    slots = pages[page0[seq] + pos // blk] * blk + pos % blk
    rec = 2 * blk * D + 128
    g = _gen(seed, 1)
    scales = _channel_scales(hkv, g)
    nblk_max = 9 + cap // blk
    per = {"none": 0, "cuboid": 2 * D, "mean": D}[c["meta"]]
    opened = _normal((B, hkv, 2, blk, D), scales[None, :, :, None], g)
    opened[:, :, 1] = opened[:, :, 1].transpose(2, 3).contiguous().view(B, hkv, blk, D)
    return {"case": c, "new": _normal((cap, hkv, 2, D), scales, g), "tok_begin": _i32(begin), "slots": _i32(slots),
            "positions": _i32(pos), "n_pages": n_pages, "nblk_max": nblk_max,
            "records": torch.zeros((hkv, n_pages, rec), dtype=torch.uint8, device="cuda"),
            "region": torch.arange(hkv, device="cuda", dtype=torch.int64).repeat(B) * (n_pages * rec),
            "open": opened.view(B, hkv, 2 * blk * D).contiguous(),
            "meta": torch.zeros((B, hkv, nblk_max, per), dtype=torch.bfloat16, device="cuda") if per else None}


def _make_records(shape, scales, blk, fmt, g):
    """Records [Hkv][n][rec] of random K and V."""
    hkv, n = shape
    out = torch.empty((hkv, n, 2 * blk * D + 128), dtype=torch.uint8, device="cuda")
    for h in range(hkv):
        k = _normal((n, blk, D), scales[h, 0], g)
        v = _normal((n, blk, D), scales[h, 1], g)
        out[h] = _pack(k.float(), v.float(), blk, fmt)
    return out


def _prepare_stored(c, seed):
    """What reads and attention find: a pool of records, tables, lengths, open blocks, queries."""
    rng = np.random.RandomState(seed % (1 << 31))
    B, hkv, blk = c["B"], c["Hkv"], c["blk"]
    rec = 2 * blk * D + 128
    g = _gen(seed, 2)
    scales = _channel_scales(hkv, g)
    length = _lens(c)
    nblk = length // blk
    s = {"case": c, "len": _i32(length), "nblk": _i32(nblk)}
    if c.get("mode") == "slots":  # a region of slots for each (sequence, head), all filled
        n = max(1, c["ctx"] // blk)
        s["records"] = _make_records((hkv, B * n), scales, blk, c["fmt"], g).view(hkv, B, n, rec).transpose(0, 1).contiguous()
        s["region"] = torch.arange(B * hkv, device="cuda", dtype=torch.int64) * (n * rec)
        s["limit"] = n
        s["capacity"] = torch.full((B * hkv,), n, dtype=torch.int32, device="cuda")
    else:
        held = _held(length, blk)
        n = int(held.sum()) + 3
        max_blocks = int(held.max()) + 1
        pages = rng.permutation(n)
        table = np.full((B, max_blocks), -1, np.int64)
        at = np.cumsum(held) - held
        for b in range(B):
            table[b, :held[b]] = pages[at[b]:at[b] + held[b]]
        s["records"] = _make_records((hkv, n), scales, blk, c["fmt"], g)
        s["region"] = torch.arange(hkv, device="cuda", dtype=torch.int64).repeat(B) * (n * rec)
        s["limit"], s["capacity"] = n, None
        s["tables"], s["max_blocks"] = _i32(table), max_blocks
        opened = _normal((B, hkv, 2, blk, D), scales[None, :, :, None], g)
        opened[:, :, 1] = opened[:, :, 1].transpose(2, 3).contiguous().view(B, hkv, blk, D)
        s["open"] = opened.view(B, hkv, 2 * blk * D).contiguous()
    if c["kind"] == "read":
        begin = np.concatenate([[0], np.cumsum(length)])
        s["row_begin"], s["rows"] = _i32(begin), int(begin[-1])
        s["out"] = torch.zeros((s["rows"], hkv, 2, D), dtype=torch.bfloat16, device="cuda")
        return s
    s["q"] = torch.randn((B, c["Hq"], D), generator=g, device="cuda").to(torch.bfloat16)
    k = c["k"]
    if c["mode"] != "dense":
        # distinct entries for each head, ascending, -1 behind the last where a sequence has fewer
        top = torch.full((B,), s["limit"], device="cuda") if c["mode"] == "slots" else s["nblk"]
        width = int(top.max()) if B else 0
        order = torch.rand((B, hkv, max(width, k)), generator=g, device="cuda")
        order[torch.arange(max(width, k), device="cuda")[None, None].expand_as(order) >= top[:, None, None]] = 2.0
        best, at = order.topk(k, dim=-1, largest=False)
        big = 1 << 30
        at = torch.where(best < 1.5, at, big).sort(dim=-1).values
        s["sel"] = torch.where(at < big, at, -1).to(torch.int32).contiguous()
    s["out"] = torch.zeros((B, c["Hq"], D), dtype=torch.float32, device="cuda")
    s["ws_bytes"] = 4 * 4096 * 16 * (D + 2)  # room for the partial results of any shape
    s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    return {"tables": _prepare_tables, "write": _prepare_write, "read": _prepare_stored,
            "attend": _prepare_stored}[case["kind"]](case, seed)


# -------------------------------------------------------------- plain forms
def _pack(k, v, blk, fmt):
    """Records [..., rec] of fp32 K and V tiles [..., blk, d]."""
    lead, t = k.shape[:-2], min(blk, 16)
    q = torch.tensor(Q_MAX[fmt], dtype=torch.float32, device=k.device)
    parts, scales = [], []
    for x, order in ((k, "k"), (v, "v")):
        m = x.abs().amax((-2, -1)).clamp_min(TINY)
        y = x * (q.expand_as(m) / m)[..., None, None]
        y = y.to(torch.float8_e4m3fn) if fmt == "e4m3" else y.round().to(torch.int8)
        y = y.view(torch.uint8)
        if order == "k":
            y = y.reshape(-1, blk // t, t, D // 16, 16).permute(0, 1, 3, 2, 4)
        else:  # t = 4*L + i, c = 8*x + 4*h + j  ->  [h][L][x][j][i]
            y = y.reshape(-1, blk // t, t // 4, 4, D // 8, 2, 4).permute(0, 1, 5, 2, 4, 6, 3)
        parts.append(y.reshape(*lead, blk * D))
        scales.append(m / q.expand_as(m))
    tail = torch.zeros((*lead, 32), dtype=torch.float32, device=k.device)
    tail[..., 0], tail[..., 1] = scales
    return torch.cat([*parts, tail.view(torch.uint8)], -1)


def _unpack(rec, blk, fmt):
    """fp32 K and V tiles [..., blk, d] of records [..., rec]."""
    lead, t = rec.shape[:-1], min(blk, 16)
    codes = rec[..., :2 * blk * D].view(torch.float8_e4m3fn if fmt == "e4m3" else torch.int8).float()
    scales = rec[..., 2 * blk * D:2 * blk * D + 8].contiguous().view(torch.float32)
    k = codes[..., :blk * D].reshape(-1, blk // t, D // 16, t, 16).permute(0, 1, 3, 2, 4).reshape(*lead, blk, D)
    v = codes[..., blk * D:].reshape(-1, blk // t, 2, t // 4, D // 8, 4, 4).permute(0, 1, 3, 6, 4, 2, 5)
    return k * scales[..., 0, None, None], v.reshape(*lead, blk, D) * scales[..., 1, None, None]


def _plain_tables(s):
    c = s["case"]
    B, blk = c["B"], c["blk"]
    length, n_free = s["len"].long(), s["n_free"].long()
    if c["join"]:
        count = torch.where(s["done"] > 0, _held(length, blk), 0)
        at = n_free + count.cumsum(0) - count
        j = torch.arange(s["max_blocks"], device="cuda")[None]
        mask = j < count[:, None]
        s["free"][(at[:, None] + j)[mask]] = s["tables"][mask]
        n_free = n_free + count.sum()
        length = torch.where(s["done"] > 0, 0, length)
    n = s["n_new"].long()
    need = _held(length + n, blk) - _held(length, blk)
    need = torch.where(_held(length + n, blk) > s["max_blocks"], 0, need)
    upto = need.cumsum(0)
    status = torch.where(_held(length + n, blk) > s["max_blocks"], 2, torch.where((need > 0) & (upto > n_free), 1, 0))
    got = torch.where(status == 0, need, 0)
    taken = torch.cat([got.new_zeros(1), got.cumsum(0)])
    begin = torch.cat([n.new_zeros(1), n.cumsum(0)])
    row = torch.arange(s["cap"], device="cuda")
    seq = torch.searchsorted(begin, row, right=True) - 1
    live = seq < B
    seq = seq.clamp_max(B - 1)
    pos = length[seq] + row - begin[seq]
    served = live & (status[seq] == 0)
    j = pos // blk
    fresh = j - _held(length, blk)[seq]
    old = s["tables"][seq, j.clamp_max(s["max_blocks"] - 1)].long()
    page = torch.where(fresh >= 0, s["free"].long()[(n_free - 1 - taken[seq] - fresh).clamp(0, s["n_pages"] - 1)], old)
    first = served & (pos % blk == 0)
    s["tables"][seq[first], j[first]] = page[first].int()
    length = length + torch.where(status == 0, n, 0)
    i = torch.int32
    out = {"tables": s["tables"], "len": length.to(i), "nblk": (length // blk).to(i),
           "n_free": (n_free - taken[-1]).to(i), "tok_begin": begin.to(i),
           "slots": torch.where(served, page * blk + pos % blk, -1).to(i),
           "positions": torch.where(served, pos, -1).to(i), "taken": taken.to(i), "status": status.to(i)}
    return {**out, "free": s["free"]} if c["join"] else out


def _written(s):
    """What a write leaves: the records' values and scales, open rows and metadata."""
    c = s["case"]
    n = 2 * c["blk"] * D
    out = {"codes": s["records"][..., :n].view(torch.float8_e4m3fn if c["fmt"] == "e4m3" else torch.int8),
           "scales": s["records"][..., n:].view(torch.float32), "open": s["open"]}
    return {**out, "meta": s["meta"]} if s["meta"] is not None else out


def _plain_write(s):
    c = s["case"]
    B, hkv, blk = c["B"], c["Hkv"], c["blk"]
    begin, slots, pos, new = s["tok_begin"].long(), s["slots"].long(), s["positions"].long(), s["new"]
    open_k = s["open"].view(B, hkv, 2, blk * D)[:, :, 0].view(B, hkv, blk, D)
    open_v = s["open"].view(B, hkv, 2, blk * D)[:, :, 1].view(B, hkv, D, blk)
    row = torch.arange(c["tokens"], device="cuda")
    seq = torch.searchsorted(begin, row, right=True) - 1
    last = (pos % blk == blk - 1).nonzero()[:, 0]  # the last tokens of blocks that fill
    if len(last):
        b = seq[last]
        rows = last[:, None] + torch.arange(1 - blk, 1, device="cuda")
        old = (rows < begin[b][:, None])[:, None, :, None]
        kv = new[rows.clamp_min(0)].permute(0, 2, 3, 1, 4)  # [blocks][head][2][blk][d]
        k = torch.where(old, open_k[b], kv[:, :, 0])
        v = torch.where(old, open_v[b].transpose(2, 3), kv[:, :, 1])
        page, j = slots[last] // blk, pos[last] // blk
        s["records"].transpose(0, 1)[page] = _pack(k.float(), v.float(), blk, c["fmt"])
        if c["meta"] == "cuboid":
            s["meta"][b, :, j] = torch.cat([k.amin(2), k.amax(2)], -1)
        elif c["meta"] == "mean":
            s["meta"][b, :, j] = k.double().mean(2).to(torch.bfloat16)
    end = pos[(begin[1:] - 1).clamp_min(0)] + 1
    rest = (pos // blk == (end // blk)[seq]).nonzero()[:, 0]
    open_k[seq[rest], :, pos[rest] % blk] = new[rest, :, 0]
    open_v[seq[rest], :, :, pos[rest] % blk] = new[rest, :, 1]
    return _written(s)


def _plain_read(s):
    c = s["case"]
    B, hkv, blk = c["B"], c["Hkv"], c["blk"]
    begin, length = s["row_begin"].long(), s["len"].long()
    open_k = s["open"].view(B, hkv, 2, blk * D)[:, :, 0].view(B, hkv, blk, D)
    open_v = s["open"].view(B, hkv, 2, blk * D)[:, :, 1].view(B, hkv, D, blk)
    row = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(begin, row, right=True) - 1
    pos = row - begin[seq]
    full = pos < (length // blk * blk)[seq]
    k, v = _unpack(s["records"], blk, c["fmt"])  # [head][page][blk][d]
    page = s["tables"].long()[seq, pos // blk]
    at = (page * blk + pos % blk)[full]
    s["out"][full, :, 0] = k.view(hkv, -1, D)[:, at].transpose(0, 1).to(torch.bfloat16)
    s["out"][full, :, 1] = v.view(hkv, -1, D)[:, at].transpose(0, 1).to(torch.bfloat16)
    rest = ~full
    s["out"][rest, :, 0] = open_k[seq[rest], :, pos[rest] % blk]
    s["out"][rest, :, 1] = open_v[seq[rest], :, :, pos[rest] % blk]
    return s["out"]


def _entries(s):
    """Page of each entry [B][Hkv][n], -1 where there is none."""
    c = s["case"]
    if c["mode"] == "slots":
        return s["sel"].long()
    if c["mode"] == "sparse":
        at = s["sel"].long()
        page = s["tables"].long()[:, None].expand(-1, c["Hkv"], -1).gather(2, at.clamp_min(0))
        return torch.where(at >= 0, page, -1)
    i = torch.arange(min(c["k"], s["max_blocks"]), device="cuda")
    page = torch.where(i[None] < s["nblk"][:, None], s["tables"].long()[:, :len(i)], -1)
    return page[:, None].expand(-1, c["Hkv"], -1)


def _plain_attend(s):
    c = s["case"]
    B, hkv, blk, G = c["B"], c["Hkv"], c["blk"], c["Hq"] // c["Hkv"]
    page = _entries(s)
    n = page.shape[-1]
    h = torch.arange(hkv, device="cuda")[None, :, None]
    if c["mode"] == "slots":
        rec = s["records"][torch.arange(B, device="cuda")[:, None, None], h, page.clamp_min(0)]
    else:
        rec = s["records"][h, page.clamp_min(0)]
    k, v = _unpack(rec, blk, c["fmt"])
    k, v = k.view(B, hkv, n * blk, D), v.view(B, hkv, n * blk, D)
    live = (page >= 0).repeat_interleave(blk, dim=-1)
    if c["mode"] == "dense":
        o = s["open"].view(B, hkv, 2, blk * D)
        k = torch.cat([k, o[:, :, 0].view(B, hkv, blk, D).float()], 2)
        v = torch.cat([v, o[:, :, 1].view(B, hkv, D, blk).transpose(2, 3).float()], 2)
        tail = torch.arange(blk, device="cuda")[None] < (s["len"] % blk)[:, None]
        live = torch.cat([live, tail[:, None].expand(-1, hkv, -1)], 2)
    z = torch.matmul(s["q"].view(B, hkv, G, D).float(), k.transpose(2, 3)) * SCALE
    z = torch.where(live[:, :, None], z, -math.inf)
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(m == -math.inf, 0.0, m))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, torch.where(live[..., None], v, 0.0)) / torch.where(total == 0, 1.0, total)
    return o.reshape(B, c["Hq"], D)


# ------------------------------------------------------------- the library
def _ss():
    from paper_2509_24626_amd import binding
    return binding


def _own_tables(s):
    ss, c = _ss(), s["case"]
    length, n_free = s["len"], s["n_free"]
    if c["join"]:
        ss.ss_block_release(length, s["done"], n_free, c["B"], c["blk"], s["max_blocks"], s["n_pages"], s["tables"],
                            s["free"], s["len_mid"], s["nblk_mid"], s["n_free_mid"])
        length, n_free = s["len_mid"], s["n_free_mid"]
    ss.ss_block_tables(length, s["n_new"], n_free, c["B"], c["blk"], s["max_blocks"], s["n_pages"], s["free"],
                       s["tables"], s["len_out"], s["nblk"], s["n_free_out"], s["tok_begin"], s["slots"],
                       s["positions"], s["cap"], s["taken"], s["status"])
    out = {"tables": s["tables"], "len": s["len_out"], "nblk": s["nblk"], "n_free": s["n_free_out"],
           "tok_begin": s["tok_begin"], "slots": s["slots"], "positions": s["positions"], "taken": s["taken"],
           "status": s["status"]}
    return {**out, "free": s["free"]} if c["join"] else out


def _own_write(s):
    ss, c = _ss(), s["case"]
    base, row = s["new"].data_ptr(), c["Hkv"] * 2 * D * 2
    ss.ss_write_kv8(base, base + 2 * D, row, 4 * D, s["tok_begin"], s["slots"], s["positions"], c["B"], c["Hkv"],
                    c["blk"], D, c["tokens"], ss.SS_KV8_E4M3 if c["fmt"] == "e4m3" else ss.SS_KV8_INT8, s["records"],
                    s["region"], s["n_pages"], s["open"], s["meta"],
                    ss.SS_META_MEAN if c["meta"] == "mean" else ss.SS_META_CUBOID, s["nblk_max"])
    return _written(s)


def _own_read(s):
    ss, c = _ss(), s["case"]
    base, row = s["out"].data_ptr(), c["Hkv"] * 2 * D * 2
    ss.ss_read_kv8(s["records"], s["region"], s["tables"], s["max_blocks"], s["limit"], s["open"], s["len"],
                   s["row_begin"], c["B"], c["Hkv"], c["blk"], D, s["rows"],
                   ss.SS_KV8_E4M3 if c["fmt"] == "e4m3" else ss.SS_KV8_INT8, base, base + 2 * D, row, 4 * D)
    return s["out"]


def _own_attend(s):
    ss, c = _ss(), s["case"]
    dense, paged = c["mode"] == "dense", c["mode"] != "slots"
    ss.ss_sparse_attention_kv8(s["q"], s["records"], s["region"], None if dense else s["sel"],
                               s["tables"] if paged else None, s["max_blocks"] if paged else 0, s["capacity"],
                               s["limit"], s["nblk"] if paged else None, s["open"] if dense else None,
                               s["len"] if dense else None, ss.SS_KV8_E4M3 if c["fmt"] == "e4m3" else ss.SS_KV8_INT8,
                               c["B"], c["Hq"], c["Hkv"], D, c["blk"], c["k"], SCALE, s["out"], s["ws"],
                               s["ws_bytes"])
    return s["out"]


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"tables": _own_tables, "write": _own_write, "read": _own_read, "attend": _own_attend}[kind](state)
    return {"tables": _plain_tables, "write": _plain_write, "read": _plain_read, "attend": _plain_attend}[kind](state)


# -------------------------------------------------------------------- work
def work(case):
    c, kind = case, case["kind"]
    if kind == "tables":
        n_join = math.ceil(c["B"] * c["join"])
        cap = c["B"] + n_join * c["ctx"]
        # lengths in and out, prefix sums, flags; slot and position of each row; pages through list and table
        return {"bytes": 40 * c["B"] + 8 * cap + (24 if n_join else 8) * (c["B"] + n_join * c["ctx"]) // c["blk"],
                "flops": 8 * cap}
    rec = 2 * c["blk"] * D + 128
    if kind == "write":
        per = {"none": 0, "cuboid": 4 * D, "mean": 2 * D}[c["meta"]]
        heads, blocks = c["tokens"] * c["Hkv"], c["tokens"] * c["Hkv"] / c["blk"]
        return {"bytes": int(heads * 4 * D + blocks * (rec + per)), "flops": heads * 2 * D * 4}
    length = _lens(c)
    if kind == "read":
        full = int((length // c["blk"]).sum()) * c["Hkv"]
        return {"bytes": full * rec + int(length.sum()) * c["Hkv"] * 4 * D, "flops": full * c["blk"] * 2 * D}
    if c["mode"] == "dense":
        blocks, rest = int((length // c["blk"]).sum()), int((length % c["blk"]).sum())
    else:
        have = np.full(c["B"], max(1, c["ctx"] // c["blk"])) if c["mode"] == "slots" else length // c["blk"]
        blocks, rest = int(np.minimum(have, c["k"]).sum()), 0
    g = c["Hq"] // c["Hkv"]
    return {"bytes": c["Hkv"] * (blocks * rec + rest * 4 * D) + c["B"] * c["Hq"] * D * 6,
            "flops": c["Hkv"] * (blocks * c["blk"] + rest) * g * D * 4}


# ------------------------------------------------- the definition in 64 bits
def _places(blk):
    """Byte of token t and channel c within a record's K part and V part: int64 [2][blk][d]."""
    t, c = np.arange(blk)[:, None], np.arange(D)[None]
    w = min(blk, 16)
    s, u = t // w, t % w
    k = s * w * D + (c // 16) * w * 16 + u * 16 + c % 16
    v = blk * D + s * w * D + (c % 8 // 4) * w * 64 + (u // 4) * 256 + (c // 8) * 16 + (c % 4) * 4 + u % 4
    return torch.from_numpy(np.stack([k, v])).cuda()


def _code_values(fmt):
    """What each of the 256 codes stands for, in 64 bits."""
    if fmt == "int8":
        return torch.from_numpy(np.arange(256, dtype=np.uint8).view(np.int8).astype(np.float64)).cuda()
    v = []
    for x in range(256):
        e, m = x >> 3 & 15, x & 7
        y = math.nan if e == 15 and m == 7 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v.append(-y if x & 128 else y)
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def _exact_tiles(rec, blk, fmt):
    """K and V in 64 bits, [n][2][blk][d], of records [n][rec]."""
    at = _places(blk).view(-1)
    codes = rec[:, at].view(-1, 2, blk, D).long()
    scales = rec[:, 2 * blk * D:2 * blk * D + 8].contiguous().view(torch.float32).double()
    return _code_values(fmt)[codes] * scales[:, :, None, None]


def _exact_codes(x, fmt):
    """Codes (as the values they stand for) and scales of 64-bit tiles [..., blk, d]."""
    m = x.abs().flatten(-2).max(-1).values.clamp_min(TINY)
    y = x * (Q_MAX[fmt] / m)[..., None, None]
    if fmt == "int8":
        return torch.round(y), m / 127.0
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(y / step) * step, m / 448.0


def _exact_write(c, s):
    B, hkv, blk = c["B"], c["Hkv"], c["blk"]
    n_pages, nm = s["n_pages"], s["nblk_max"]
    codes = torch.zeros((hkv, n_pages, 2 * blk * D), dtype=torch.float64, device="cuda")
    scales = torch.zeros((hkv, n_pages, 32), dtype=torch.float64, device="cuda")
    opened = s["open"].double().clone()
    meta = None if s["meta"] is None else torch.zeros(s["meta"].shape, dtype=torch.float64, device="cuda")
    begin, pos, slots = (s[k].cpu().numpy() for k in ("tok_begin", "positions", "slots"))
    place = _places(blk).view(2, -1)
    for b in range(B):
        i0, i1 = int(begin[b]), int(begin[b + 1])
        if i0 == i1:
            continue
        p0 = int(pos[i0]) % blk
        o = opened[b].view(hkv, 2, blk * D)
        old = torch.stack([o[:, 0].view(hkv, blk, D), o[:, 1].view(hkv, D, blk).transpose(1, 2)], 1)[:, :, :p0]
        kv = torch.cat([old, s["new"][i0:i1].double().permute(1, 2, 0, 3)], 2)  # [head][2][rows][d]
        full = kv.shape[2] // blk
        if full:
            tiles = kv[:, :, :full * blk].reshape(hkv, 2, full, blk, D)
            y, m = _exact_codes(tiles, c["fmt"])
            ends = i0 + np.arange(1, full + 1) * blk - p0 - 1
            page = torch.from_numpy(slots[ends].astype(np.int64) // blk).cuda()
            first = int(pos[i0]) // blk
            for part in range(2):
                flat = torch.zeros((hkv, full, 2 * blk * D), dtype=torch.float64, device="cuda")
                flat[:, :, place[part]] = y[:, part].reshape(hkv, full, -1)
                codes[:, page] += flat
                scales[:, page, part] = m[:, part]
            if meta is not None:
                k = tiles[:, 0]
                meta[b, :, first:first + full] = (k.mean(2) if c["meta"] == "mean" else
                                                  torch.cat([k.min(2).values, k.max(2).values], -1))
        rest = kv.shape[2] - full * blk
        lo = 0 if full else p0
        if rest > lo:
            tail = kv[:, :, full * blk + lo:]
            o[:, 0].view(hkv, blk, D)[:, lo:rest] = tail[:, 0]
            o[:, 1].view(hkv, D, blk)[:, :, lo:rest] = tail[:, 1].transpose(1, 2)
    out = {"codes": codes, "scales": scales, "open": opened}
    return out if meta is None else {**out, "meta": meta}


def _exact_read(c, s):
    hkv, blk = c["Hkv"], c["blk"]
    out = torch.empty((s["rows"], hkv, 2, D), dtype=torch.float64, device="cuda")
    length, begin, table = s["len"].cpu().numpy(), s["row_begin"].cpu().numpy(), s["tables"].long()
    for b in range(c["B"]):
        n, full = int(length[b]), int(length[b]) // blk
        for h in range(hkv):
            r0 = int(begin[b])
            if full:
                kv = _exact_tiles(s["records"][h, table[b, :full]], blk, c["fmt"])
                out[r0:r0 + full * blk, h] = kv.transpose(1, 2).reshape(full * blk, 2, D)
            o, rest = s["open"][b, h].double().view(2, -1), n - full * blk
            out[r0 + full * blk:r0 + n, h, 0] = o[0].view(blk, D)[:rest]
            out[r0 + full * blk:r0 + n, h, 1] = o[1].view(D, blk).t()[:rest]
    return out


def _exact_attend(c, s):
    hkv, blk, G = c["Hkv"], c["blk"], c["Hq"] // c["Hkv"]
    out = torch.zeros((c["B"], c["Hq"], D), dtype=torch.float64, device="cuda")
    length = s["len"].cpu().numpy()
    for b in range(c["B"]):
        for h in range(hkv):
            if c["mode"] == "dense":
                page = s["tables"][b, :int(length[b]) // blk][:c["k"]].long()
            else:
                page = s["sel"][b, h].long()
                page = page[page >= 0]
                if c["mode"] == "sparse":
                    page = s["tables"][b].long()[page]
            kv = _exact_tiles((s["records"][b, h] if c["mode"] == "slots" else s["records"][h])[page], blk, c["fmt"])
            k, v = kv[:, 0].reshape(-1, D), kv[:, 1].reshape(-1, D)
            if c["mode"] == "dense":
                o, rest = s["open"][b, h].double().view(2, -1), int(length[b]) % blk
                k = torch.cat([k, o[0].view(blk, D)[:rest]])
                v = torch.cat([v, o[1].view(D, blk).t()[:rest]])
            if not len(k):
                continue
            z = (s["q"][b, h * G:(h + 1) * G].double() @ k.t().contiguous()) / math.sqrt(D)
            out[b, h * G:(h + 1) * G] = torch.softmax(z, -1) @ v
    return out


def exact(case, seed):
    if case["kind"] == "tables":
        return None  # whole numbers
    s = prepare(case, seed)
    return {"write": _exact_write, "read": _exact_read, "attend": _exact_attend}[case["kind"]](case, s)
