"""Cases of the operators around the 4-bit KV cache, with their plain forms and their 64-bit definitions.

  pages    pages taken and given back for a batch of growing / shrinking requests, with slot and position per token
  rope     RMS norm of every query and key head and the position rotation, from the projections to what the path takes
  store    tokens into 4-bit blocks through a slot map, and the blocks read back as bf16
  append   one decode step's token into pool and store, with the slot taken for a block that has just been opened
  attn     one layer's sparse decode attention over a pool of 4-bit blocks

Layout of a 4-bit block: [kv head][16-token tile][2560 bytes], the whole padded to a multiple of 4096 bytes.  A tile is
K codes [16][64 B], V codes [16][64 B], K scales [16][4 groups][scale, minimum] bf16, V scales likewise.  Channel
d = 32 j + 8 c + i of a K row is nibble i of the 32-bit word at byte 16 c + 4 j; channel d = 32 j + 4 r + i of a V row is
nibble i of the 16-bit word at byte 8 r + 2 j.  The value is scale * code + minimum.
"""
import math
import random

import torch

own = False

D = 128
TILE = 2560
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _ceil(a, b):
    return -(-a // b)


def _block_bytes(case):
    return _ceil(case["kv_heads"] * case["block"] * 160, 4096) * 4096


# ------------------------------------------------------------------ cases
def listed():
    return [
        # a decode step of 16 long sequences, 4 draft tokens each, then the rejected drafts rolled back
        {"name": "pages 16 x 4 drafts", "op": "pages", "batch": 16, "kv_heads": 8, "block": 16, "row": 2048, "start": 32000, "grow": 4, "ragged": True},
        # 64 prompts of up to 131 072 tokens admitted at once, later retired
        {"name": "pages 64 prompts", "op": "pages", "batch": 64, "kv_heads": 8, "block": 32, "row": 4096, "start": 0, "grow": 131072, "ragged": True},
        # one decode step of the 8B-shaped model with 16 sequences, projections fused into one tensor
        {"name": "rope 16 tokens", "op": "rope", "tokens": 16, "heads": 32, "kv_heads": 8, "dtype": "bf16", "fused": True, "norm": True, "rot": 128, "interleaved": False, "span": 32768, "pad": 0},
        # a prompt chunk of the 70B-shaped model, half of each head rotated in neighbouring pairs, fp16 projections, odd length
        {"name": "rope 2049 tokens fp16", "op": "rope", "tokens": 2049, "heads": 64, "kv_heads": 8, "dtype": "fp16", "fused": False, "norm": True, "rot": 64, "interleaved": True, "span": 131072, "pad": 5},
        # a whole 32 768-token prompt
        {"name": "rope 32768 tokens", "op": "rope", "tokens": 32768, "heads": 32, "kv_heads": 8, "dtype": "bf16", "fused": True, "norm": True, "rot": 128, "interleaved": False, "span": 32768, "pad": 0},
        # a prompt's tail: a ragged handful of tokens into scattered pages
        {"name": "store 333 tokens", "op": "store", "tokens": 333, "kv_heads": 8, "block": 16, "pages": 32, "pad": 3},
        # a full context of the long-context workload
        {"name": "store 131072 tokens", "op": "store", "tokens": 131072, "kv_heads": 8, "block": 32, "pages": 4096, "pad": 0},
        # a decode step's append at the 8B shape, and at the long-context one with 64 sequences
        {"name": "append 16", "op": "append", "batch": 16, "kv_heads": 8, "block": 16, "row": 2048, "slots": 409, "sink": 1, "local": 8, "ctx": 32000},
        {"name": "append 64 x 32-token blocks", "op": "append", "batch": 64, "kv_heads": 8, "block": 32, "row": 512, "slots": 64, "sink": 1, "local": 4, "ctx": 15000},
        # one sequence with a small budget: latency
        {"name": "attn 1 x 64 blocks", "op": "attn", "batch": 1, "heads": 32, "kv_heads": 8, "block": 16, "budget": 64, "slots": 128, "ctx": 8192, "ragged": False},
        # the 8B-shaped layer step
        {"name": "attn 16 x 128 blocks", "op": "attn", "batch": 16, "heads": 32, "kv_heads": 8, "block": 16, "budget": 128, "slots": 409, "ctx": 32768, "ragged": False},
        # the long-context workload, ragged: some sequences shorter than the budget
        {"name": "attn 64 x 64 blocks of 32", "op": "attn", "batch": 64, "heads": 32, "kv_heads": 8, "block": 32, "budget": 64, "slots": 409, "ctx": 131072, "ragged": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["pages", "rope", "rope", "store", "append", "attn", "attn", "attn"])
    kv = rng.choice([1, 2, 4, 8, 8, 16])
    block = rng.choice([16, 16, 32, 64])
    if op == "pages":
        batch = _log(rng, 1, 64)
        row = _log(rng, 16, 4096)
        start = rng.choice([0, _log(rng, 1, row * block // 2)])
        grow = _log(rng, 1, min(131072, row * block - start))
        return {"op": op, "batch": batch, "kv_heads": 8, "block": block, "row": row, "start": start, "grow": grow, "ragged": rng.random() < 0.8}
    if op == "rope":
        heads = kv * rng.choice([1, 2, 4, 5, 7, 8, 16])
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        most = 32768 * 40 * 512 // ((heads + kv) * D * (6 if dtype == "fp32" else 4))
        tokens = _log(rng, 1, min(32768, most))
        return {"op": op, "tokens": tokens, "heads": heads, "kv_heads": kv, "dtype": dtype, "fused": rng.random() < 0.5, "norm": rng.random() < 0.8,
                "rot": rng.choice([128, 128, 64, 32, 96, 2]), "interleaved": rng.random() < 0.4, "span": _log(rng, 1, 1 << 20), "pad": rng.choice([0, 0, 1, tokens // 3])}
    if op == "store":
        tokens = _log(rng, 1, 131072 * 8 // max(8, kv))
        return {"op": op, "tokens": tokens, "kv_heads": kv, "block": block, "pages": _ceil(tokens, block) + rng.randrange(0, 3), "pad": rng.choice([0, tokens // 4])}
    if op == "append":
        slots = _log(rng, 16, 409)
        row = slots + _log(rng, 2, 512)
        return {"op": op, "batch": _log(rng, 1, 64), "kv_heads": rng.choice([1, 2, 4, 8]), "block": block, "row": row, "slots": slots, "sink": rng.choice([0, 1]), "local": rng.choice([1, 4, 8]),
                "ctx": rng.randrange(slots * block, (row - 1) * block)}
    group = rng.choice([1, 2, 3, 4, 4, 6, 8, 8, 12, 16])
    batch = _log(rng, 1, 64)
    most = max(2, min(1024, 64 * 64 * 32 * 8 // (batch * kv * block)))
    budget = _log(rng, 2, most)
    ctx = max(1, _log(rng, 1, min(131072, 8192 * block)))
    return {"op": op, "batch": batch, "heads": kv * group, "kv_heads": kv, "block": block, "budget": budget, "slots": budget + rng.randrange(0, 64), "ctx": ctx, "ragged": rng.random() < 0.7}


def _lengths(case):
    """New tokens per sequence, and where each starts (pages): the same for every seed, so that the work is known."""
    r = random.Random(case["batch"] * 1000003 + case["grow"])
    most = case["row"] * case["block"]
    old = [max(0, case["start"] - (r.randrange(0, case["block"] * 4) if case["ragged"] and case["start"] else 0)) for _ in range(case["batch"])]
    add = [r.randrange(_ceil(case["grow"], 8), case["grow"] + 1) if case["ragged"] else case["grow"] for _ in range(case["batch"])]
    return old, [min(most, o + a) for o, a in zip(old, add)]


def _contexts(case):
    """Context length of every sequence (attn, append)."""
    r = random.Random(case["batch"] * 7919 + case["ctx"])
    if case["op"] == "append":
        lo = (case["sink"] + case["local"] + 1) * case["block"]
        return [max(lo, case["ctx"] - r.randrange(0, 4 * case["block"])) if i % 5 else max(lo, case["ctx"]) // case["block"] * case["block"] for i in range(case["batch"])]
    if not case["ragged"]:
        return [case["ctx"]] * case["batch"]
    got = [r.randrange(1, case["ctx"] + 1) for _ in range(case["batch"])]
    if case["batch"] > 3:
        got[1] = 0  # a sequence that has just been retired: nothing selected
        got[2] = min(case["ctx"], case["budget"] * case["block"] // 2 + 1)
    return got


# ------------------------------------------------------------------ handles
_contexts_kept = {}


def _handle(case):
    """The framework's context of a model shape: one per shape, kept by the program."""
    from paper_2609_34555_b200 import PulseInfer
    op = case["op"]
    key = dict(n_layers=1, n_q_heads=case.get("heads", case["kv_heads"]), n_kv_heads=case["kv_heads"], block_tokens=case.get("block", 16),
               budget_blocks=case.get("budget", 16), n_sink_blocks=case.get("sink", 0) if op == "append" else 0, n_local_blocks=case.get("local", 1) if op == "append" else 0,
               pool_slots=case.get("slots", 16), max_batch=case.get("batch", 1), max_blocks=case.get("row", _ceil(max(1, case.get("ctx", 1)), case.get("block", 16))))
    key["budget_blocks"] = max(key["budget_blocks"], key["n_sink_blocks"] + key["n_local_blocks"])
    name = tuple(sorted(key.items()))
    if name not in _contexts_kept:
        _contexts_kept[name] = PulseInfer(solo_head=[0], **key)
    return _contexts_kept[name]


# ------------------------------------------------------------------ the 4-bit format, plainly
def _quantise(x):
    """x fp32 [..., 128] -> codes int32 [..., 128], scale and minimum fp32 [..., 4] (both bf16 numbers)."""
    g = x.unflatten(-1, (4, 32))
    lo = g.amin(-1)
    s = ((g.amax(-1) - lo) / 15).to(torch.bfloat16).float()
    c = torch.where(s[..., None] > 0, torch.round((g - lo[..., None]) / s[..., None]), torch.zeros_like(g)).clamp(0, 15)
    return c.flatten(-2).to(torch.int32), s, lo


def _code_bytes(code, value):
    """codes [..., 128] -> bytes [..., 64] in the order of K rows (value False) or V rows."""
    if value:
        c = code.unflatten(-1, (4, 8, 4)).transpose(-3, -2)  # [r][j][i]
    else:
        c = code.unflatten(-1, (4, 4, 8)).transpose(-3, -2)  # [c][j][i]
    c = c.flatten(-3).unflatten(-1, (64, 2))
    return (c[..., 0] + 16 * c[..., 1]).to(torch.uint8)


def _scale_bytes(s, lo):
    return torch.stack((s, lo), -1).to(torch.bfloat16).flatten(-2).view(torch.uint8)


def _dequantise(tiles):
    """tiles uint8 [..., 2560] -> K, V fp32 [..., 16, 128]."""
    def nibbles(b):
        b = b.to(torch.int32)
        return torch.stack((b & 15, b >> 4), -1).flatten(-2).float()
    k = nibbles(tiles[..., :1024].unflatten(-1, (16, 4, 4, 4))).transpose(-3, -2)        # [16][j][c][8]
    v = nibbles(tiles[..., 1024:2048].unflatten(-1, (16, 8, 4, 2))).transpose(-3, -2)    # [16][j][r][4]
    sz = tiles[..., 2048:].contiguous().view(torch.bfloat16).unflatten(-1, (2, 16, 4, 2)).float()
    k = k.flatten(-2) * sz[..., 0, :, :, 0, None] + sz[..., 0, :, :, 1, None]
    v = v.flatten(-2) * sz[..., 1, :, :, 0, None] + sz[..., 1, :, :, 1, None]
    return k.flatten(-2), v.flatten(-2)


def _tiles(blocks, case):
    """blocks uint8 [..., block bytes] -> [..., kv heads, tiles, 2560]."""
    n = case["kv_heads"] * case["block"] * 160
    return blocks[..., :n].unflatten(-1, (case["kv_heads"], case["block"] // 16, TILE))


def _values(blocks, case):
    """blocks uint8 [n, block bytes] -> bf16 [n][kv heads][2][block][128]."""
    k, v = _dequantise(_tiles(blocks, case))
    return torch.stack((k.flatten(2, 3), v.flatten(2, 3)), 2).to(torch.bfloat16)


def _rows(k, v):
    """K and V rows bf16 [...][128] -> the bytes of one token's place in a tile: K codes 64, V codes 64, K scales 16, V scales 16."""
    ck, sk, zk = _quantise(k.float())
    cv, sv, zv = _quantise(v.float())
    return _code_bytes(ck, False), _code_bytes(cv, True), _scale_bytes(sk, zk), _scale_bytes(sv, zv)


def _into_tile(tiles, where, rows):
    """tiles [n][h][t][2560] with the rows ([n][h][bytes]) at the tokens where `where` [n][t][16] is true."""
    w = where[:, None, :, :, None]
    parts = [(0, 1024, 64), (1024, 2048, 64), (2048, 2304, 16), (2304, 2560, 16)]
    got = [torch.where(w, r[:, :, None, None, :], tiles[..., a:b].unflatten(-1, (16, size))).flatten(-2) for (a, b, size), r in zip(parts, rows)]
    return torch.cat(got, -1)


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    st = {"case": case, "pi": _handle(case) if own else None}
    i32 = dict(dtype=torch.int32, device=DEV)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    op = case["op"]
    if op == "pages":
        old, new = _lengths(case)
        B = case["block"]
        held = sum(_ceil(o, B) for o in old)
        n = held + sum(_ceil(b, B) - _ceil(a, B) for a, b in zip(old, new)) + 37
        perm = torch.randperm(n, generator=g, device=DEV).to(torch.int32)
        st["old"], st["new"] = torch.tensor(old, **i32), torch.tensor(new, **i32)
        ob = (st["old"] + B - 1) // B
        j = torch.arange(case["row"], **i32)[None]
        at = (ob.cumsum(0) - ob)[:, None] + j
        st["table"] = torch.where(j < ob[:, None], perm[at.clamp(max=n - 1).long()], -1).to(torch.int32).contiguous()
        st["ring"] = torch.cat((perm[held:], torch.full((held,), -1, **i32))).contiguous()
        st["state"] = torch.tensor([0, n - held, 0, 0], dtype=torch.int64, device=DEV)
        total = sum(b - a for a, b in zip(old, new))
        st["total"] = total + 5  # a token buffer a little larger than the batch
        st["slots"] = torch.zeros(st["total"], dtype=torch.int64, device=DEV)
        st["positions"] = torch.zeros(st["total"], **i32)
        st["starts"] = torch.zeros(case["batch"] + 1, **i32)
    elif op == "rope":
        T, Hq, Hk, dt = case["tokens"], case["heads"], case["kv_heads"], DTYPES[case["dtype"]]
        if case["fused"]:  # one projection: queries, keys and values of a token side by side
            x = normal(T, (Hq + 2 * Hk) * D).mul_(1.5).to(dt)
            st["q"], st["k"] = x[:, :Hq * D].unflatten(1, (Hq, D)), x[:, Hq * D:(Hq + Hk) * D].unflatten(1, (Hk, D))
        else:
            st["q"], st["k"] = normal(T, Hq, D).mul_(1.5).to(dt), normal(T, Hk, D).mul_(1.5).to(dt)
        st["positions"] = torch.randint(0, case["span"], (T,), generator=g, **i32)
        if case["pad"]:
            st["positions"][T - case["pad"]:] = -1  # padding behind the last sequence
        st["inv_freq"] = (500000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=DEV) / case["rot"])).float()
        st["wq"] = 1 + 0.2 * normal(D) if case["norm"] else None
        st["wk"] = 1 + 0.2 * normal(D) if case["norm"] else None
        st["q_out"] = torch.zeros((T, Hq, D), dtype=torch.bfloat16, device=DEV)
        st["k_out"] = torch.zeros((T, Hk, D), dtype=torch.bfloat16, device=DEV)
    elif op == "store":
        T, H = case["tokens"], case["kv_heads"]
        kv = normal(T, 2 * H * D).to(torch.bfloat16)
        st["k"], st["v"] = kv[:, :H * D].unflatten(1, (H, D)), kv[:, H * D:].unflatten(1, (H, D))
        page = torch.randperm(case["pages"], generator=g, device=DEV)
        t = torch.arange(T, device=DEV)
        st["slots"] = page[t // case["block"]] * case["block"] + t % case["block"]
        if case["pad"]:
            st["slots"][T - case["pad"]:] = -1
        st["store"] = torch.zeros((case["pages"], _block_bytes(case)), dtype=torch.uint8, device=DEV)
        st["out"] = torch.zeros((case["pages"], H, 2, case["block"], D), dtype=torch.bfloat16, device=DEV)
    elif op == "append":
        n, H, B, NB, C = case["batch"], case["kv_heads"], case["block"], case["row"], case["slots"]
        ctx = torch.tensor(_contexts(case), **i32)
        st["ctx"], st["step"] = ctx, 1000
        cur = ctx // B
        j = torch.arange(NB, **i32)[None].expand(n, NB)
        keep = (j < case["sink"]) | (j > (cur - case["local"])[:, None])
        may = (j < cur[:, None]) | ((j == cur[:, None]) & (ctx % B > 0)[:, None])
        score = torch.rand((n, NB), generator=g, device=DEV) + 2.0 * keep - 8.0 * ~may
        top = score.topk(C, dim=1)
        order = torch.rand((n, C), generator=g, device=DEV).argsort(1)
        blocks = torch.where(top.values > -4, top.indices, -1).gather(1, order)
        st["slot_block"] = blocks.to(torch.int32).contiguous()
        table = torch.full((n, NB + 1), -1, **i32)
        table.scatter_(1, torch.where(blocks < 0, NB, blocks), torch.arange(C, **i32)[None].expand(n, C).contiguous())
        st["table"] = table[:, :NB].contiguous()
        st["stamp"] = torch.randint(0, 900, (n, C), generator=g, **i32)
        st["k"], st["v"] = normal(n, H, D).to(torch.bfloat16), normal(n, H, D).to(torch.bfloat16)
        st["digest"] = torch.stack((normal(n, NB, D) - 2, normal(n, NB, D) + 2), 2).to(torch.bfloat16)
        # the block that is being filled already holds rows; the others are not looked at
        st["pool"] = torch.zeros((n, C, _block_bytes(case)), dtype=torch.uint8, device=DEV)
        st["store"] = torch.zeros((n, NB, _block_bytes(case)), dtype=torch.uint8, device=DEV)
        st["store_ids"] = (torch.arange(n, **i32) * NB + cur).contiguous()
        first = torch.arange(n, **i32) * C
        st["first"], st["cur"] = first, cur[:, None].long().contiguous()
        held = st["table"].gather(1, st["cur"])[:, 0]
        some = _tiles_of(normal(n, H, 2, B, D), case)
        st["store"].view(n * NB, -1)[st["store_ids"].long()] = some
        at = (first + held.clamp(min=0)).long()
        st["pool"].view(n * C, -1)[at] = torch.where(held[:, None] >= 0, some, st["pool"].view(n * C, -1)[at])
        st["pool_out"] = torch.zeros((n, H, 2, B, D), dtype=torch.bfloat16, device=DEV)
        st["store_out"] = torch.zeros((n, H, 2, B, D), dtype=torch.bfloat16, device=DEV)
    else:
        n, H, B, K, C = case["batch"], case["kv_heads"], case["block"], case["budget"], case["slots"]
        lens = _contexts(case)
        st["ctx"] = torch.tensor(lens, **i32)
        nb = (st["ctx"] + B - 1) // B
        NB = _ceil(max(1, max(lens)), B)
        st["count"] = nb.clamp(max=K).to(torch.int32)
        # selected: the newest block and others at random, ascending; slots of the pool at random
        j = torch.arange(NB, **i32)[None].expand(n, NB)
        score = torch.rand((n, NB), generator=g, device=DEV) + 2.0 * (j == nb[:, None] - 1) - 8.0 * (j >= nb[:, None])
        top = score.topk(min(K, NB), dim=1)
        sel = torch.where(top.values > -4, top.indices, 1 << 30).sort(1).values
        sel = torch.nn.functional.pad(sel, (0, K - sel.shape[1]), value=1 << 30)
        st["blocks"] = torch.where(sel < 1 << 30, sel, -1).to(torch.int32).contiguous()
        slots = torch.rand((n, C), generator=g, device=DEV).argsort(1)[:, :K].to(torch.int32)
        st["slots"] = torch.where(st["blocks"] >= 0, slots, -1).contiguous()
        st["q"] = normal(n, case["heads"], D).to(torch.bfloat16)
        st["pool"] = torch.empty((n, C, _block_bytes(case)), dtype=torch.uint8, device=DEV)
        for s in range(n):
            st["pool"][s] = _tiles_of(normal(C, H, 2, B, D) * (1 + 0.3 * normal(1, H, 2, 1, D)), case)
        st["out"] = torch.zeros((n, case["heads"], D), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.zeros((n, case["heads"]), dtype=torch.float32, device=DEV)
    return st


def _tiles_of(kv, case):
    """fp32 [n][h][2][block][128] -> whole 4-bit blocks uint8 [n][block bytes]."""
    n, H, B = kv.shape[0], case["kv_heads"], case["block"]
    rows = _rows(kv[:, :, 0].to(torch.bfloat16), kv[:, :, 1].to(torch.bfloat16))     # each [n][h][B][bytes]
    tiles = torch.cat([r.reshape(n, H, B // 16, -1) for r in rows], -1)
    return torch.nn.functional.pad(tiles.reshape(n, -1), (0, _block_bytes(case) - H * B * 160))


# ------------------------------------------------------------------ one pass
def run(st):
    case, pi, op = st["case"], st["pi"], st["case"]["op"]
    if own:
        if op == "pages":
            pi.assign_pages(st["old"], st["new"], st["table"], st["ring"], st["state"], st["starts"], st["slots"], st["positions"])
            pi.assign_pages(st["new"], st["old"], st["table"], st["ring"], st["state"])
            return st["slots"], st["positions"], st["starts"], st["table"], st["ring"], st["state"]
        if op == "rope":
            pi.qk_norm_rope(st["q"], st["k"], st["positions"], st["inv_freq"], st["q_out"], st["k_out"], q_weight=st["wq"], k_weight=st["wk"],
                            eps=1e-6, interleaved=case["interleaved"])
            return st["q_out"], st["k_out"]
        if op == "store":
            pi.kv4_store(st["k"], st["v"], st["store"], st["slots"])
            pi.kv4_load(st["store"], st["out"])
            return st["out"]
        if op == "append":
            pi.append_kv4(0, st["step"], st["k"], st["v"], st["ctx"], st["store"], st["pool"], st["table"], st["slot_block"], st["stamp"], st["digest"])
            ids = st["table"].gather(1, st["cur"])[:, 0] + st["first"]
            pi.kv4_load(st["pool"], st["pool_out"], ids)
            pi.kv4_load(st["store"], st["store_out"], st["store_ids"])
            return st["table"], st["slot_block"], st["stamp"], st["digest"], st["pool_out"], st["store_out"]
        pi.sparse_decode_attn_kv4(0, st["q"], st["pool"], st["slots"], st["blocks"], st["count"], st["ctx"], st["out"], st["lse"])
        return st["out"], st["lse"]
    return {"pages": _plain_pages, "rope": _plain_rope, "store": _plain_store, "append": _plain_append, "attn": _plain_attn}[op](st)


def _plain_assign(st, old, new):
    """Table, ring and state after the change of lengths."""
    case, n = st["case"], st["ring"].shape[0]
    B = case["block"]
    ob, nb = (old + B - 1) // B, (new + B - 1) // B
    grow, shrink = (nb - ob).clamp(min=0).long(), (ob - nb).clamp(min=0).long()
    g0, s0 = grow.cumsum(0) - grow, shrink.cumsum(0) - shrink
    head, tail = st["state"][0], st["state"][1]
    j = torch.arange(case["row"], device=DEV)[None]
    taken = (j >= ob[:, None]) & (j < nb[:, None])
    freed = (j >= nb[:, None]) & (j < ob[:, None])
    page = st["ring"][(head + g0[:, None] + j - ob[:, None]).clamp(min=0) % n]
    ring = torch.cat((st["ring"], st["ring"][:1]))  # one more place, for what is not freed
    ring.scatter_(0, torch.where(freed, (tail + s0[:, None] + j - nb[:, None]) % n, n).flatten(), st["table"].flatten())
    st["ring"].copy_(ring[:n])
    st["table"].copy_(torch.where(taken, page, torch.where(freed, -1, st["table"])))
    st["state"][0] += grow.sum()
    st["state"][1] += shrink.sum()


def _plain_pages(st):
    case, old, new, T = st["case"], st["old"], st["new"], st["total"]
    B = case["block"]
    _plain_assign(st, old, new)
    add = (new - old).clamp(min=0)
    starts = torch.nn.functional.pad(add.cumsum(0), (1, 0)).to(torch.int32)
    t = torch.arange(T, device=DEV, dtype=torch.int32)
    s = torch.searchsorted(starts, t, right=True).clamp(max=case["batch"]) - 1
    real = t < starts[-1]
    pos = torch.where(real, old[s] + t - starts[s], 0)
    slot = st["table"].flatten()[s * case["row"] + pos // B].long() * B + pos % B
    slots, positions = torch.where(real, slot, -1), torch.where(real, pos, -1).to(torch.int32)
    _plain_assign(st, new, old)
    return slots, positions, starts, st["table"], st["ring"], st["state"]


def _plain_rope(st):
    case, rot = st["case"], st["case"]["rot"]
    angle = st["positions"].double()[:, None] * st["inv_freq"].double()
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def one(x, w, before):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
        r = x[..., :rot]
        a, b = (r[..., 0::2], r[..., 1::2]) if case["interleaved"] else (r[..., :rot // 2], r[..., rot // 2:])
        u, v = a * c - b * s, b * c + a * s
        r = torch.stack((u, v), -1).flatten(-2) if case["interleaved"] else torch.cat((u, v), -1)
        y = torch.cat((r, x[..., rot:]), -1).to(torch.bfloat16)
        return torch.where(st["positions"][:, None, None] >= 0, y, before)

    return one(st["q"], st["wq"], st["q_out"]), one(st["k"], st["wk"], st["k_out"])


def _plain_store(st):
    case, H, B = st["case"], st["case"]["kv_heads"], st["case"]["block"]
    kc, vc, ks, vs = _rows(st["k"], st["v"])
    slot = torch.where(st["slots"] >= 0, st["slots"], case["pages"] * B)  # one page more, for what is not stored
    page, at = slot // B, slot % B
    tiles = torch.nn.functional.pad(_tiles(st["store"], case).flatten(1), (0, 0, 0, 1)).view(case["pages"] + 1, H, B // 16, TILE)
    base = tiles.permute(0, 2, 1, 3)[page, at // 16]  # only for its shape: [T][H][2560]
    row = (at % 16)[:, None, None]
    lane64, lane16 = torch.arange(64, device=DEV), torch.arange(16, device=DEV)
    index = torch.cat((row * 64 + lane64, 1024 + row * 64 + lane64, 2048 + row * 16 + lane16, 2304 + row * 16 + lane16), -1).expand(base.shape[0], H, 160)
    head = torch.arange(H, device=DEV)[None, :, None]
    flat = ((page[:, None, None] * H + head) * (B // 16) + (at // 16)[:, None, None]) * TILE + index
    out = tiles.flatten().scatter(0, flat.flatten(), torch.cat((kc, vc, ks, vs), -1).flatten())
    blocks = out.view(case["pages"] + 1, -1)[:-1]
    st["store"][:, :H * B * 160].copy_(blocks)
    return _values(blocks, case)


def _plain_append(st):
    case, n, B, C, NB = st["case"], st["case"]["batch"], st["case"]["block"], st["case"]["slots"], st["case"]["row"]
    cur, t = st["cur"], (st["ctx"] % B).long()
    slot = st["table"].gather(1, cur)[:, 0].long()
    opens = (t == 0) & (slot < 0)
    sb = st["slot_block"]
    pinned = (sb >= 0) & ((sb < case["sink"]) | (sb >= cur + 1 - case["local"]))
    key = torch.where(pinned, 1 << 62, (st["stamp"].long() << 32) + torch.arange(C, device=DEV))
    victim = key.argmin(1)
    old = sb.gather(1, victim[:, None])[:, 0].long()
    at = torch.where(opens & (old >= 0), old, cur[:, 0])
    st["table"].scatter_(1, at[:, None], -1)
    slot = torch.where(opens, victim, slot)
    st["table"].scatter_(1, cur, slot[:, None].to(torch.int32))
    sb.scatter_(1, slot[:, None], cur.to(torch.int32))
    st["stamp"].scatter_(1, slot[:, None], st["step"])
    rows = _rows(st["k"], st["v"])
    token = torch.arange(B, device=DEV).view(1, B // 16, 16) == t[:, None, None]
    ids = st["first"].long() + slot

    def write(buffer, ids):
        blocks = buffer.flatten(0, 1)[ids]
        tiles = _into_tile(torch.where((t == 0)[:, None, None, None], 0, _tiles(blocks, case)), token, rows)
        blocks = torch.nn.functional.pad(tiles.flatten(1), (0, blocks.shape[1] - tiles[0].numel()))
        buffer.flatten(0, 1).index_copy_(0, ids, blocks)
        return _values(blocks, case)

    pool, store = write(st["pool"], ids), write(st["store"], st["store_ids"].long())
    d = st["digest"].flatten(0, 1)[st["store_ids"].long()]
    k = st["k"][:, 0]
    new = torch.where((t == 0)[:, None, None], torch.stack((k, k), 1), torch.stack((torch.minimum(d[:, 0], k), torch.maximum(d[:, 1], k)), 1))
    st["digest"].flatten(0, 1).index_copy_(0, st["store_ids"].long(), new)
    return st["table"], sb, st["stamp"], st["digest"], pool, store


def _plain_attn(st):
    case, n, H, B, K = st["case"], st["case"]["batch"], st["case"]["kv_heads"], st["case"]["block"], st["case"]["budget"]
    slots = st["slots"].clamp(min=0).long() + torch.arange(n, device=DEV)[:, None] * case["slots"]
    tiles = _tiles(st["pool"].flatten(0, 1)[slots], case)  # [n][K][H][tiles][2560]
    k, v = (x.flatten(3, 4).transpose(1, 2).flatten(2, 3) for x in _dequantise(tiles))  # [n][H][K * B][128]
    q = st["q"].float().unflatten(1, (H, case["heads"] // H))
    s = (q @ k.transpose(-1, -2)) / math.sqrt(D)
    token = st["blocks"][:, :, None] * B + torch.arange(B, device=DEV)
    seen = (st["blocks"] >= 0)[:, :, None] & (token < st["ctx"][:, None, None]) & (torch.arange(K, device=DEV)[:, None] < st["count"][:, None, None])
    seen = seen.flatten(1)[:, None, None]
    s = torch.where(seen, s, -math.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - m)
    l = p.sum(-1, keepdim=True)
    o = p @ torch.where(seen.transpose(-1, -2), v, 0.0) / torch.where(l > 0, l, 1.0)
    return o.flatten(1, 2).to(torch.bfloat16), (m + torch.log(l))[..., 0].flatten(1)


# ------------------------------------------------------------------ work of a pass
def work(case):
    op = case["op"]
    if op == "pages":
        old, new = _lengths(case)
        B = case["block"]
        pages = sum(_ceil(b, B) - _ceil(a, B) for a, b in zip(old, new))
        tokens = sum(b - a for a, b in zip(old, new)) + 5
        # lengths twice; a page is read from the ring and written to the table, then the other way round
        return {"bytes": case["batch"] * 20 + pages * (4 + 4 + 4 + 4 + 4) + tokens * 12, "flops": 0}
    if op == "rope":
        values = (case["tokens"] - case["pad"]) * (case["heads"] + case["kv_heads"]) * D
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": values * (size + 2) + case["tokens"] * 4 + case["rot"] * 2, "flops": values * 8}
    if op == "store":
        rows = (case["tokens"] - case["pad"]) * case["kv_heads"]
        held = case["pages"] * case["block"] * case["kv_heads"]
        return {"bytes": rows * (512 + 160) + case["tokens"] * 8 + held * (160 + 512), "flops": (rows + held) * 256 * 3}
    if op == "append":
        B, H = case["block"], case["kv_heads"]
        # new rows in, pool and store rows out, the digest, a scan of the slots' blocks and stamps; the block read back twice
        return {"bytes": case["batch"] * (H * (512 + 2 * 160) + 1024 + case["slots"] * 8 + 2 * B * H * (160 + 512)), "flops": case["batch"] * H * B * 256 * 4}
    tokens = sum(min(c, case["budget"] * case["block"]) for c in _contexts(case))
    return {"bytes": tokens * case["kv_heads"] * 160 + case["batch"] * (case["heads"] * (D * 4 + 4) + case["budget"] * 8), "flops": 4 * tokens * case["heads"] * D}


# ------------------------------------------------------------------ the definitions in 64 bits
def _places():
    """For each channel: byte and shift in a K row, byte and shift in a V row."""
    kb, ks, vb, vs = [], [], [], []
    for d in range(D):
        j, x = divmod(d, 32)
        kb.append(16 * (x // 8) + 4 * j + (x % 8) // 2)
        ks.append(4 * (x % 2))
        vb.append(8 * (x // 4) + 2 * j + (x % 4) // 2)
        vs.append(4 * (x % 2))
    return [torch.tensor(x, device=DEV) for x in (kb, ks, vb, vs)]


def _read64(blocks, case):
    """Packed blocks [n][bytes] -> K, V float64 [n][h][block][128], channel by channel."""
    H, B = case["kv_heads"], case["block"]
    t = blocks[:, :H * B * 160].reshape(blocks.shape[0], H, B // 16, TILE)
    kb, ks, vb, vs = _places()
    group = torch.arange(D, device=DEV) // 32
    got = []
    for code, scale, byte, shift in ((0, 2048, kb, ks), (1024, 2304, vb, vs)):
        rows = t[..., code:code + 1024].reshape(blocks.shape[0], H, B, 64)
        sz = t[..., scale:scale + 256].reshape(blocks.shape[0], H, B, 8, 2).to(torch.int32)
        f = ((sz[..., 0] + 256 * sz[..., 1]) << 16).view(torch.float32).double()  # a bf16 number is the upper half of an fp32 one
        c = (rows[..., byte].to(torch.int32) >> shift) & 15
        got.append(f[..., 0::2][..., group] * c.double() + f[..., 1::2][..., group])
    return got


def _round64(x):
    """What 4 bits keep of rows [..., 128], in 64 bits."""
    g = x.double().reshape(x.shape[:-1] + (4, 32))
    lo, hi = g.min(-1, keepdim=True).values, g.max(-1, keepdim=True).values
    s = ((hi - lo) / 15).to(torch.bfloat16).double()
    c = torch.round((g - lo) / torch.where(s > 0, s, torch.ones_like(s))).clamp(0, 15)
    return torch.where(s > 0, lo + s * c, lo).reshape(x.shape)


def exact(case, seed):
    op = case["op"]
    if op == "pages":
        return None  # whole numbers only
    global own
    kept, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = kept
    if op == "rope":
        rot, half = case["rot"], case["rot"] // 2
        out = []
        for x, w in ((st["q"], st["wq"]), (st["k"], st["wk"])):
            x = x.double()
            if w is not None:
                x = x / (x.pow(2).sum(-1, keepdim=True) / D + 1e-6).sqrt() * w.double()
            z = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), st["positions"].double()[:, None] * st["inv_freq"].double()[None])[:, None]
            i = torch.arange(half, device=DEV)
            a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
            turned = torch.complex(x[..., a], x[..., b]) * z
            x[..., a], x[..., b] = turned.real, turned.imag
            x[st["positions"] < 0] = 0
            out.append(x)
        return tuple(out)
    if op == "store":
        H, B = case["kv_heads"], case["block"]
        out = torch.zeros((case["pages"], H, 2, B, D), dtype=torch.float64, device=DEV)
        real = st["slots"] >= 0
        p, r = st["slots"][real] // B, st["slots"][real] % B
        out[p, :, 0, r] = _round64(st["k"][real])
        out[p, :, 1, r] = _round64(st["v"][real])
        return out
    if op == "append":
        ctx = _contexts(case)
        B = case["block"]
        rows = st["store"].flatten(0, 1)[st["store_ids"].long()]
        k, v = _read64(rows, case)
        digest = st["digest"].double()
        for s, c in enumerate(ctx):
            b, t = divmod(c, B)
            if t == 0:
                k[s], v[s] = 0, 0
            k[s, :, t], v[s, :, t] = _round64(st["k"][s]), _round64(st["v"][s])
            x = st["k"][s, 0].double()
            digest[s, b, 0] = x if t == 0 else torch.minimum(digest[s, b, 0], x)
            digest[s, b, 1] = x if t == 0 else torch.maximum(digest[s, b, 1], x)
        both = torch.stack((k, v), 2)
        return None, None, None, digest, both, both
    G, B = case["heads"] // case["kv_heads"], case["block"]
    ctx = _contexts(case)
    out = torch.zeros((case["batch"], case["heads"], D), dtype=torch.float64, device=DEV)
    lse = torch.full((case["batch"], case["heads"]), -math.inf, dtype=torch.float64, device=DEV)
    for s, c in enumerate(ctx):
        count = min(_ceil(c, B), case["budget"])
        if count == 0:
            continue
        k, v = _read64(st["pool"][s][st["slots"][s, :count].long()], case)
        token = (st["blocks"][s, :count, None] * B + torch.arange(B, device=DEV)).flatten() < c
        k, v = (x.transpose(0, 1).flatten(1, 2)[:, token] for x in (k, v))
        q = st["q"][s].double().reshape(-1, G, D)
        z = torch.einsum("hgd,htd->hgt", q, k) / math.sqrt(D)
        lse[s] = torch.logsumexp(z, -1).flatten()
        out[s] = torch.einsum("hgt,htd->hgd", torch.softmax(z, -1), v).reshape(-1, D)
    return out, lse
