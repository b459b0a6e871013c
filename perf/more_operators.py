"""Cases of the attention over packed prompts and of the operators around the 8-bit KV cache, with their plain forms and their
64-bit definitions.

  prompt   causal attention of a packed batch of prompts or prompt chunks: sequence s has the queries q_start[s] .. q_start[s + 1] and
           the keys k_start[s] .. k_start[s + 1]; its last query sees all of its keys, each one before it a key less
  store    tokens into 8-bit blocks through a slot map, and the blocks read back as bf16
  append   one decode step's token into pool and store, with the slot taken for a block that has just been opened
  attn     one layer's sparse decode attention over a pool of 8-bit blocks

Layout of an 8-bit block: [kv head][K, V][token][128] e4m3 numbers, then [kv head][K, V] scales in fp32, the whole padded to a
multiple of 128 bytes.  A scale is a power of two that all tokens of the block share, 2^-7 of the one at or below the largest
magnitude among them (at least 2^-117); the value is scale * number.  A token that joins a block keeps the block's scale where that is
enough; where it is not, the tokens that the block holds are rounded again under the larger one.  A block whose first
token is among the new ones begins anew.
"""
import math
import random

import torch

own = False

D = 128
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
MOST = 32 * 8192 * 8192  # scores of the largest prompt


def _ceil(a, b):
    return -(-a // b)


def _block_bytes(case):
    return case["kv_heads"] * case["block"] * 256 + _ceil(case["kv_heads"] * 8, 128) * 128


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one short prompt: latency
        {"name": "prompt 77 tokens", "op": "prompt", "batch": 1, "heads": 32, "kv_heads": 8, "dtype": "bf16", "new": 77, "past": 0, "ragged": False, "pad": 0},
        # a batch of prompts of many lengths out of one fused projection, padded to a fixed capacity
        {"name": "prompt 23 ragged", "op": "prompt", "batch": 23, "heads": 32, "kv_heads": 8, "dtype": "bf16", "new": 1500, "past": 0, "ragged": True, "pad": 41},
        # a whole prompt of the 8B-shaped model
        {"name": "prompt 8192 tokens", "op": "prompt", "batch": 1, "heads": 32, "kv_heads": 8, "dtype": "bf16", "new": 8192, "past": 0, "ragged": False, "pad": 0},
        # a chunk of a long prompt of the 70B-shaped model, fp16, over the 65 536 tokens before it
        {"name": "prompt 500 after 65536", "op": "prompt", "batch": 1, "heads": 64, "kv_heads": 8, "dtype": "fp16", "new": 500, "past": 65536, "ragged": False, "pad": 0},
        # a decode step of 16 sequences whose keys lie one behind the other: a single new token each
        {"name": "prompt 16 x 1 after 16384", "op": "prompt", "batch": 16, "heads": 32, "kv_heads": 8, "dtype": "bf16", "new": 1, "past": 16384, "ragged": True, "pad": 0},
        # a prompt's tail: a ragged handful of tokens into scattered pages, the first of them partly filled
        {"name": "store 333 tokens", "op": "store", "tokens": 333, "kv_heads": 8, "block": 16, "pages": 32, "at": 5, "pad": 3},
        # a full context of the long-context workload
        {"name": "store 131072 tokens", "op": "store", "tokens": 131072, "kv_heads": 8, "block": 32, "pages": 4096, "at": 0, "pad": 0},
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
    op = rng.choice(["prompt", "prompt", "prompt", "prompt", "store", "append", "attn", "attn", "attn"])
    kv = rng.choice([1, 2, 4, 8, 8, 16])
    block = rng.choice([16, 16, 32, 64])
    if op == "prompt":
        heads = kv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 8, 16])
        batch = _log(rng, 1, 32)
        most = MOST // (batch * heads)
        new = _log(rng, 1, min(8192, math.isqrt(most)))
        past = rng.choice([0, 0, _log(rng, 1, max(1, min(131072, most // new - new, (1 << 22) // (batch * kv))))])
        return {"op": op, "batch": batch, "heads": heads, "kv_heads": kv, "dtype": rng.choice(["bf16", "bf16", "fp16"]), "new": new, "past": past,
                "ragged": rng.random() < 0.7, "pad": rng.choice([0, 0, 1, 100])}
    if op == "store":
        tokens = _log(rng, 1, 131072 * 8 // max(8, kv))
        at = rng.choice([0, rng.randrange(0, block)])
        return {"op": op, "tokens": tokens, "kv_heads": kv, "block": block, "pages": _ceil(tokens + at, block) + rng.randrange(0, 3), "at": at, "pad": rng.choice([0, tokens // 4])}
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
    """Queries and keys of every sequence (prompt): the same for every seed, so that the work is known."""
    r = random.Random(case["batch"] * 1000003 + case["new"] * 31 + case["past"])
    n = [r.randrange(1, case["new"] + 1) if case["ragged"] else case["new"] for _ in range(case["batch"])]
    p = [r.randrange(0, case["past"] + 1) if case["ragged"] else case["past"] for _ in range(case["batch"])]
    if case["ragged"] and case["batch"] > 3:
        n[1] = 0  # a request with nothing left to do
        n[2], p[2] = case["new"], case["past"]
    return n, [a + b for a, b in zip(n, p)]


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


# ------------------------------------------------------------------ the 8-bit format, plainly
def _scale_for(most):
    """Largest magnitude (fp32) -> the scale it asks for."""
    exponent = torch.where(most > 0, torch.frexp(most)[1] - 8, -117).clamp(min=-117)
    return ((exponent + 127) << 23).to(torch.int32).view(torch.float32)


def _codes(x, scale):
    """x fp32, scale fp32 -> bytes of the e4m3 numbers."""
    return (x / scale).to(torch.float8_e4m3fn).view(torch.uint8)


def _numbers(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _parts(blocks, case):
    """blocks uint8 [n, block bytes] -> codes [n][h][2][block][128], scales fp32 [n][h][2]."""
    H, B = case["kv_heads"], case["block"]
    codes = blocks[:, :H * B * 256].unflatten(1, (H, 2, B, D))
    scales = blocks[:, H * B * 256:H * B * 256 + H * 8].contiguous().view(torch.float32).unflatten(1, (H, 2))
    return codes, scales


def _packed(codes, scales, case):
    """The reverse; what pads a block is 0."""
    H, B = case["kv_heads"], case["block"]
    blocks = torch.cat((codes.flatten(1), scales.contiguous().view(torch.uint8).flatten(1)), 1)
    return torch.nn.functional.pad(blocks, (0, _block_bytes(case) - blocks.shape[1]))


def _blocks_of(kv, case):
    """bf16 numbers in fp32 [n][h][2][block][128] -> whole 8-bit blocks."""
    scale = _scale_for(kv.abs().amax((-1, -2)))
    return _packed(_codes(kv, scale[..., None, None]), scale, case)


def _values(blocks, case):
    codes, scales = _parts(blocks, case)
    return (_numbers(codes) * scales[..., None, None]).to(torch.bfloat16)


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    st = {"case": case, "pi": _handle(case) if own else None}
    i32 = dict(dtype=torch.int32, device=DEV)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    def cached(*shape):
        """Keys or values [..., 128]: four channels are eight times as large."""
        x = normal(*shape)
        x[..., [7, 40, 77, 121]] *= 8
        return x

    op = case["op"]
    if op == "prompt":
        Hq, Hk, dt = case["heads"], case["kv_heads"], DTYPES[case["dtype"]]
        n, m = _lengths(case)
        T, Tk = sum(n) + case["pad"], sum(m) + case["pad"]
        if case["past"] == 0:  # one projection: queries, keys and values of a token side by side
            x = normal(T, (Hq + 2 * Hk) * D).to(dt)
            x[:, (Hq + Hk - 1) * D + 5] *= 8
            st["q"], st["k"], st["v"] = (x[:, a * D:b * D].unflatten(1, (b - a, D)) for a, b in ((0, Hq), (Hq, Hq + Hk), (Hq + Hk, Hq + 2 * Hk)))
        else:
            st["q"] = normal(T, Hq, D).to(dt)
            st["k"], st["v"] = cached(Tk, Hk, D).to(dt), cached(Tk, Hk, D).to(dt)
        st["q_start"] = torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], **i32)
        st["k_start"] = torch.tensor([sum(m[:i]) for i in range(len(m) + 1)], **i32)
        st["n"], st["m"] = max(n), max(m)
        st["out"] = torch.zeros((T, Hq, D), dtype=dt, device=DEV)
        st["lse"] = torch.zeros((T, Hq), dtype=torch.float32, device=DEV)
    elif op == "store":
        T, H, B = case["tokens"], case["kv_heads"], case["block"]
        kv = cached(T, 2 * H, D).to(torch.bfloat16)
        st["k"], st["v"] = kv[:, :H], kv[:, H:]
        page = torch.randperm(case["pages"], generator=g, device=DEV)
        t = torch.arange(T, device=DEV) + case["at"]
        st["slots"] = page[t // B] * B + t % B
        if case["pad"]:
            st["slots"][T - case["pad"]:] = -1
        st["store"] = torch.zeros((case["pages"], _block_bytes(case)), dtype=torch.uint8, device=DEV)
        if case["at"]:  # what the first page holds already, smaller by half or so than what comes
            st["store"][page[0]] = _blocks_of((0.5 * cached(1, H, 2, B, D)).to(torch.bfloat16).float(), case)[0]
        st["out"] = torch.zeros((case["pages"], H, 2, B, D), dtype=torch.bfloat16, device=DEV)
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
        st["k"], st["v"] = cached(n, H, D).to(torch.bfloat16), cached(n, H, D).to(torch.bfloat16)
        st["digest"] = torch.stack((normal(n, NB, D) - 2, normal(n, NB, D) + 2), 2).to(torch.bfloat16)
        # the block that is being filled already holds rows; the others are not looked at
        st["pool"] = torch.zeros((n, C, _block_bytes(case)), dtype=torch.uint8, device=DEV)
        st["store"] = torch.zeros((n, NB, _block_bytes(case)), dtype=torch.uint8, device=DEV)
        st["store_ids"] = (torch.arange(n, **i32) * NB + cur).contiguous()
        first = torch.arange(n, **i32) * C
        st["first"], st["cur"] = first, cur[:, None].long().contiguous()
        held = st["table"].gather(1, st["cur"])[:, 0]
        filled = torch.arange(B, device=DEV)[None] < (ctx % B)[:, None]
        some = _blocks_of(torch.where(filled[:, None, None, :, None], cached(n, H, 2, B, D), 0.0).to(torch.bfloat16).float(), case)
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
            st["pool"][s] = _blocks_of(cached(C, H, 2, B, D).to(torch.bfloat16).float(), case)
        st["out"] = torch.zeros((n, case["heads"], D), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.zeros((n, case["heads"]), dtype=torch.float32, device=DEV)
    return st


# ------------------------------------------------------------------ one pass
def run(st):
    case, pi, op = st["case"], st["pi"], st["case"]["op"]
    if own:
        if op == "prompt":
            pi.prompt_attn(st["q"], st["k"], st["v"], st["q_start"], st["out"], k_start=st["k_start"], lse=st["lse"])
            return st["out"], st["lse"]
        if op == "store":
            pi.kv8_store(st["k"], st["v"], st["store"], st["slots"])
            pi.kv8_load(st["store"], st["out"])
            return st["out"]
        if op == "append":
            pi.append_kv8(0, st["step"], st["k"], st["v"], st["ctx"], st["store"], st["pool"], st["table"], st["slot_block"], st["stamp"], st["digest"])
            ids = st["table"].gather(1, st["cur"])[:, 0] + st["first"]
            pi.kv8_load(st["pool"], st["pool_out"], ids)
            pi.kv8_load(st["store"], st["store_out"], st["store_ids"])
            return st["table"], st["slot_block"], st["stamp"], st["digest"], st["pool_out"], st["store_out"]
        pi.sparse_decode_attn_kv8(0, st["q"], st["pool"], st["slots"], st["blocks"], st["count"], st["ctx"], st["out"], st["lse"])
        return st["out"], st["lse"]
    return {"prompt": _plain_prompt, "store": _plain_store, "append": _plain_append, "attn": _plain_attn}[op](st)


def _softmax_of(s):
    """In place: scores, -inf where masked -> weights, their sums (0 where nothing is seen) and their log-sum-exp."""
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    return p, torch.where(l > 0, l, 1.0), m + torch.log(l)


def _plain_prompt(st):
    """The sequences side by side, padded to the longest."""
    case, H = st["case"], st["case"]["kv_heads"]
    q0, k0 = st["q_start"].long(), st["k_start"].long()
    i, j = torch.arange(st["n"], device=DEV), torch.arange(st["m"], device=DEV)
    n, m = q0.diff()[:, None], k0.diff()[:, None]
    qi, kj = (q0[:-1, None] + i).clamp(max=st["q"].shape[0] - 1), (k0[:-1, None] + j).clamp(max=st["k"].shape[0] - 1)
    q = st["q"][qi].float().unflatten(2, (H, -1)).permute(0, 2, 3, 1, 4)  # [batch][h][g][i][128]
    k, v = (torch.where((j < m)[..., None, None], x[kj], 0).float().transpose(1, 2)[:, :, None] for x in (st["k"], st["v"]))
    s = (q @ k.transpose(-1, -2)).mul_(1 / math.sqrt(D))
    s.masked_fill_(~((j <= i[:, None] + (m - n)[..., None]) & (j < m)[:, None])[:, None, None], -math.inf)
    p, l, lse = _softmax_of(s)
    o = (p @ v) / l
    real = i < n
    st["out"][qi[real]] = o.permute(0, 3, 1, 2, 4).flatten(2, 3)[real].to(st["out"].dtype)
    st["lse"][qi[real]] = lse[..., 0].permute(0, 3, 1, 2).flatten(2, 3)[real]
    return st["out"], st["lse"]


def _plain_store(st):
    case, B = st["case"], st["case"]["block"]
    real = st["slots"] >= 0
    page, at = torch.where(real, st["slots"] // B, case["pages"]), torch.where(real, st["slots"] % B, 0)  # one page more, for what is not stored
    x = torch.stack((st["k"], st["v"]), 2).float()  # [T][h][2][128]
    codes, scales = _parts(torch.nn.functional.pad(st["store"], (0, 0, 0, 1)), case)
    begins = torch.zeros(case["pages"] + 1, dtype=torch.bool, device=DEV).index_put((page[(at == 0) & real],), torch.ones((), dtype=torch.bool, device=DEV))
    most = torch.zeros_like(scales).scatter_reduce(0, page[:, None, None].expand(x.shape[:3]), x.abs().amax(-1), "amax")
    touched = torch.zeros(case["pages"] + 1, dtype=torch.bool, device=DEV).index_put((page,), torch.ones((), dtype=torch.bool, device=DEV))
    need = _scale_for(most)
    scale = torch.where(begins[:, None, None], need, torch.where(touched[:, None, None], torch.maximum(scales, need), scales))
    held = torch.where(begins[:, None, None, None, None], 0.0, _numbers(codes) * scales[..., None, None])
    codes = _codes(held, torch.where(scale > 0, scale, 1.0)[..., None, None])
    codes[page, :, :, at] = _codes(x, scale[page][..., None])
    st["store"].copy_(_packed(codes, scale, case)[:-1])
    return _values(st["store"], case)


def _plain_append(st):
    case, n, B, C = st["case"], st["case"]["batch"], st["case"]["block"], st["case"]["slots"]
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
    x = torch.stack((st["k"], st["v"]), 2).float()  # [n][h][2][128]
    need = _scale_for(x.abs().amax(-1))
    here = (torch.arange(B, device=DEV) == t[:, None])[:, None, None, :, None]
    opened = (t == 0)[:, None, None]

    def write(buffer, ids):
        codes, scales = _parts(buffer.flatten(0, 1)[ids], case)
        scale = torch.where(opened, need, torch.maximum(scales, need))
        held = torch.where(opened[..., None, None], 0.0, _numbers(codes) * scales[..., None, None])
        blocks = _packed(_codes(torch.where(here, x[:, :, :, None], held), scale[..., None, None]), scale, case)
        buffer.flatten(0, 1).index_copy_(0, ids, blocks)
        return _values(blocks, case)

    pool, store = write(st["pool"], st["first"].long() + slot), write(st["store"], st["store_ids"].long())
    d = st["digest"].flatten(0, 1)[st["store_ids"].long()]
    k = st["k"][:, 0]
    new = torch.where(opened, torch.stack((k, k), 1), torch.stack((torch.minimum(d[:, 0], k), torch.maximum(d[:, 1], k)), 1))
    st["digest"].flatten(0, 1).index_copy_(0, st["store_ids"].long(), new)
    return st["table"], sb, st["stamp"], st["digest"], pool, store


def _plain_attn(st):
    case, n, H, B, K = st["case"], st["case"]["batch"], st["case"]["kv_heads"], st["case"]["block"], st["case"]["budget"]
    slots = st["slots"].clamp(min=0).long() + torch.arange(n, device=DEV)[:, None] * case["slots"]
    codes, scales = _parts(st["pool"].flatten(0, 1)[slots].flatten(0, 1), case)
    kv = (_numbers(codes) * scales[..., None, None]).unflatten(0, (n, K)).transpose(1, 2)  # [n][h][K][2][B][128]
    k, v = kv[:, :, :, 0].flatten(2, 3), kv[:, :, :, 1].flatten(2, 3)
    q = st["q"].float().unflatten(1, (H, case["heads"] // H))
    s = (q @ k.transpose(-1, -2)) / math.sqrt(D)
    token = st["blocks"][:, :, None] * B + torch.arange(B, device=DEV)
    seen = (st["blocks"] >= 0)[:, :, None] & (token < st["ctx"][:, None, None]) & (torch.arange(K, device=DEV)[:, None] < st["count"][:, None, None])
    seen = seen.flatten(1)[:, None, None]
    p, l, lse = _softmax_of(s.masked_fill_(~seen, -math.inf))
    o = p @ torch.where(seen.transpose(-1, -2), v, 0.0) / l
    return o.flatten(1, 2).to(torch.bfloat16), lse[..., 0].flatten(1)


# ------------------------------------------------------------------ work of a pass
def work(case):
    op = case["op"]
    if op == "prompt":
        n, m = _lengths(case)
        pairs = sum(a * b - a * (a - 1) // 2 for a, b in zip(n, m))  # the i-th last query sees i keys less
        return {"bytes": sum(n) * case["heads"] * (4 * D + 4) + sum(b for a, b in zip(n, m) if a) * case["kv_heads"] * 4 * D + case["batch"] * 8, "flops": 4 * D * case["heads"] * pairs}
    if op == "store":
        rows = (case["tokens"] - case["pad"]) * case["kv_heads"]
        held = case["pages"] * case["block"] * case["kv_heads"]
        return {"bytes": rows * (512 + 256) + case["tokens"] * 8 + held * (256 + 512) + case["pages"] * case["kv_heads"] * 16, "flops": (rows + held) * 256 * 3}
    if op == "append":
        B, H = case["block"], case["kv_heads"]
        # new rows in, pool and store rows out, the digest, a scan of the slots' blocks and stamps; the block read back twice
        return {"bytes": case["batch"] * (H * (512 + 2 * 256 + 4 * 8) + 1024 + case["slots"] * 8 + 2 * B * H * (256 + 512)), "flops": case["batch"] * H * B * 256 * 4}
    tokens = sum(min(c, case["budget"] * case["block"]) for c in _contexts(case))
    blocks = sum(min(_ceil(c, case["block"]), case["budget"]) for c in _contexts(case))
    return {"bytes": tokens * case["kv_heads"] * 256 + blocks * (case["kv_heads"] * 8 + 8) + case["batch"] * case["heads"] * (D * 4 + 4), "flops": 4 * tokens * case["heads"] * D}


# ------------------------------------------------------------------ the definitions in 64 bits
def _power64(e):
    """2^e of whole numbers, exactly."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _round64(x, unit):
    """Multiples of `unit` times what three bits after the leading one hold, and of 2^-9 below 2^-6: the e4m3 numbers, in 64 bits."""
    y = x / unit
    e = ((y.view(torch.int64) >> 52) & 2047) - 1023  # floor(log2 |y|)
    step = _power64(e.clamp(min=-6) - 3)
    return torch.round(y / step) * step * unit


def _unit64(x):
    """The scale that magnitudes [...] ask for."""
    return _power64(((x.clamp(min=2.0 ** -110).view(torch.int64) >> 52) & 2047) - 1030)


def _read64(blocks, case):
    """Blocks [n][bytes] -> values [n][h][2][block][128] and scales [n][h][2] in 64 bits, byte by byte."""
    H, B = case["kv_heads"], case["block"]
    b = blocks[:, :H * B * 256].reshape(-1, H, 2, B, D).to(torch.int32)
    e, f = ((b >> 3) & 15).double(), (b & 7).double()
    size = torch.where(e > 0, (8 + f) * _power64(e - 10), f * 2.0 ** -9)
    scale = blocks[:, H * B * 256:H * B * 256 + 8 * H].reshape(-1, 4).to(torch.int64)
    exponent = ((scale[:, 3] << 1) + (scale[:, 2] >> 7)).reshape(-1, H, 2)
    scale = torch.where(exponent > 0, _power64(exponent - 127), 0.0)
    return torch.where(b < 128, size, -size) * scale[..., None, None], scale


def exact(case, seed):
    op = case["op"]
    global own
    kept, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = kept
    if op == "prompt":
        G = case["heads"] // case["kv_heads"]
        out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
        lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device=DEV)
        a = b = 0
        for n, m in zip(*_lengths(case)):
            for h in range(case["kv_heads"] if n else 0):
                k, v = st["k"][b:b + m, h].double(), st["v"][b:b + m, h].double()
                last = torch.arange(m - n, m, device=DEV)
                for head in range(h * G, h * G + G):
                    z = st["q"][a:a + n, head].double() @ k.T / math.sqrt(D)
                    z[last[:, None] < torch.arange(m, device=DEV)] = -math.inf
                    lse[a:a + n, head] = torch.logsumexp(z, -1)
                    out[a:a + n, head] = torch.softmax(z, -1) @ v
            a, b = a + n, b + m
        return out, lse
    if op == "store":
        B = case["block"]
        held, unit = _read64(st["store"], case)
        real = st["slots"] >= 0
        p, r = st["slots"][real] // B, st["slots"][real] % B
        new = torch.stack((st["k"][real], st["v"][real]), 2).double()
        asked = _unit64(new.abs().amax(-1))
        ask = torch.zeros_like(unit).scatter_reduce(0, p[:, None, None].expand(asked.shape), asked, "amax")
        fresh = torch.zeros(case["pages"], dtype=torch.bool, device=DEV)
        fresh[p[r == 0]] = True
        unit = torch.where(fresh[:, None, None], ask, torch.maximum(unit, ask))
        held[fresh] = 0
        held[p, :, :, r] = new
        return _round64(held, torch.where(unit > 0, unit, 1.0)[..., None, None])
    if op == "append":
        ctx, B = _contexts(case), case["block"]
        held, unit = _read64(st["store"].flatten(0, 1)[st["store_ids"].long()], case)
        digest = st["digest"].double()
        for s, c in enumerate(ctx):
            b, t = divmod(c, B)
            new = torch.stack((st["k"][s], st["v"][s]), 1).double()
            ask = _unit64(new.abs().amax(-1))
            if t == 0:
                held[s], unit[s] = 0, 0
            unit[s] = torch.maximum(unit[s], ask)
            held[s, :, :, t] = new
            x = st["k"][s, 0].double()
            digest[s, b, 0] = x if t == 0 else torch.minimum(digest[s, b, 0], x)
            digest[s, b, 1] = x if t == 0 else torch.maximum(digest[s, b, 1], x)
        both = _round64(held, unit[..., None, None])
        return None, None, None, digest, both, both
    G, B = case["heads"] // case["kv_heads"], case["block"]
    out = torch.zeros((case["batch"], case["heads"], D), dtype=torch.float64, device=DEV)
    lse = torch.full((case["batch"], case["heads"]), -math.inf, dtype=torch.float64, device=DEV)
    for s, c in enumerate(_contexts(case)):
        count = min(_ceil(c, B), case["budget"])
        if count == 0:
            continue
        kv, _ = _read64(st["pool"][s][st["slots"][s, :count].long()], case)
        token = (st["blocks"][s, :count, None] * B + torch.arange(B, device=DEV)).flatten() < c
        k, v = (kv[:, :, i].transpose(0, 1).flatten(1, 2)[:, token] for i in (0, 1))
        q = st["q"][s].double().reshape(-1, G, D)
        z = torch.einsum("hgd,htd->hgt", q, k) / math.sqrt(D)
        lse[s] = torch.logsumexp(z, -1).flatten()
        out[s] = torch.einsum("hgt,htd->hgd", torch.softmax(z, -1), v).reshape(-1, D)
    return out, lse
