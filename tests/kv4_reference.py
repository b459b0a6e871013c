"""Plain references of the 4-bit cache and the calls around it: numpy on the CPU, written from the definitions in
include/pulseinfer.h, in 64 bits where the kernels round."""
import numpy as np

D = 128
TILE = 2560


def bf16(x):
    """Nearest bf16 of float32 values (ties to even), as float32; NaN and infinities keep."""
    x = np.asarray(x, dtype=np.float32)
    u = x.view(np.uint32)
    r = ((u.astype(np.uint64) + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint32) << 16
    return np.where(np.isfinite(x), r.view(np.float32), x).astype(np.float32)


def block_bytes(n_kv_heads: int, block_tokens: int) -> int:
    return -(-n_kv_heads * block_tokens * 160 // 4096) * 4096


def round_rows(x):
    """x float32 [..., 128] holding bf16 numbers -> codes uint8 [..., 128], scale and minimum float32 [..., 4]."""
    g = np.asarray(x, dtype=np.float32).reshape(x.shape[:-1] + (4, 32))
    with np.errstate(all="ignore"):
        lo, hi = g.min(-1), g.max(-1)                                   # numpy's min and max hand NaN on
        s = bf16((hi - lo) / np.float32(15))
        q = np.rint((g - lo[..., None]) / s[..., None])
        q = np.where(np.isnan(q), 0, np.clip(q, 0, 15))
        q = np.where(s[..., None] > 0, q, 0)
    return q.reshape(x.shape).astype(np.uint8), s, lo


def values(codes, s, lo):
    """What codes, scale and minimum stand for, in 64 bits."""
    with np.errstate(all="ignore"):
        g = codes.reshape(codes.shape[:-1] + (4, 32)).astype(np.float64)
        return (s[..., None].astype(np.float64) * g + lo[..., None].astype(np.float64)).reshape(codes.shape)


def k_place(d: int):
    """(byte in a K row, shift) of channel d."""
    j, c, i = d // 32, d % 32 // 8, d % 8
    return 16 * c + 4 * j + i // 2, 4 * (i % 2)


def v_place(d: int):
    j, r, i = d // 32, d % 32 // 4, d % 4
    return 8 * r + 2 * j + i // 2, 4 * (i % 2)


def _codes_to_bytes(codes, place):
    out = np.zeros(codes.shape[:-1] + (64,), dtype=np.uint8)
    for d in range(D):
        b, sh = place(d)
        out[..., b] |= codes[..., d] << sh
    return out


def _bytes_to_codes(row, place):
    return np.stack([(row[..., place(d)[0]] >> place(d)[1]) & 15 for d in range(D)], -1)


def _pair_bytes(s, lo):
    both = np.stack((s, lo), -1).astype(np.float32)                      # [..., 4, 2], bf16 numbers
    half = (both.view(np.uint32) >> 16).astype(np.uint16)
    return half.reshape(half.shape[:-2] + (8,)).view(np.uint8)


def write_token(blocks, slot: int, k, v, block_tokens: int) -> None:
    """blocks uint8 [n][bytes]; k, v float32 [Hkv][128] (bf16 numbers) into token `slot`."""
    b, t = divmod(slot, block_tokens)
    per_head = block_tokens // 16 * TILE
    for h in range(k.shape[0]):
        tile = blocks[b, h * per_head + t // 16 * TILE:][:TILE]
        r = t % 16
        for x, place, codes_at, scales_at in ((k[h], k_place, 0, 2048), (v[h], v_place, 1024, 2304)):
            c, s, lo = round_rows(x)
            tile[codes_at + 64 * r:codes_at + 64 * r + 64] = _codes_to_bytes(c, place)
            tile[scales_at + 16 * r:scales_at + 16 * r + 16] = _pair_bytes(s, lo)


def pack(kv, block_tokens: int):
    """kv float32 [n][Hkv][2][B][128] (bf16 numbers) -> uint8 [n][bytes]."""
    n, H = kv.shape[:2]
    parts = []
    for i, place in ((0, k_place), (1, v_place)):
        c, s, lo = round_rows(kv[:, :, i])
        parts.append((_codes_to_bytes(c, place), _pair_bytes(s, lo)))
    tiles = block_tokens // 16
    cut = lambda a: a.reshape(n, H, tiles, -1)                           # noqa: E731
    body = np.concatenate((cut(parts[0][0]), cut(parts[1][0]), cut(parts[0][1]), cut(parts[1][1])), -1).reshape(n, -1)
    return np.pad(body, ((0, 0), (0, block_bytes(H, block_tokens) - body.shape[1])))


def unpack(blocks, n_kv_heads: int, block_tokens: int):
    """uint8 [n][bytes] -> float64 [n][Hkv][2][B][128]."""
    n, H, B = blocks.shape[0], n_kv_heads, block_tokens
    t = blocks[:, :H * B * 160].reshape(n, H, B // 16, TILE)
    out = np.empty((n, H, 2, B, D))
    for i, (place, codes_at, scales_at) in enumerate(((k_place, 0, 2048), (v_place, 1024, 2304))):
        codes = _bytes_to_codes(t[..., codes_at:codes_at + 1024].reshape(n, H, B, 64), place)
        half = np.ascontiguousarray(t[..., scales_at:scales_at + 256]).view(np.uint16).reshape(n, H, B, 4, 2)
        f = (half.astype(np.uint32) << 16).view(np.float32)
        out[:, :, i] = values(codes, f[..., 0], f[..., 1])
    return out


def attention(q, kv_of, sel_blocks, sel_slots, count: int, ctx: int, block_tokens: int):
    """One sequence.  q float64 [Hq][128]; kv_of(slot) -> float64 [Hkv][2][B][128]; returns out [Hq][128], lse [Hq], the
    largest |v| per KV head, and a bound of the scores' rounding (natural-log units) per query head: the 32 products of a
    group run through a 32-bit accumulator, off by at most 32 roundings of 2^-23 of the sum of their magnitudes (an
    accumulator that cuts off instead of rounding is off by 2^-23); a code counts up to 128 + 15 there."""
    Hq = q.shape[0]
    out, lse, vmax, eps = np.zeros((Hq, D)), np.full(Hq, -np.inf), None, np.zeros(Hq)
    ks, vs = [], []
    for j in range(count):
        b, s = int(sel_blocks[j]), int(sel_slots[j])
        n = min(block_tokens, ctx - b * block_tokens)
        if b < 0 or n <= 0:
            continue
        kv = kv_of(s)
        ks.append(kv[:, 0, :n]); vs.append(kv[:, 1, :n])
    if not ks:
        return out, lse, np.zeros(1), eps
    k, v = np.concatenate(ks, 1), np.concatenate(vs, 1)
    H = k.shape[0]
    G = Hq // H
    vmax = np.abs(v).max((1, 2))
    for g in range(Hq):
        z = k[g // G] @ q[g] / np.sqrt(D)
        m = z.max()
        p = np.exp(z - m)
        out[g] = p @ v[g // G] / p.sum()
        lse[g] = m + np.log(p.sum())
        spread = np.abs(k[g // G]).max(0).reshape(4, 32).max(1)        # at least half of scale * 15 in each group, or the minimum
        eps[g] = 32 * 2.0 ** -23 * (np.abs(q[g]).reshape(4, 32).sum(1) * spread * (2 * 143 / 15 + 1)).sum() / np.sqrt(D)
    return out, lse, vmax, eps


def rope(x, positions, inv_freq, weight, eps: float, interleaved: bool):
    """x float64 [T][H][128] -> float64; inv_freq float32 [rot / 2] or None."""
    x = x.copy()
    if weight is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * weight.astype(np.float64)
    if inv_freq is None or len(inv_freq) == 0:
        return x
    half = len(inv_freq)
    a = positions[:, None, None].astype(np.float64) * inv_freq.astype(np.float64)
    c, s = np.cos(a), np.sin(a)
    i = np.arange(half)
    p, r = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    u, v = x[..., p].copy(), x[..., r].copy()
    x[..., p], x[..., r] = u * c - v * s, v * c + u * s
    return x


class Pages:
    """The free ring and the tables, one step at a time."""

    def __init__(self, table, ring, state, block_tokens: int):
        self.table, self.ring, self.state, self.B = table.copy(), ring.copy(), list(state), block_tokens

    def step(self, old, new):
        """(slots, positions, starts) of the new tokens."""
        B, n = self.B, len(self.ring)
        taken, freed, slots, positions, starts = [], [], [], [], [0]
        head, tail = self.state[0], self.state[1]
        for s, (o, w) in enumerate(zip(old, new)):
            ob, nb = -(-o // B), -(-w // B)
            for j in range(ob, nb):
                taken.append((s, j))
            for j in range(nb, ob):
                freed.append((s, j))
        ring = self.ring.copy()
        for i, (s, j) in enumerate(taken):
            self.table[s, j] = self.ring[(head + i) % n]
        for i, (s, j) in enumerate(freed):
            ring[(tail + i) % n] = self.table[s, j]
            self.table[s, j] = -1
        self.ring = ring
        self.state[0] += len(taken)
        self.state[1] += len(freed)
        for s, (o, w) in enumerate(zip(old, new)):
            for p in range(o, w):
                slots.append(int(self.table[s, p // B]) * B + p % B)
                positions.append(p)
            starts.append(len(slots))
        return np.asarray(slots, dtype=np.int64), np.asarray(positions, dtype=np.int32), np.asarray(starts, dtype=np.int32)


class Appender:
    """The append on one sequence after the other (see pi_append_kv), the rows in 4 bits."""

    def __init__(self, table, slot_block, stamp, digest, pool, store, cfg, h_star: int):
        self.table, self.slot_block, self.stamp = table.copy(), slot_block.copy(), stamp.copy()
        self.digest, self.pool, self.store = digest.copy(), pool.copy(), store.copy()
        self.cfg, self.h = cfg, h_star

    def step(self, ctx, k, v, step: int, page_table=None):
        c = self.cfg
        B = c.block_tokens
        for s in range(len(ctx)):
            b, t = divmod(int(ctx[s]), B)
            slot = int(self.table[s, b])
            if t == 0 and slot < 0:
                best = None
                for i in range(self.slot_block.shape[1]):
                    ob = int(self.slot_block[s, i])
                    if ob >= 0 and (ob < c.n_sink_blocks or ob >= b + 1 - c.n_local_blocks):
                        continue
                    if best is None or (int(self.stamp[s, i]), i) < best:
                        best = (int(self.stamp[s, i]), i)
                slot = best[1]
                old = int(self.slot_block[s, slot])
                if old >= 0:
                    self.table[s, old] = -1
                self.table[s, b], self.slot_block[s, slot] = slot, b
            where = b if page_table is None else None
            rows = self.store[s] if page_table is None else self.store
            at = where if page_table is None else int(page_table[s, b])
            if t == 0:
                self.pool[s, slot] = 0
                rows[at] = 0
            write_token(self.pool[s], slot * B + t, k[s], v[s], B)
            write_token(rows, at * B + t, k[s], v[s], B)
            self.stamp[s, slot] = step
            x = k[s, self.h]
            if t == 0:
                self.digest[s, b, 0], self.digest[s, b, 1] = x, x
            else:
                self.digest[s, b, 0] = np.where(x < self.digest[s, b, 0], x, self.digest[s, b, 0])
                self.digest[s, b, 1] = np.where(x > self.digest[s, b, 1], x, self.digest[s, b, 1])
