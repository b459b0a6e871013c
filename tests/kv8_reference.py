"""The 8-bit cache in numpy, from its definition: e4m3 numbers by table, scales as exponents, sums in 64 bits."""
import numpy as np

from tests.kv4_reference import bf16  # noqa: F401  (rounds to bf16 numbers in float32)

D = 128
LEAST = -117                                              # exponent of the smallest scale


def _table():
    """The e4m3 number of every byte."""
    out = np.empty(256)
    for b in range(256):
        e, f = (b >> 3) & 15, b & 7
        x = f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
        out[b] = np.nan if b & 127 == 127 else -x if b & 128 else x
    return out


TABLE = _table()
SIZES = TABLE[:127]                                       # ascending, 0 .. 448


def round_numbers(x):
    """float64 (|x| <= 448, or not a number) -> bytes: the nearest number, of two equally near the even one."""
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(SIZES, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    below, above = a - SIZES[lo], SIZES[hi] - a
    code = np.where(below < above, lo, np.where(below > above, hi, np.where(lo % 2 == 0, lo, hi))).astype(np.uint8)
    code = np.where(a == SIZES[hi], hi, code).astype(np.uint8)
    code = code | np.where(np.signbit(x), 128, 0).astype(np.uint8)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8)


def block_bytes(heads: int, block: int) -> int:
    return heads * block * 256 + -(-heads * 8 // 128) * 128


def _exponent(values) -> int:
    a = np.abs(values[np.isfinite(values)])
    return max(int(np.frexp(a.max())[1]) - 8, LEAST) if a.size and a.max() > 0 else LEAST


def parts(block, heads: int, B: int):
    """One block's bytes -> views: codes [heads][2][B][128], scales float32 [heads][2]."""
    n = heads * B * 256
    return block[:n].reshape(heads, 2, B, D), block[n:n + heads * 8].view(np.float32).reshape(heads, 2)


def store(blocks, k, v, slots, B: int) -> None:
    """blocks uint8 [n][bytes]; k, v float32 [T][heads][128] (bf16 numbers); tokens of one block stand together."""
    heads = k.shape[1]
    todo = {}
    for t, s in enumerate(slots):
        if 0 <= s < len(blocks) * B:
            todo.setdefault(int(s) // B, []).append((t, int(s) % B))
    for b, tokens in todo.items():
        codes, scales = parts(blocks[b], heads, B)
        fresh = any(r == 0 for _, r in tokens)
        for h in range(heads):
            for i, x in ((0, k), (1, v)):
                rows = np.stack([x[t, h] for t, _ in tokens]).astype(np.float64)
                e = _exponent(rows)
                if fresh:
                    codes[h, i] = 0
                    scales[h, i] = 2.0 ** e
                elif 2.0 ** e > scales[h, i]:
                    old = TABLE[codes[h, i]] * np.float64(scales[h, i])
                    nan = np.isnan(old)
                    signs = codes[h, i] & 128
                    codes[h, i] = np.where(nan, codes[h, i], round_numbers(np.where(nan, 0, old / 2.0 ** e)) & 127 | signs)
                    scales[h, i] = 2.0 ** e
                for (_, r), row in zip(tokens, rows):
                    codes[h, i, r] = round_numbers(row / np.float64(scales[h, i]))


def write_token(blocks, slot: int, k, v, B: int) -> None:
    store(blocks, k[None], v[None], [slot], B)


def pack(kv, B: int):
    """kv float32 [n][heads][2][B][128] (bf16 numbers) -> uint8 [n][bytes]."""
    n, H = kv.shape[:2]
    x = kv.astype(np.float64)
    a = np.abs(np.where(np.isfinite(x), x, 0.0)).max((-1, -2))
    e = np.where(a > 0, np.maximum(np.frexp(a)[1] - 8, LEAST), LEAST)
    unit = np.ldexp(1.0, e)
    out = np.zeros((n, block_bytes(H, B)), dtype=np.uint8)
    out[:, :H * B * 256] = round_numbers(x / unit[..., None, None]).reshape(n, -1)
    out[:, H * B * 256:H * B * 256 + 8 * H] = unit.astype(np.float32).reshape(n, -1).view(np.uint8)
    return out


def unpack(blocks, heads: int, B: int):
    """uint8 [n][bytes] -> float64 [n][heads][2][B][128]."""
    n = blocks.shape[0]
    codes = blocks[:, :heads * B * 256].reshape(n, heads, 2, B, D)
    scales = np.ascontiguousarray(blocks[:, heads * B * 256:heads * B * 256 + 8 * heads]).view(np.float32).reshape(n, heads, 2)
    return TABLE[codes] * scales.astype(np.float64)[..., None, None]


def attention(q, kv_of, sel_blocks, sel_slots, count: int, ctx: int, B: int):
    """One sequence.  q float64 [Hq][128]; kv_of(slot) -> float64 [heads][2][B][128].  out [Hq][128], lse [Hq], and what they may be off by:

    scores: eight products of 16 channels run through a 32-bit accumulator, off by at most 2^-23 of the sum of magnitudes each (and as much
    for an accumulator that cuts off), and four roundings of 2^-24: eps.  Weights: 2 eps, the exponential's 2^-22, and
    one rounding to fp16, 2^-11 of itself, or 2^-24 of the largest weight times its block's largest value."""
    Hq = q.shape[0]
    out, lse, tol, eps = np.zeros((Hq, D)), np.full(Hq, -np.inf), np.zeros((Hq, D)), np.zeros(Hq)
    ks, vs, tops = [], [], []
    for j in range(count):
        b, s = int(sel_blocks[j]), int(sel_slots[j])
        n = min(B, ctx - b * B)
        if b < 0 or n <= 0:
            continue
        kv = kv_of(s)
        ks.append(kv[:, 0, :n]); vs.append(kv[:, 1, :n])
        whole = np.where(np.isfinite(kv[:, 1]), np.abs(kv[:, 1]), 0.0).max((1, 2))
        tops.append(np.repeat(whole[:, None], n, 1))
    if not ks:
        return out, lse, tol, eps
    k, v, top = np.concatenate(ks, 1), np.concatenate(vs, 1), np.concatenate(tops, 1)
    G = Hq // k.shape[0]
    for g in range(Hq):
        h = g // G
        z = k[h] @ q[g] / np.sqrt(D)
        m = z.max()
        p = np.exp(z - m)
        w = p / p.sum()
        out[g] = w @ v[h]
        lse[g] = m + np.log(p.sum())
        eps[g] = (8 * 2.0 ** -23 * (np.abs(k[h]) @ np.abs(q[g])).max() + 4 * 2.0 ** -24 * np.abs(k[h] @ q[g]).max()) / np.sqrt(D)
        spread = w @ np.abs(v[h])
        tol[g] = 2.0 ** -8 * np.abs(out[g]) + (2 * eps[g] + 2.0 ** -11 + 2.0 ** -20) * spread + len(w) * 2.0 ** -24 * (w * top[h]).max()
    return out, lse, tol + 1e-35, eps


class Appender:
    """The append on one sequence after the other (see pi_append_kv), the rows in 8 bits."""

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
                free = [(int(self.stamp[s, i]), i) for i in range(self.slot_block.shape[1])
                        if not (self.slot_block[s, i] >= 0 and (self.slot_block[s, i] < c.n_sink_blocks or self.slot_block[s, i] >= b + 1 - c.n_local_blocks))]
                slot = min(free)[1]
                if self.slot_block[s, slot] >= 0:
                    self.table[s, self.slot_block[s, slot]] = -1
                self.table[s, b], self.slot_block[s, slot] = slot, b
            rows, at = (self.store[s], b) if page_table is None else (self.store, int(page_table[s, b]))
            if t == 0:
                self.pool[s, slot] = 0
                rows[at] = 0
            write_token(self.pool[s], slot * B + t, k[s], v[s], B)
            write_token(rows, at * B + t, k[s], v[s], B)
            self.stamp[s, slot] = step
            x, d = k[s, self.h], self.digest[s, b]
            if t == 0:
                d[0], d[1] = x, x
            else:
                d[0], d[1] = np.where(x < d[0], x, d[0]), np.where(x > d[1], x, d[1])
