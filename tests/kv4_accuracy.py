"""How near an attention over 4-bit blocks has to come to 64 bits as a whole: not value by value, where a bound has to allow for
the worst of every rounding, but in the mean square over an output, where the roundings of many weights do not add up."""
import numpy as np

from tests import kv4_reference as ref

D = 128


def parts(blocks, n_kv_heads: int, block_tokens: int):
    """uint8 [n][bytes] -> codes float64 [n][Hkv][2][B][128], scales and minima float64 [n][Hkv][2][B][4]."""
    n, H, B = blocks.shape[0], n_kv_heads, block_tokens
    t = blocks[:, :H * B * 160].reshape(n, H, B // 16, ref.TILE)
    codes, s, lo = np.empty((n, H, 2, B, D)), np.empty((n, H, 2, B, 4)), np.empty((n, H, 2, B, 4))
    for i, (place, codes_at, scales_at) in enumerate(((ref.k_place, 0, 2048), (ref.v_place, 1024, 2304))):
        codes[:, :, i] = ref._bytes_to_codes(t[..., codes_at:codes_at + 1024].reshape(n, H, B, 64), place)
        half = np.ascontiguousarray(t[..., scales_at:scales_at + 256]).view(np.uint16).reshape(n, H, B, 4, 2)
        f = (half.astype(np.uint32) << 16).view(np.float32)
        s[:, :, i], lo[:, :, i] = f[..., 0], f[..., 1]
    return codes, s, lo


def tokens(pool, slots, blocks, count: int, ctx: int, n_kv_heads: int, block_tokens: int):
    """Codes, scales and minima [Hkv][2][tokens][...] of one sequence's listed tokens; pool uint8 [C][bytes]."""
    take = [(int(slots[j]), min(block_tokens, ctx - int(blocks[j]) * block_tokens)) for j in range(count) if blocks[j] >= 0]
    take = [(s, n) for s, n in take if n > 0]
    c, s, lo = parts(pool[[s for s, _ in take]], n_kv_heads, block_tokens)
    return [np.concatenate([x[i, :, :, :n] for i, (_, n) in enumerate(take)], 2) for x in (c, s, lo)]


def softmax(q, codes, s, lo):
    """q float64 [G][128] of one KV head, K's codes, scales, minima -> weights [G][tokens] that sum to 1, lse [G]."""
    k = codes * np.repeat(s, 32, -1) + np.repeat(lo, 32, -1)
    z = q @ k.T / np.sqrt(D)
    m = z.max(1, keepdims=True)
    p = np.exp(z - m)
    return p / p.sum(1, keepdims=True), (m + np.log(p.sum(1, keepdims=True)))[:, 0]


def allowed(p, codes, s, lo):
    """Weights [G][tokens] and V of one KV head -> result [G][128] in 64 bits and the mean square [G][128] that an output may be
    off by before its last rounding: weight times scale has 11 bits, an error of 2^-11 / sqrt(3) of the power of two below it in
    the mean square, and stands before a code that is counted from the middle, -8 .. 7; errors of different tokens
    are independent.  (The weights' 16 bits for the minima and the scores' 32-bit sums are 2^-5 of that and less.)"""
    w = np.repeat(s, 32, -1)
    want = p @ (codes * w + np.repeat(lo, 32, -1))
    return want, (p ** 2) @ ((w * (codes - 8)) ** 2) * (2.0 ** -22 / 3)


def check(out, want, before) -> None:
    """All outputs of a call together, [...][128]: out as bf16 numbers, want and before as of `allowed`.  The last rounding takes
    what it takes on the exact result; 2 % are left for chance (32768 outputs and more: their sum of squares varies by 1 %)."""
    assert out.size >= 32768
    last = ((ref.bf16(want.astype(np.float32)) - want) ** 2).sum()
    have, most = ((out - want) ** 2).sum(), 1.02 * (last + before.sum())
    assert have <= most, f"squared error {have / last:.4f} of the last rounding's, {most / last:.4f} allowed"
