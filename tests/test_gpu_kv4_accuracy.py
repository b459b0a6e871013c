"""Attention over 4-bit blocks where its arithmetic is hardest put to it: tokens without any weight beside values of any size."""
import numpy as np
import pytest
import torch

from tests import kv4_accuracy as acc
from tests import kv4_reference as ref
from tests.test_gpu_kv4 import attention_case, bf, clean, context, dev, i32, run_attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def two_classes(pi, heavy, q_sign, v_heavy, v_light, key):
    """One sequence of len(heavy) tokens.  Keys are constant rows (stored exactly): +key for the heavy tokens, -key for the light
    ones; queries are q_sign * key.  Returns out and lse of the kernel, the 64-bit result, and per (head, channel) the sums of
    weight * largest |value| of the channel's group over the tokens of the head's own class and over the others."""
    c = pi.cfg
    B, H, K, C, n = c.block_tokens, c.n_kv_heads, c.budget_blocks, c.pool_slots, len(heavy)
    nb = -(-n // B)
    kv = np.zeros((C, H, 2, B, 128), dtype=np.float32)
    slots = np.random.default_rng(n).permutation(C)[:nb]
    for t in range(n):
        kv[slots[t // B], :, 0, t % B] = key if heavy[t] else -key
        kv[slots[t // B], :, 1, t % B] = v_heavy[t] if heavy[t] else v_light[t]
    pool = ref.pack(ref.bf16(kv), B)
    held = ref.unpack(pool, H, B)
    q = np.repeat(np.asarray(q_sign, dtype=np.float32)[:, None] * np.float32(key), 128, 1)
    assert np.array_equal(q, ref.bf16(q)) and q.shape[0] == c.n_q_heads
    blocks = np.full((1, K), -1, dtype=np.int32)
    where = np.full((1, K), -1, dtype=np.int32)
    blocks[0, :nb], where[0, :nb] = np.arange(nb), slots
    out, lse = torch.zeros((1, c.n_q_heads, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((1, c.n_q_heads), device=DEV)
    pi.sparse_decode_attn_kv4(0, bf(q[None]), dev(pool[None]), dev(where), dev(blocks), i32([nb]), i32([n]), out, lse)
    clean(pi)
    want, own, other = [np.zeros((c.n_q_heads, 128)) for _ in range(3)]
    want_lse = np.zeros(c.n_q_heads)
    heavy = np.asarray(heavy)
    for g in range(c.n_q_heads):
        h = g // (c.n_q_heads // H)
        k, v = [np.concatenate([held[s, h, i] for s in slots])[:n] for i in (0, 1)]
        z = k @ q[g].astype(np.float64) / np.sqrt(128)
        p = np.exp(z - z.max())
        want_lse[g] = z.max() + np.log(p.sum())
        p /= p.sum()
        want[g] = p @ v
        size = np.repeat(np.abs(v).reshape(n, 4, 32).max(2), 32, 1)
        mine = heavy if q_sign[g] > 0 else ~heavy
        own[g], other[g] = p[mine] @ size[mine], p[~mine] @ size[~mine]
    return out[0].double().cpu().numpy(), lse[0].double().cpu().numpy(), want, want_lse, own, other


PLACES = {
    "side by side": [True, False],                                             # one step
    "light ones behind": [True] * 2200 + [False] * 2200,                       # several steps of every warp each
    "light ones first": [False] * 2200 + [True] * 2200,
    "in turn": [True, False, False] * 1400,
}


@pytest.mark.parametrize("Hq,Hkv", [(4, 1), (8, 1), (16, 2), (16, 1)])
@pytest.mark.parametrize("place", PLACES)
@pytest.mark.parametrize("heads", ["alike", "both ways"])
def test_attention_with_tokens_of_no_weight_and_values_of_any_size(Hq, Hkv, place, heads):
    """What the light tokens hold must not be seen in the heavy ones' result: keys of 3 put their scores 204 below (weights
    of 2^-294, which are 0 in 32 bits), keys of 1.875 80 below (2^-115).  The other way round for the heads whose query is turned."""
    pi = context(n_q_heads=Hq, n_kv_heads=Hkv, budget_blocks=300, pool_slots=300, max_batch=1, max_blocks=300, n_sink_blocks=0, n_local_blocks=1)
    heavy, n = PLACES[place], len(PLACES[place])
    rng = np.random.default_rng(n)
    sign = np.ones(Hq) if heads == "alike" else np.where(np.arange(Hq) % 3 == 1, -1.0, 1.0)
    for size in (4e3, 2.0 ** 24, 1e12, 1e30):
        light = np.where(np.arange(128) % 2 == 0, 0.0, size)[None].repeat(n, 0)
        for key in (3.0, 1.875):
            for values in ("none", "constant", "any"):
                v = {"none": np.zeros((n, 128)), "constant": np.full((n, 128), 2.5), "any": rng.standard_normal((n, 128))}[values]
                out, lse, want, want_lse, own, other = two_classes(pi, heavy, sign, v, light, key)
                # one rounding to bf16.  Tokens of one class have the same score to the bit, so only weight times scale is
                # rounded for them: by at most 2^-11, at most 15 codes of it, and 15 scales are at most twice the
                # largest |v| of the group.  The weights of the other class carry the scores' error as well: a constant
                # row has one product, of the minimum and the query's sum, and no more than 32 roundings of 2^-23
                score = 128 * key * key / np.sqrt(128)
                eps = 2 * 32 * 2.0 ** -23 * score
                tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * own + (2.0 ** -10 + 2 * eps) * other + 1e-30
                assert (np.abs(out - want) <= tol).all(), (size, key, values, np.abs(out - want).max(), int(np.isnan(out).sum()))
                assert (np.abs(lse - want_lse) <= eps + 2.0 ** -18).all()
    pi.close()


@pytest.mark.parametrize("Hq,Hkv,B,K,n", [(32, 8, 16, 64, 8), (64, 8, 32, 16, 4), (128, 8, 16, 40, 2), (8, 2, 64, 20, 32), (4, 1, 16, 300, 64)])
def test_attention_is_as_near_as_its_bits_allow(Hq, Hkv, B, K, n):
    """Ordinary keys and values; the outputs' error in the mean square, and the logarithms of the sums."""
    pi = context(n_q_heads=Hq, n_kv_heads=Hkv, block_tokens=B, budget_blocks=K, pool_slots=K + 3, max_batch=n, max_blocks=2 * K, n_sink_blocks=0, n_local_blocks=1)
    rng = np.random.default_rng(Hq * 1000 + K)
    case = attention_case(pi, rng.integers(K * B // 2, 2 * K * B + 1, n), Hq + K, garbage=False)
    kv = ref.bf16(rng.standard_normal((n * (K + 3), Hkv, 2, B, 128)))                # (means of 0: the outputs' last rounding hides least)
    case["pool"] = ref.pack(kv, B).reshape(case["pool"].shape)
    out, lse = run_attention(pi, case)
    out, lse = out.double().cpu().numpy().reshape(n, Hkv, Hq // Hkv, 128), lse.double().cpu().numpy().reshape(n, Hkv, Hq // Hkv)
    want, before = np.empty_like(out), np.empty_like(out)
    for s in range(n):
        codes, scales, lows = acc.tokens(case["pool"][s], case["slots"][s], case["blocks"][s], int(case["count"][s]), int(case["ctx"][s]), Hkv, B)
        for h in range(Hkv):
            q = case["q"][s].astype(np.float64).reshape(Hkv, Hq // Hkv, 128)[h]
            p, want_lse = acc.softmax(q, codes[h, 0], scales[h, 0], lows[h, 0])
            want[s, h], before[s, h] = acc.allowed(p, codes[h, 1], scales[h, 1], lows[h, 1])
            # A score is the sum of four groups, each of two products that are added up in 32 bits and may be cut: by 2^-23 of
            # a sum below 128 * 4 (every second code carries 64, queries are below 2, of either sign), times a scale of
            # about 0.3, the queries' power of two (at most 4) and 1 / sqrt(D): 2 * 2 * 2^-23 * 512 * 0.3 * 0.35 = 2^-15.3 where
            # all eight cuts of all tokens went the same way and were as large as they can be
            assert (np.abs(lse[s, h] - want_lse) <= 2.0 ** -15).all()
    acc.check(out, want, before)
    pi.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6])
@pytest.mark.parametrize("rot,inter", [(128, False), (64, False), (52, False), (128, True)])
def test_norm_of_rows_of_any_size(dtype, eps, rot, inter):
    """From numbers whose squares are lost below 32 bits to those whose squares are beyond, side by side."""
    pi = context(n_q_heads=10, n_kv_heads=2)
    sizes = np.asarray([1.0, 1e-38, 1e-30, 1e-22, 1e-15, 1e-3, 1e3, 1e17, 1e19, 1e22, 1e30, 5e37])
    g = torch.Generator().manual_seed(4)
    T = 24
    x = torch.randn((T, 12, 128), generator=g, dtype=torch.float64)
    for t in range(T):
        x[t] *= torch.from_numpy(np.roll(sizes, t))[:, None]
    x = x.to(dtype).to(DEV)
    q, k = x[:, :10].contiguous(), x[:, 10:].contiguous()
    pos = np.random.default_rng(0).integers(0, 1 << 17, T).astype(np.int32)
    freq = (500000.0 ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)
    w = (1 + 0.3 * np.random.default_rng(9).standard_normal((2, 128))).astype(np.float32)
    qo, ko = torch.empty_like(q, dtype=torch.bfloat16), torch.empty_like(k, dtype=torch.bfloat16)
    pi.qk_norm_rope(q, k, i32(pos), dev(freq), qo, ko, q_weight=dev(w[0]), k_weight=dev(w[1]), eps=eps, interleaved=inter)
    clean(pi)
    for got, src, weight in ((qo, q, w[0]), (ko, k, w[1])):
        want = ref.rope(src.double().cpu().numpy(), pos, freq, weight, float(np.float32(eps)), inter)
        # one rounding to bf16; before it the norm and the turn in 32 bits, under 2^-19 of the row's largest pair
        tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * np.abs(want).max(-1, keepdims=True) * np.sqrt(2) + 1e-37
        bad = ~(np.abs(got.double().cpu().numpy() - want) <= tol)
        assert not bad.any(), np.argwhere(bad.any(-1))[:5]
    pi.close()
