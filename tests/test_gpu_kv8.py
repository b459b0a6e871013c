"""The 8-bit cache on the GPU, against the plain references of kv8_reference."""
import numpy as np
import pytest
import torch

from tests import kv8_reference as ref
from tests.test_gpu_kv4 import bf, clean, context, dev, i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def tokens_of(rng, T, heads, spread=2.0):
    """k, v as bf16 numbers, sizes that differ from token to token."""
    kv = ref.bf16(rng.standard_normal((T, 2, heads, 128)) * np.exp(rng.standard_normal((T, 2, heads, 1)) * spread))
    return kv[:, 0], kv[:, 1]


def slots_of(rng, T, B, pages, at=0):
    """Runs of tokens in order through scattered pages, the first from place `at` on."""
    order = rng.permutation(pages)
    t = np.arange(T) + at
    return (order[t // B] * B + t % B).astype(np.int64)


# ------------------------------------------------------------------ store and load
@pytest.mark.parametrize("heads,block", [(1, 16), (2, 32), (4, 16), (8, 16), (8, 64), (16, 32)])
@pytest.mark.parametrize("tokens,at", [(1, 0), (1, 15), (7, 3), (130, 0), (333, 9)])
def test_store_writes_the_reference_bytes_and_nothing_else(heads, block, tokens, at):
    pi = context(n_q_heads=heads, n_kv_heads=heads, block_tokens=block)
    rng = np.random.default_rng(heads * 1000 + block + tokens)
    pages = -(-(tokens + at) // block) + 2
    k, v = tokens_of(rng, tokens, heads)
    if tokens > 5:
        k, v = k.copy(), v.copy()
        k[0], v[1] = 0, np.float32(1e-39)                                              # nothing, subnormal
        k[3, 0, 5], v[4, 0, 7], v[4, 0, 8] = np.nan, np.inf, -np.inf
    slots = slots_of(rng, tokens, block, pages, at)
    if tokens > 8:
        slots[-3:] = -1                                                                # padding
    before = ref.pack(ref.bf16(rng.standard_normal((pages, heads, 2, block, 128)) * np.exp(rng.standard_normal((pages, heads, 2, 1, 1)) * 3)), block)
    want = before.copy()
    ref.store(want, k, v, slots, block)
    store = dev(before)
    pi.kv8_store(bf(k), bf(v), store, dev(slots))
    clean(pi)
    got = store.cpu().numpy()
    assert got.shape[1] == pi.kv8_block_bytes == ref.block_bytes(heads, block)
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]
    out = torch.full((pages, heads, 2, block, 128), 5.0, dtype=torch.bfloat16, device=DEV)
    pi.kv8_load(store, out)
    clean(pi)
    assert np.array_equal(out.double().cpu().numpy(), ref.unpack(want, heads, block), equal_nan=True)       # products are exact
    pi.close()


def test_store_in_two_calls_raises_scales_and_begins_blocks_anew():
    """A block filled by several calls: small tokens, then large ones (scales grow, old tokens are rounded again), then small ones (scales
    stay); then its first token again."""
    pi = context(n_q_heads=2, n_kv_heads=2, block_tokens=32)
    rng = np.random.default_rng(3)
    store = torch.full((3, pi.kv8_block_bytes), 255, dtype=torch.uint8, device=DEV)    # never written: NaN all over
    want = store.cpu().numpy()
    for places, size in ((range(0, 5), 1e-3), (range(5, 9), 1.0), (range(9, 12), 1e-30), (range(12, 13), 2.0 ** 100), (range(13, 32), 3.0), ([0, 1], 1e-6), (range(2, 6), 0.0)):
        n = len(places)
        k, v = ref.bf16(rng.standard_normal((2, n, 2, 128)) * np.float64(size))
        slots = np.asarray(places, dtype=np.int64) + 32
        pi.kv8_store(bf(k), bf(v), store, dev(slots))
        clean(pi)
        ref.store(want, k, v, slots, 32)
        assert np.array_equal(store.cpu().numpy(), want), size
    pi.close()


def test_store_of_the_largest_and_smallest_values():
    pi = context(n_q_heads=1, n_kv_heads=1, block_tokens=16)
    top = np.float32(3.3895313892515355e38)                                            # the largest bf16 number
    k = np.zeros((3, 1, 128), dtype=np.float32)
    k[0, 0, :4] = top, -top, top / 2, 2.0 ** 127
    k[1, 0, :4] = 2.0 ** -126, 2.0 ** -110, -(2.0 ** -118), 2.0 ** -133
    k[2, 0, :4] = 1.0, 2.0 ** -60, np.inf, -1.75
    slots = np.asarray([0, 16, 32], dtype=np.int64)
    store = torch.zeros((3, pi.kv8_block_bytes), dtype=torch.uint8, device=DEV)
    want = store.cpu().numpy()
    pi.kv8_store(bf(k), bf(-k), store, dev(slots))
    clean(pi)
    ref.store(want, k, -k, slots, 16)
    assert np.array_equal(store.cpu().numpy(), want)
    out = torch.zeros((3, 1, 2, 16, 128), dtype=torch.bfloat16, device=DEV)
    pi.kv8_load(store, out)
    clean(pi)
    o = out.double().cpu().numpy()
    assert np.isinf(o[0, 0, 0, 0, :2]).all() and o[0, 0, 0, 0, 3] == 2.0 ** 127 and o[1, 0, 0, 0, 1] == 2.0 ** -110 and np.isnan(o[2, 0, 0, 0, 2]) and o[2, 0, 1, 0, 3] == 1.75
    pi.close()


def test_store_of_runs_of_tokens_equals_store_token_by_token_and_a_pinned_store():
    pi = context(n_q_heads=4, n_kv_heads=4, block_tokens=16)
    rng = np.random.default_rng(7)
    for N, M in ((3, 16), (5, 7), (40, 1), (1, 100)):
        kv = bf(rng.standard_normal((N, 4, 2, M, 128)))
        k, v = kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)                # [N][M][head][128]
        pages = N * M // 16 + 1
        whole, pinned = torch.zeros((pages, pi.kv8_block_bytes), dtype=torch.uint8, device=DEV), torch.zeros((pages, pi.kv8_block_bytes), dtype=torch.uint8).pin_memory()
        pi.kv8_store(k, v, whole)
        pi.kv8_store(k.reshape(N * M, 4, 128), v.reshape(N * M, 4, 128), pinned, torch.arange(N * M, device=DEV))
        clean(pi)
        assert torch.equal(whole.cpu(), pinned)
        want = np.zeros((pages, pi.kv8_block_bytes), dtype=np.uint8)
        ref.store(want, k.float().cpu().numpy().reshape(N * M, 4, 128), v.float().cpu().numpy().reshape(N * M, 4, 128), range(N * M), 16)
        assert np.array_equal(pinned.numpy(), want)
        out = [torch.zeros((pages, 4, 2, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        pi.kv8_load(whole, out[0])
        pi.kv8_load(pinned, out[1])
        clean(pi)
        assert torch.equal(*out)
    pi.close()


def test_store_and_load_skip_and_report_what_lies_beyond_the_store():
    pi = context(n_q_heads=2, n_kv_heads=2, block_tokens=16)
    rng = np.random.default_rng(5)
    k, v = tokens_of(rng, 6, 2)
    slots = np.asarray([0, 1, 48, 1 << 40, -(1 << 50), 17], dtype=np.int64)
    store = torch.zeros((3, pi.kv8_block_bytes), dtype=torch.uint8, device=DEV)
    want = store.cpu().numpy()
    ref.store(want, k, v, slots, 16)
    pi.kv8_store(bf(k), bf(v), store, dev(slots))
    got = clean(pi, -8)
    assert got[1] == 6 and got[2] in (2, 3) and np.array_equal(store.cpu().numpy(), want)
    out = torch.full((3, 2, 2, 16, 128), 4.0, dtype=torch.bfloat16, device=DEV)
    pi.kv8_load(store, out, i32([1, 3, 0]))
    assert clean(pi, -8)[1] == 6
    held = ref.unpack(want, 2, 16)
    o = out.double().cpu().numpy()
    assert np.array_equal(o[0], held[1]) and (o[1] == 4).all() and np.array_equal(o[2], held[0])
    pi.kv8_store(bf(k)[:0], bf(v)[:0], store)                                          # no token: nothing happens
    pi.kv8_load(store, out[:0], i32([]))
    clean(pi)
    assert np.array_equal(store.cpu().numpy(), want)
    pi.close()


def test_the_front_end_checks_devices_types_and_shapes():
    pi = context()
    n = pi.kv8_block_bytes
    k = torch.zeros((4, 2, 128), dtype=torch.bfloat16, device=DEV)
    store, pool, small = torch.zeros((4, n), dtype=torch.uint8, device=DEV), torch.zeros((1, 24, n), dtype=torch.uint8, device=DEV), torch.zeros((4, pi.kv4_block_bytes), dtype=torch.uint8, device=DEV)
    with pytest.raises(TypeError):
        pi.kv8_store(k, k, small)                                                      # 4-bit blocks
    with pytest.raises(TypeError):
        pi.kv4_store(k, k, store)                                                      # 8-bit blocks
    with pytest.raises(TypeError):
        pi.kv8_store(k.float(), k.float(), store)
    with pytest.raises(ValueError):
        pi.kv8_store(k, k[:3], store)
    with pytest.raises(Exception) as e:
        pi.kv8_store(k, k, torch.zeros((4, n), dtype=torch.uint8))                     # pageable
    assert getattr(e.value, "code", None) == -5
    with pytest.raises(ValueError):
        pi.kv8_load(store, torch.zeros((4, 2, 2, 32, 128), dtype=torch.bfloat16, device=DEV))
    q, sel, one = torch.zeros((1, 8, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((1, 16), dtype=torch.int32, device=DEV), i32([1])
    with pytest.raises(ValueError):
        pi.sparse_decode_attn_kv8(0, q, pool[:, :20].contiguous(), sel, sel, one, one, torch.zeros_like(q))
    with pytest.raises(TypeError):
        pi.sparse_decode_attn(0, q, pool, sel, sel, one, one, torch.zeros_like(q))     # the bf16 call
    with pytest.raises(Exception) as e:
        pi.sparse_decode_attn_kv8(3, q, pool, sel, sel, one, one, torch.zeros_like(q))
    assert getattr(e.value, "code", None) == -1
    clean(pi)
    pi.close()


# ------------------------------------------------------------------ append and recall
@pytest.mark.parametrize("heads,block,paged,dev_step", [(2, 16, False, False), (8, 16, True, True), (1, 64, False, True), (4, 32, True, False)])
def test_append_over_block_borders(heads, block, paged, dev_step):
    pi = context(n_q_heads=heads, n_kv_heads=heads, block_tokens=block, pool_slots=20, max_blocks=40, solo_head=[heads - 1])
    rng = np.random.default_rng(heads + block)
    n, NB, C = 3, 40, 20
    ctx = np.asarray([12 * block + block - 2, 25 * block, 5 * block + 1])
    table, slot_block = np.full((n, NB), -1, dtype=np.int32), np.full((n, C), -1, dtype=np.int32)
    stamp = rng.integers(0, 50, (n, C)).astype(np.int32)
    for s in range(n):
        cur = -(-int(ctx[s]) // block)
        must = sorted({0} | set(range(max(0, cur - 2), cur)))
        other = [b for b in rng.permutation(cur) if b not in must][:C - len(must) - (2 if s == 0 else 0)]
        for slot, b in zip(rng.permutation(C), must + other):
            table[s, b], slot_block[s, slot] = slot, b
    digest = ref.bf16(np.stack((rng.standard_normal((n, NB, 128)) - 1, rng.standard_normal((n, NB, 128)) + 1), 2))
    pool = np.empty((n, C, pi.kv8_block_bytes), dtype=np.uint8)
    pages = rng.permutation(n * NB).astype(np.int32).reshape(n, NB) if paged else None
    store = ref.pack(ref.bf16(rng.standard_normal((n * NB, heads, 2, block, 128)) * np.exp(2 * rng.standard_normal((n * NB, heads, 2, 1, 1)))), block)
    for s in range(n):                                                                 # pool and store hold the same
        for slot in range(C):
            b = slot_block[s, slot]
            pool[s, slot] = 77 if b < 0 else store[pages[s, b] if paged else s * NB + b]
    if not paged:
        store = store.reshape(n, NB, -1)
    sim = ref.Appender(table, slot_block, stamp, digest, pool, store, pi.cfg, heads - 1)
    d = [dev(table), dev(slot_block), dev(stamp), bf(digest)]
    pool_d, store_d = dev(pool), torch.from_numpy(store.copy()).pin_memory()
    pt = dev(pages) if paged else None
    for step in range(100, 106):
        k, v = ref.bf16(rng.standard_normal((2, n, heads, 128)) * np.exp(2.5 * rng.standard_normal((2, n, heads, 1))))
        if step == 104:
            k[0, 0, 3], v[1, heads - 1, 4] = np.nan, np.inf
            k[0, heads - 1], v[2] = ref.bf16(np.nan_to_num(k[0, heads - 1])), 0
        st = i32([step]) if dev_step else step
        pi.append_kv8(0, st, bf(k), bf(v), i32(ctx), store_d, pool_d, d[0], d[1], d[2], d[3], page_table=pt)
        clean(pi)
        sim.step(ctx, k, v, step, pages)
        assert np.array_equal(d[0].cpu().numpy(), sim.table) and np.array_equal(d[1].cpu().numpy(), sim.slot_block)
        assert np.array_equal(d[2].cpu().numpy(), sim.stamp) and np.array_equal(d[3].float().cpu().numpy(), sim.digest)
        assert np.array_equal(pool_d.cpu().numpy(), sim.pool) and np.array_equal(store_d.numpy(), sim.store), step
        ctx = ctx + 1
    pi.close()


def test_append_reports_what_cannot_be_appended():
    pi = context(pool_slots=16, max_blocks=10)
    store = torch.zeros((2, 10, pi.kv8_block_bytes), dtype=torch.uint8, device=DEV)
    pool = torch.zeros((2, 16, pi.kv8_block_bytes), dtype=torch.uint8, device=DEV)
    k = torch.ones((2, 2, 128), dtype=torch.bfloat16, device=DEV)

    def tables():
        return (torch.full((2, 10), -1, dtype=torch.int32, device=DEV), torch.full((2, 16), -1, dtype=torch.int32, device=DEV),
                torch.zeros((2, 16), dtype=torch.int32, device=DEV), torch.zeros((2, 10, 2, 128), dtype=torch.bfloat16, device=DEV))

    pi.append_kv8(0, 1, k, k, i32([160, 0]), store, pool, *tables())                   # block 10 of ten
    assert clean(pi, -9)[1] == 5
    pi.append_kv8(0, 1, k, k, i32([5, 0]), store, pool, *tables())                     # the block being filled is not resident
    assert clean(pi, -8)[1] == 5
    pages = torch.full((2, 10), 20, dtype=torch.int32, device=DEV)
    pi.append_kv8(0, 1, k, k, i32([0, 0]), store, pool, *tables(), page_table=pages)   # page 20 of twenty
    assert clean(pi, -8)[1] == 5
    assert int(store[:, 1:].sum()) == 0 and int(pool[:, 2:].sum()) == 0
    pi.close()


@pytest.mark.parametrize("heads,block,paged", [(1, 16, False), (2, 16, True), (8, 16, True), (16, 64, False)])
def test_recall_moves_whole_blocks_and_skips_what_leaves_the_pool(heads, block, paged):
    pi = context(n_q_heads=heads, n_kv_heads=heads, block_tokens=block, pool_slots=16, max_blocks=30)
    rng = np.random.default_rng(heads)
    n, NB, C, size = 3, 30, 16, pi.kv8_block_bytes
    host = torch.from_numpy(rng.integers(0, 256, (n, NB, size), dtype=np.uint8)).pin_memory()
    pages = rng.permutation(n * NB).astype(np.int32).reshape(n, NB) if paged else None
    logical = host.numpy() if not paged else host.numpy().reshape(n * NB, -1)[pages]
    lists = np.zeros((n, 16, 4), dtype=np.int32)
    lists[0, :3] = [[2, 0, 3, 0], [9, 5, 1, 3], [20, 12, 4, 4]]
    lists[2, :1] = [[29, 15, 1, 0]]
    pool = torch.full((n, C, size), 3, dtype=torch.uint8, device=DEV)
    want = np.full((n, C, size), 3, dtype=np.uint8)
    for s, cnt in ((0, 3), (2, 1)):
        for src, dst, m, _ in lists[s, :cnt]:
            want[s, dst:dst + m] = logical[s, src:src + m]
    pi.recall_kv8(0, host, pool, dev(lists), i32([3, 0, 1]), page_table=None if pages is None else dev(pages))
    clean(pi)
    assert np.array_equal(pool.cpu().numpy(), want)
    lists[1, :1] = [[0, 15, 2, 0]]                                                     # its second block would land behind the pool's sequence
    pi.recall_kv8(0, host, pool, dev(lists), i32([0, 1, 0]), page_table=None if pages is None else dev(pages))
    got = clean(pi, -8)
    want[1, 15] = logical[1, 0]
    assert got[1] == 3 and np.array_equal(pool.cpu().numpy(), want)
    lists[1, :1] = [[29, 2, 2, 0]]                                                     # and one that leaves the store
    pi.recall_kv8(0, host, pool, dev(lists), i32([0, 1, 0]), page_table=None if pages is None else dev(pages))
    got = clean(pi, -8)
    want[1, 2] = logical[1, 29]
    assert got[1] == 3 and np.array_equal(pool.cpu().numpy(), want)
    pi.close()


# ------------------------------------------------------------------ attention
def attention_case(pi, ctx, seed, garbage=True, spread=1.0):
    """Pool, lists and queries for the given lengths: the newest block and others, in scattered slots; blocks of different sizes."""
    c = pi.cfg
    rng = np.random.default_rng(seed)
    n, K, C, B, H = len(ctx), c.budget_blocks, c.pool_slots, c.block_tokens, c.n_kv_heads
    kv = rng.standard_normal((n * C, H, 2, B, 128)) * np.exp(spread * rng.standard_normal((n * C, H, 2, 1, 1)) * np.asarray([0.3, 2.0])[:, None, None])
    kv[..., [3, 90]] *= 8
    pool = ref.pack(ref.bf16(kv), B).reshape(n, C, -1)
    blocks, slots = np.full((n, K), -1, dtype=np.int32), np.full((n, K), -1, dtype=np.int32)
    count = np.zeros(n, dtype=np.int32)
    for s in range(n):
        nb = -(-int(ctx[s]) // B)
        count[s] = min(nb, K)
        if nb:
            rest = rng.permutation(nb - 1)[:count[s] - 1] if nb > 1 else []
            blocks[s, :count[s]] = np.sort(np.append(rest, nb - 1))
            slots[s, :count[s]] = rng.permutation(C)[:count[s]]
        last = int(ctx[s]) % B
        if nb and last and garbage:                                                    # behind the last token: NaN
            ref.parts(pool[s, slots[s, count[s] - 1]], H, B)[0][:, :, last:] = 255
    q = ref.bf16(rng.standard_normal((n, c.n_q_heads, 128)))
    return dict(pool=pool, blocks=blocks, slots=slots, count=count, ctx=np.asarray(ctx), q=q)


def check_attention(pi, case, out, lse):
    c = pi.cfg
    out, lse = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    for s in range(len(case["ctx"])):
        def kv_of(slot):
            return ref.unpack(case["pool"][s, slot][None], c.n_kv_heads, c.block_tokens)[0]
        want, want_lse, tol, eps = ref.attention(case["q"][s].astype(np.float64), kv_of, case["blocks"][s], case["slots"][s], int(case["count"][s]), int(case["ctx"][s]), c.block_tokens)
        assert (np.abs(out[s] - want) <= tol).all(), (s, (np.abs(out[s] - want) / tol).max())
        if lse is not None:
            if np.isinf(want_lse).any():
                assert (lse[s] == -np.inf).all() and (out[s] == 0).all()
            else:
                assert (np.abs(lse[s] - want_lse) <= eps + 2.0 ** -20 * np.abs(want_lse) + 2.0 ** -18).all()


def run_attention(pi, case, lse=True, stream=None):
    n, c = len(case["ctx"]), pi.cfg
    out = torch.full((n + 1, c.n_q_heads, 128), 9.0, dtype=torch.bfloat16, device=DEV)
    l = torch.full((n + 1, c.n_q_heads), 9.0, dtype=torch.float32, device=DEV)
    pi.sparse_decode_attn_kv8(0, bf(case["q"]), dev(case["pool"]), dev(case["slots"]), dev(case["blocks"]), dev(case["count"]), i32(case["ctx"]),
                              out[:n], l[:n] if lse else None, stream=stream)
    clean(pi)
    assert (out[n] == 9).all() and (l[n] == 9).all()                                   # rows behind the last sequence
    return out[:n], l[:n] if lse else None


@pytest.mark.parametrize("Hq,Hkv,B,K,ctx", [
    (8, 2, 16, 16, [1, 0, 250, 256]),
    (1, 1, 16, 1, [1, 16, 700]),
    (2, 2, 64, 3, [63, 64, 65, 5]),
    (3, 1, 32, 24, [700, 31, 33]),                    # three query heads per KV head
    (16, 4, 16, 40, [640, 641, 3999]),
    (5, 1, 16, 9, [100, 7]),                          # five
    (64, 8, 16, 64, [1024, 500]),                     # eight
    (12, 1, 16, 9, [100, 7]),                         # twelve
    (32, 2, 32, 8, [255, 256, 0]),                    # sixteen
    (16, 16, 64, 5, [320, 1]),                        # sixteen KV heads
    (32, 8, 16, 64, [8192]),                          # one sequence: a cluster an item
    (8, 8, 16, 3, [40] * 40),                         # many items: one CTA each
    (4, 1, 16, 300, [4795, 16, 4800]),                # more than 32 tiles a warp
    (20, 2, 16, 300, [4800, 3]),
    (8, 1, 64, 70, [4480, 0, 77]),
])
def test_attention(Hq, Hkv, B, K, ctx):
    pi = context(n_q_heads=Hq, n_kv_heads=Hkv, block_tokens=B, budget_blocks=K, pool_slots=K + 3, max_batch=max(8, len(ctx)), max_blocks=max(256, 2 * K), n_sink_blocks=0, n_local_blocks=1)
    case = attention_case(pi, ctx, Hq * 100 + K)
    out, lse = run_attention(pi, case)
    check_attention(pi, case, out, lse)
    again, _ = run_attention(pi, case, lse=False)
    assert torch.equal(out, again)
    pi.close()


@pytest.mark.parametrize("Hq,Hkv,B", [(8, 1, 64), (32, 8, 16), (48, 4, 32)])
def test_attention_random_shapes(Hq, Hkv, B):
    rng = np.random.default_rng(Hq + B)
    for _ in range(6):
        K, batch = int(rng.integers(1, 80)), int(rng.integers(1, 12))
        pi = context(n_q_heads=Hq, n_kv_heads=Hkv, block_tokens=B, budget_blocks=K, pool_slots=K + int(rng.integers(0, 9)), max_batch=batch,
                     max_blocks=2 * K, n_sink_blocks=0, n_local_blocks=1)
        case = attention_case(pi, rng.integers(0, 2 * K * B + 1, batch), int(rng.integers(1 << 30)))
        out, lse = run_attention(pi, case)
        check_attention(pi, case, out, lse)
        pi.close()


@pytest.mark.parametrize("batch,B,K", [(12, 16, 64), (12, 16, 33), (12, 32, 9), (13, 64, 4), (21, 16, 40), (30, 32, 5), (40, 16, 17)])
def test_attention_of_many_sequences(batch, B, K):
    """A CTA for each (sequence, KV head), of 4, 8 or 16 warps; ragged, some sequences empty."""
    rng = np.random.default_rng(batch + K)
    pi = context(n_q_heads=32, n_kv_heads=8, block_tokens=B, budget_blocks=K, pool_slots=K + 2, max_batch=batch, max_blocks=2 * K, n_sink_blocks=0, n_local_blocks=1)
    ctx = rng.integers(1, 2 * K * B + 1, batch)
    ctx[[1, batch - 1]] = 0, 2 * K * B
    case = attention_case(pi, ctx, batch)
    out, lse = run_attention(pi, case)
    check_attention(pi, case, out, lse)
    pi.close()


@pytest.mark.parametrize("spread", [6.0, 12.0])
def test_attention_over_blocks_of_very_different_sizes(spread):
    """V's scales differ by many powers of two between blocks, and scores are in the hundreds: what has the weight keeps its bits, however
    small its values are next to a block's that has none."""
    pi = context(budget_blocks=20)
    case = attention_case(pi, [300, 17], 3, spread=spread)
    for factor in (1.0, 30.0):
        case["q"] = ref.bf16(case["q"] * np.float32(factor))
        out, lse = run_attention(pi, case)
        check_attention(pi, case, out, lse)
    pi.close()


@pytest.mark.parametrize("size", [1e-30, 1e-3, 1e4, 1e30])
def test_attention_with_small_and_large_values(size):
    pi = context(budget_blocks=20)
    case = attention_case(pi, [300, 17], 4)
    rng = np.random.default_rng(1)
    kv = ref.bf16(rng.standard_normal((2 * pi.cfg.pool_slots, 2, 2, 16, 128)))
    kv[:, :, 1] = ref.bf16(kv[:, :, 1] * np.float32(size))                             # V; scores stay ordinary
    case["pool"] = ref.pack(kv, 16).reshape(case["pool"].shape)
    out, lse = run_attention(pi, case)
    check_attention(pi, case, out, lse)
    kv = ref.bf16(rng.standard_normal((2 * pi.cfg.pool_slots, 2, 2, 16, 128)))
    kv[:, :, 0] = ref.bf16(kv[:, :, 0] * np.float32(size))                             # K, and queries as much the other way
    case["q"] = ref.bf16(case["q"] / np.float32(size))
    case["pool"] = ref.pack(kv, 16).reshape(case["pool"].shape)
    out, lse = run_attention(pi, case)
    check_attention(pi, case, out, lse)
    pi.close()


@pytest.mark.parametrize("size", [1e4, 1e9, 1e20, 1e32])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_attention_with_scores_of_any_size(size, sign):
    """Equal scores, then one that stands out, anywhere in the range of 32 bits."""
    pi = context(budget_blocks=20)
    c = pi.cfg
    case = attention_case(pi, [300, 17], 5, garbage=False)
    rng = np.random.default_rng(2)
    kv = ref.bf16(rng.standard_normal((2 * c.pool_slots, 2, 2, 16, 128)))
    key = float(np.float32(2.0 ** round(np.log2(size ** 0.5))))
    kv[:, :, 0] = key
    q = float(ref.bf16(np.float32(sign * 1.71 * size ** 0.5)))
    case["q"][:] = q
    case["pool"] = ref.pack(kv, 16).reshape(case["pool"].shape)
    score = 128 * q * key / 128 ** 0.5
    out, lse = run_attention(pi, case)
    held = ref.unpack(case["pool"].reshape(2 * c.pool_slots, -1), 2, 16).reshape(2, c.pool_slots, 2, 2, 16, 128)
    pick = []
    for s, n in enumerate((300, 17)):
        v = np.concatenate([held[s, case["slots"][s, i], :, 1, :min(16, n - 16 * case["blocks"][s, i])] for i in range(case["count"][s])], axis=1)
        assert v.shape[1] == n
        want, spread = np.repeat(v.mean(axis=1), 4, axis=0), np.repeat(np.abs(v).mean(axis=1), 4, axis=0)
        # weights are all alike but for their rounding to fp16; the score carries eight cuts of 2^-23 and four roundings of 2^-24: below 2^-19 of itself
        assert (np.abs(out[s].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * spread).all()
        assert (np.abs(lse[s].double().cpu().numpy() - (score + np.log(n))) <= 2.0 ** -19 * abs(score) + 2.0 ** -18).all()
        pick.append(v[:, 0])
    # the first token of each list half as far from 0 (scores below it) or twice as far (above it): the others' weights are nothing
    for s in range(2):
        kv.reshape(2, c.pool_slots, 2, 2, 16, 128)[s, case["slots"][s, 0], :, 0, 0] = key * (2.0 if sign > 0 else 0.5)
    case["pool"] = ref.pack(kv, 16).reshape(case["pool"].shape)
    out, lse = run_attention(pi, case)
    for s in range(2):
        want = np.repeat(pick[s], 4, axis=0)
        assert (np.abs(out[s].double().cpu().numpy() - want) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(want) + 1e-30).all()
        top = score * (2.0 if sign > 0 else 0.5)
        assert (np.abs(lse[s].double().cpu().numpy() - top) <= 2.0 ** -19 * abs(top) + 2.0 ** -18).all()
    pi.close()


def test_attention_reports_bad_lists_and_leaves_the_other_sequences_alone():
    pi = context(budget_blocks=16)
    case = attention_case(pi, [250, 250, 250, 250], 8)
    good, _ = run_attention(pi, case)
    case["count"][1] = 17
    case["slots"][2, 3] = 24
    case["slots"][3, 2], case["blocks"][3, 2] = -1, -1                                 # an entry that names nothing is skipped silently
    out = torch.zeros((4, 8, 128), dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros((4, 8), dtype=torch.float32, device=DEV)
    pi.sparse_decode_attn_kv8(0, bf(case["q"]), dev(case["pool"]), dev(case["slots"]), dev(case["blocks"]), dev(case["count"]), i32(case["ctx"]), out, lse)
    torch.cuda.synchronize()
    assert pi.status()[0] in (-8, -9) and pi.status()[1] == 4
    pi.clear_status()
    assert torch.equal(out[0], good[0]) and (out[1] == 0).all() and (lse[1] == -float("inf")).all()
    case["count"][1] = 0
    case["blocks"][2, 3] = -1                                                          # what the kernel skipped, the reference skips
    check_attention(pi, case, out, lse)
    # NaN in one sequence's cache stays in that sequence, and in V in its channel
    case = attention_case(pi, [250, 250], 9)
    ref.parts(case["pool"][1, case["slots"][1, 0]], 2, 16)[0][0, 1, 0, 77] = 127
    out, _ = run_attention(pi, case)
    bad = torch.isnan(out.float())
    assert not bad[0].any() and bad[1, :4, 77].all() and int(bad[1].sum()) == 4
    pi.close()


def test_attention_takes_a_list_as_it_is():
    """Entries behind the count are not looked at, a block named twice counts twice, a block behind the context not at all;
    a head whose query is not a number leaves the others alone."""
    pi = context(n_q_heads=8, n_kv_heads=2, budget_blocks=16)
    case = attention_case(pi, [250, 250, 100, 250], 21)
    case["blocks"][0, 3], case["slots"][0, 3] = case["blocks"][0, 4], case["slots"][0, 4]
    case["blocks"][1, 2] = 200                                                         # far behind the context
    case["count"][3] = 5
    case["blocks"][3, 5:], case["slots"][3, 5:] = 123456, -77
    out, lse = run_attention(pi, case)
    check_attention(pi, case, out, lse)
    before = out.clone()
    q = case["q"].copy()
    case["q"][:, 5, 17] = np.nan
    out, lse = run_attention(pi, case)
    keep = [g for g in range(8) if g != 5]
    assert torch.equal(out[:, keep], before[:, keep]) and torch.isnan(out[:, 5].float()).all() and torch.isnan(lse[:, 5]).all()
    case["q"] = q
    case["pool"][:] = 0                                                                # a pool that was never written: all values zero
    out, lse = run_attention(pi, case)
    check_attention(pi, case, out, lse)
    assert (out == 0).all()
    pi.close()


def test_attention_with_pool_offsets_beyond_32_bits():
    pi = context(n_q_heads=16, n_kv_heads=16, block_tokens=64, budget_blocks=4, pool_slots=8192, max_batch=4)
    small = attention_case(context(n_q_heads=16, n_kv_heads=16, block_tokens=64, budget_blocks=4, pool_slots=8, max_batch=4), [250, 3, 256, 200], 4)
    pool = torch.zeros((4, 8192, pi.kv8_block_bytes), dtype=torch.uint8, device=DEV)   # 8.6 GB
    far = np.asarray([8191, 5000, 8000, 1, 8190, 4096, 77, 3000])
    pool[:, torch.from_numpy(far).to(DEV)] = dev(small["pool"])
    slots = np.where(small["slots"] >= 0, far[np.maximum(small["slots"], 0)], -1).astype(np.int32)
    out, lse = torch.zeros((4, 16, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((4, 16), device=DEV)
    pi.sparse_decode_attn_kv8(0, bf(small["q"]), pool, dev(slots), dev(small["blocks"]), dev(small["count"]), i32(small["ctx"]), out, lse)
    clean(pi)
    check_attention(pi, small, out, lse)
    pi.close()


def test_attention_on_two_streams_at_once_and_in_a_replayed_graph():
    pi = context(n_q_heads=32, n_kv_heads=8, budget_blocks=64, pool_slots=70, max_batch=4)
    cases = [attention_case(pi, [1000, 37, 1024], s) for s in (1, 2)]
    want = [run_attention(pi, c)[0].clone() for c in cases]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    args = [[bf(c["q"]), dev(c["pool"]), dev(c["slots"]), dev(c["blocks"]), dev(c["count"]), i32(c["ctx"])] for c in cases]
    outs = [torch.zeros((3, 32, 128), dtype=torch.bfloat16, device=DEV) for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for a, o, s in zip(args, outs, streams):
            pi.sparse_decode_attn_kv8(0, *a, o, stream=s)
    clean(pi)
    for o, w in zip(outs, want):
        assert torch.equal(o, w)
    static = [t.clone() for t in args[0]]
    out = torch.zeros_like(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pi.sparse_decode_attn_kv8(0, *static, out)
    for a, w in zip(args, want):
        for s, t in zip(static, a):
            s.copy_(t)
        graph.replay()
        clean(pi)
        assert torch.equal(out, w)
    pi.close()


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("paged", [False, True])
def test_a_session_in_8_bits_with_appends_eager_and_replayed(paged):
    """Two layers, four steps with appends: eager and graph-replayed sessions agree bit for bit, every layer's attention is
    what the reference makes of the session's own lists and pool, and pool and host store agree on every resident block."""
    from paper_2609_34555_b200 import PulseInfer
    from paper_2609_34555_b200.runner import DecodeSession
    from workloads import generate as gen, tiny_config
    cfg = tiny_config(batch=3, ctx=1200, n_layers=2, n_q_heads=16, n_kv_heads=4, budget_blocks=24, resident_frac=0.4)
    lens = [1150, 700, 433]
    sessions = []
    for _ in range(2):
        pi = PulseInfer.from_workload(cfg)
        sess = DecodeSession(pi, cfg.batch, cfg.n_layers, paged=paged, kv_bits=8)
        sess.ctx_len.copy_(i32(lens))
        for l in range(cfg.n_layers):
            res = np.stack([np.pad(gen.initial_resident(cfg.replace(ctx=n, batch=1), l)[0][:cfg.pool_slots],
                                   (0, max(0, cfg.pool_slots - len(gen.initial_resident(cfg.replace(ctx=n, batch=1), l)[0]))), constant_values=-1) for n in lens])
            sess.load_layer(l, gen.make_kv(cfg, l, device=torch.device(DEV)), i32(res))
        torch.cuda.synchronize()
        sessions.append((pi, sess))
    g = torch.Generator().manual_seed(1)
    qs = [torch.randn((2, 3, 16, 128), generator=g).to(torch.bfloat16).to(DEV) for _ in range(4)]
    new = [tuple((torch.randn((2, 3, 4, 128), generator=g) * 4 ** i).to(torch.bfloat16).to(DEV) for _ in range(2)) for i in range(4)]
    (pi, sess), (pi2, sess2) = sessions
    q_static, kv_static = torch.empty_like(qs[0]), tuple(torch.empty_like(t) for t in new[0])
    graph = sess2.capture_step(q_static, new_kv_static=kv_static)
    misses = 0
    for step in range(4):
        out = sess.decode_step(qs[step], new_kv=new[step]).clone()
        q_static.copy_(qs[step]); kv_static[0].copy_(new[step][0]); kv_static[1].copy_(new[step][1])
        sess2.replay_step(graph)
        clean(pi)
        clean(pi2)
        assert torch.equal(out, sess2.out)
        misses += sess.miss_blocks()
        for l in range(2):
            b = sess.bufs[l]
            case = dict(pool=b.pool.cpu().numpy(), blocks=b.sel_blocks.cpu().numpy(), slots=b.sel_slots.cpu().numpy(), count=b.sel_count.cpu().numpy(),
                        ctx=sess.ctx_len.cpu().numpy(), q=qs[step][l].float().cpu().numpy())
            check_attention(pi, case, out[l], None)
            host = sess.logical_host(l).numpy()
            table = b.block_table.cpu().numpy()
            for s in range(3):
                for blk in np.nonzero(table[s] >= 0)[0]:
                    assert np.array_equal(case["pool"][s, table[s, blk]], host[s, blk]), (step, l, s, blk)
    assert misses > 0
    with pytest.raises(ValueError):
        DecodeSession(pi, 3, 2, kv_bits=8, split_attention=True)
    with pytest.raises(ValueError):
        DecodeSession(pi, 3, 2, kv_bits=6)
    pi.close()
    pi2.close()


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_prompts_into_a_session_and_a_decode_step_over_them(bits):
    """Prompts of different lengths (none, a token, more than the pool holds): their attention, the cache that they leave, and the next token's
    attention over the whole of it, which is one more row of the prompt's attention but for the cache's rounding."""
    from paper_2609_34555_b200.runner import DecodeSession
    lens = [70, 0, 1, 130]
    pi = context(n_q_heads=8, n_kv_heads=2, budget_blocks=10, pool_slots=10, max_blocks=12, max_batch=4, n_sink_blocks=1, n_local_blocks=2, n_layers=2)
    sess = DecodeSession(pi, 4, 2, kv_bits=bits)
    g = torch.Generator().manual_seed(bits)
    T = sum(lens) + 4                                                                  # and padding behind the last prompt
    starts = i32(np.concatenate(([0], np.cumsum(lens))))
    layers = []
    for l in range(2):
        q, k, v = ((torch.randn((T, h, 128), generator=g) * s).to(torch.bfloat16).to(DEV) for h, s in ((8, 1.0), (2, 1.0), (2, 3.0)))
        out, lse = torch.full((T, 8, 128), 3.0, dtype=torch.bfloat16, device=DEV), torch.zeros((T, 8), device=DEV)
        sess.load_prompts(l, q, k, v, starts, out, lse)
        clean(pi)
        assert (out[-4:] == 3).all() and sess.ctx_len.tolist() == lens
        layers.append((q, k, v, out, lse))
    step_q = torch.stack([torch.stack([q[max(0, int(e) - 1)] for e in starts[1:]]) for q, *_ in layers])      # the last token's query once more
    got = sess.decode_step(step_q)
    clean(pi)
    for l, (q, k, v, out, lse) in enumerate(layers):
        for s, n in enumerate(lens):
            if n == 0:
                assert (got[l, s] == 0).all()
                continue
            last = out[int(starts[s + 1]) - 1].float()
            # (weights of a cache in few bits are off by the keys' rounding: 2^-5 of a score of a few units, and half a step of 4 bits, 1 / 30 of a spread of about 6)
            tol = {16: 0.05, 8: 0.5, 4: 1.0}[bits]
            assert float((got[l, s].float() - last).abs().max()) <= tol, (l, s)
        b = sess.bufs[l]
        assert b.slot_block[0].tolist()[:5] == [0, 1, 2, 3, 4] and b.slot_block[3].tolist() == [0, 1, 2, 3, 4, 5, 6, 7, 8, -1]
    with pytest.raises(ValueError):
        sess.load_prompts(0, q, k, v, starts[:-1], out)
    pi.close()


def test_prompt_to_attention_through_pages_rotation_prompt_attention_store_recall():
    """A ragged batch of prompts: pages, norm + rotation, attention over the prompts, store into an arena, recall into a pool, attention of
    the last token over everything, against the chain in 64 bits."""
    from tests.prompt_reference import check, reference
    pi = context(n_q_heads=8, n_kv_heads=2, budget_blocks=16, pool_slots=16, max_blocks=16, max_batch=4, n_sink_blocks=1, n_local_blocks=1)
    lens = np.asarray([100, 1, 0, 256])
    rng = np.random.default_rng(12)
    cap = int(lens.sum()) + 11
    table = torch.full((4, 16), -1, dtype=torch.int32, device=DEV)
    ring, counters = pi.free_page_ring(40)
    ring.copy_(dev(rng.permutation(40).astype(np.int32)))
    slots, pos, starts = torch.empty(cap, dtype=torch.int64, device=DEV), torch.empty(cap, dtype=torch.int32, device=DEV), torch.empty(5, dtype=torch.int32, device=DEV)
    pi.assign_pages(i32([0] * 4), i32(lens), table, ring, counters, token_start=starts, slot_map=slots, positions=pos)
    qkv = bf(rng.standard_normal((cap, 12 * 128)))
    q, k, v = qkv[:, :1024].unflatten(1, (8, 128)), qkv[:, 1024:1280].unflatten(1, (2, 128)), qkv[:, 1280:].unflatten(1, (2, 128))
    freq = (1e4 ** (-np.arange(0, 128, 2) / 128)).astype(np.float32)
    qo, ko = torch.zeros((cap, 8, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((cap, 2, 128), dtype=torch.bfloat16, device=DEV)
    pi.qk_norm_rope(q, k, pos, dev(freq), qo, ko)
    out, lse = torch.full((cap, 8, 128), 3.0, dtype=torch.bfloat16, device=DEV), torch.zeros((cap, 8), device=DEV)
    pi.prompt_attn(qo, ko, v, starts, out, lse=lse)                                    # the starts that the pages came with
    arena = torch.zeros((40, pi.kv8_block_bytes), dtype=torch.uint8).pin_memory()
    pi.kv8_store(ko, v, arena, slots)
    nb = -(-lens // 16)
    lists = np.zeros((4, 16, 4), dtype=np.int32)
    for s in range(4):
        lists[s, 0] = [0, 0, nb[s], 0]
    pool = torch.zeros((4, 16, pi.kv8_block_bytes), dtype=torch.uint8, device=DEV)
    pi.recall_kv8(0, arena, pool, dev(lists), i32((nb > 0).astype(np.int32)), page_table=table)
    sel = np.where(np.arange(16)[None] < nb[:, None], np.arange(16)[None], -1).astype(np.int32)
    begin = np.concatenate(([0], np.cumsum(lens)))
    qd = qo[torch.from_numpy(np.maximum(begin[1:] - 1, 0)).to(DEV)].contiguous()
    o1, l1 = torch.zeros((4, 8, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((4, 8), device=DEV)
    pi.sparse_decode_attn_kv8(0, qd, pool, dev(sel), dev(sel), i32(nb), i32(lens), o1, l1)
    clean(pi)
    assert starts.tolist() == begin.tolist() and (out[int(begin[-1]):] == 3).all()
    check(torch.bfloat16, out, lse, reference(qo, ko, v, begin.tolist(), begin.tolist()))
    kb, vb = ko.float().cpu().numpy(), v.float().cpu().numpy()
    pools = np.zeros((4, 16, pi.kv8_block_bytes), dtype=np.uint8)
    for s in range(4):
        ref.store(pools[s], kb[begin[s]:begin[s + 1]], vb[begin[s]:begin[s + 1]], range(lens[s]), 16)
    assert np.array_equal(pool.cpu().numpy(), pools)
    check_attention(pi, dict(pool=pools, blocks=sel, slots=sel, count=nb, ctx=lens, q=qd.float().cpu().numpy()), o1, l1)
    pi.close()


@pytest.mark.parametrize("nats", [5.0, 14.0, 17.0])
@pytest.mark.parametrize("Hq,B,K,at", [(4, 64, 1024, 0), (4, 64, 1024, 40000), (16, 64, 1024, 70), (8, 32, 1000, 31999)])
def test_a_long_tail_under_one_large_score(Hq, B, K, at, nats):
    """One key far above all others, of value 0: the result is what the others' small weights make of it.  The products' weights are counted 2^7
    times as large as under their reference, the largest weight times scale at most: each is off by half a step (2^-11 of itself) or by
    2^-25-7 of the reference, times a number of up to 2^8 that is twice its block's largest value over its scale at most."""
    pi = context(n_q_heads=Hq, n_kv_heads=1, block_tokens=B, budget_blocks=K, pool_slots=K, max_blocks=K, max_batch=1)
    rng = np.random.default_rng(Hq + B)
    kv = rng.standard_normal((K, 1, 2, B, 128)) * np.asarray([0.1, 1.0])[:, None, None]
    kv[:, :, 1] += 2
    kv[:, :, 0, :, 0] = 0
    kv[at // B, 0, 0, at % B, 0], kv[at // B, 0, 1, at % B] = nats, 0
    pool = ref.pack(ref.bf16(kv), B)[None]
    q = ref.bf16(rng.standard_normal((1, Hq, 128)))
    q[..., 0] = ref.bf16(np.float64(128 ** 0.5))
    order = np.arange(K, dtype=np.int32)[None]
    case = dict(pool=pool, blocks=order, slots=order, count=np.asarray([K], dtype=np.int32), ctx=np.asarray([K * B]), q=q)
    out, lse = run_attention(pi, case)
    check_attention(pi, case, out, lse)
    k, v = (x.reshape(K * B, 128) for x in np.moveaxis(ref.unpack(pool[0], 1, B)[:, 0], 1, 0))
    top = np.repeat(np.abs(v).reshape(K, B * 128).max(1), B)
    for g in range(Hq):
        z = k @ q[0, g].astype(np.float64) / np.sqrt(128)
        w = np.exp(z - z.max())
        w /= w.sum()
        eps = (8 * 2.0 ** -23 * (np.abs(k) @ np.abs(q[0, g].astype(np.float64))).max() + 4 * 2.0 ** -24 * np.abs(z).max() * np.sqrt(128)) / np.sqrt(128)
        want, spread = w @ v, w @ np.abs(v)
        tol = 2.0 ** -8 * np.abs(want) + (2 * eps + 2.0 ** -11 + 2.0 ** -20) * spread + K * B * 2.0 ** -31 * (w * top).max()
        over = (np.abs(out[0, g].double().cpu().numpy() - want) / tol).max()
        assert over <= 1, over
    pi.close()


@pytest.mark.parametrize("Hq,Hkv", [(64, 16), (128, 8)])
@pytest.mark.parametrize("nats", [14.0, 17.0])
def test_a_long_tail_under_one_large_score_in_many_sequences(Hq, Hkv, nats):
    """As above, with so many sequences that four warps have all tokens of one: a fourth of the tail is counted from the large score's reference."""
    n, K, B = 13, 16, 64
    pi = context(n_q_heads=Hq, n_kv_heads=Hkv, block_tokens=B, budget_blocks=K, pool_slots=K, max_blocks=K, max_batch=n)
    rng = np.random.default_rng(Hq)
    kv = rng.standard_normal((K, Hkv, 2, B, 128)) * np.asarray([0.1, 1.0])[:, None, None]
    kv[:, :, 1] += 2
    kv[:, :, 0, :, 0] = 0
    kv[3, :, 0, 20, 0], kv[3, :, 1, 20] = nats, 0
    pool = ref.pack(ref.bf16(kv), B)
    q = ref.bf16(rng.standard_normal((1, Hq, 128)))
    q[..., 0] = ref.bf16(np.float64(128 ** 0.5))
    order = np.tile(np.arange(K, dtype=np.int32), (n, 1))
    case = dict(pool=np.tile(pool, (n, 1, 1)), blocks=order, slots=order, count=np.full(n, K, dtype=np.int32), ctx=np.full(n, K * B), q=np.tile(q, (n, 1, 1)))
    out, lse = run_attention(pi, case)
    assert torch.equal(out, out[:1].expand_as(out)) and torch.equal(lse, lse[:1].expand_as(lse))
    values = ref.unpack(pool, Hkv, B)
    for g in range(Hq):
        k, v = (values[:, g * Hkv // Hq, i].reshape(K * B, 128) for i in (0, 1))
        top = np.repeat(np.abs(v).reshape(K, B * 128).max(1), B)
        z = k @ q[0, g].astype(np.float64) / np.sqrt(128)
        w = np.exp(z - z.max())
        w /= w.sum()
        eps = (8 * 2.0 ** -23 * (np.abs(k) @ np.abs(q[0, g].astype(np.float64))).max() + 4 * 2.0 ** -24 * np.abs(z).max() * np.sqrt(128)) / np.sqrt(128)
        want, spread = w @ v, w @ np.abs(v)
        tol = 2.0 ** -8 * np.abs(want) + (2 * eps + 2.0 ** -11 + 2.0 ** -20) * spread + K * B * 2.0 ** -31 * (w * top).max()
        over = (np.abs(out[0, g].double().cpu().numpy() - want) / tol).max()
        assert over <= 1, over
    pi.close()


@pytest.mark.parametrize("slots,first,run,block", [
    (list(range(10)) + [-1] + list(range(11, 20)), 0, 10, 0),                          # a token skipped inside a block
    ([64, 65, 0, 1, 66], 0, 2, 2),                                                     # a block that comes back behind another one
    ([32, 33, 34, 34, 34, 35] + [36] * 30, 0, 32, 1),                                  # more tokens than a block has
])
def test_store_reports_a_block_that_comes_back(slots, first, run, block):
    pi = context(n_q_heads=2, n_kv_heads=2, block_tokens=32)
    rng = np.random.default_rng(9)
    k, v = tokens_of(rng, len(slots), 2)
    store = torch.zeros((4, pi.kv8_block_bytes), dtype=torch.uint8, device=DEV)
    pi.kv8_store(bf(k), bf(v), store, dev(np.asarray(slots, dtype=np.int64)))
    assert clean(pi, -8)[1:5] == [6, first, run, block]
    rest = [b for b in range(4) if b not in {s // 32 for s in slots if s >= 0}]
    assert int(store[rest].sum()) == 0
    pi.close()


@pytest.mark.parametrize("block", [16, 32, 64])
def test_store_reports_nothing_of_maps_in_order(block):
    """Runs that begin and end anywhere, skipped tokens between blocks, single tokens of many blocks."""
    pi = context(n_q_heads=2, n_kv_heads=2, block_tokens=block)
    rng = np.random.default_rng(block)
    for _ in range(30):
        order, slots = rng.permutation(40), []
        for b in order[:rng.integers(1, 40)]:
            a = rng.integers(0, block)
            slots += list(b * block + np.arange(a, a + rng.integers(1, block - a + 1)) % block) + [-1] * rng.integers(0, 3)
        k, v = tokens_of(rng, len(slots), 2)
        store = torch.zeros((40, pi.kv8_block_bytes), dtype=torch.uint8, device=DEV)
        want = store.cpu().numpy()
        pi.kv8_store(bf(k), bf(v), store, dev(np.asarray(slots, dtype=np.int64)))
        clean(pi)
        ref.store(want, k, v, np.asarray(slots, dtype=np.int64), block)
        assert np.array_equal(store.cpu().numpy(), want)
    pi.close()
