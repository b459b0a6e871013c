"""The 4-bit cache and the calls around it on the GPU, against the plain references of kv4_reference."""
import numpy as np
import pytest
import torch

from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def context(**kw):
    from paper_2609_34555_b200 import PulseInfer
    base = dict(n_layers=1, n_q_heads=8, n_kv_heads=2, block_tokens=16, budget_blocks=16, n_sink_blocks=1, n_local_blocks=2,
                pool_slots=24, max_batch=8, max_blocks=256, solo_head=[0])
    base.update(kw)
    base["solo_head"] = (list(base["solo_head"]) * base["n_layers"])[:base["n_layers"]]
    return PulseInfer(**base)


def bf(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).to(DEV)


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    return t if dtype is None else t.to(dtype)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def clean(pi, code=0):
    torch.cuda.synchronize()
    got = pi.status()
    assert got[0] == code, got
    pi.clear_status()
    return got


# ------------------------------------------------------------------ store and load
@pytest.mark.parametrize("heads,block", [(1, 16), (2, 32), (4, 16), (8, 16), (8, 64), (16, 32)])
@pytest.mark.parametrize("tokens", [1, 7, 130])
def test_store_writes_the_reference_bytes_and_nothing_else(heads, block, tokens):
    pi = context(n_q_heads=heads, n_kv_heads=heads, block_tokens=block)
    rng = np.random.default_rng(heads * 1000 + block + tokens)
    pages = -(-tokens // block) + 2
    kv = ref.bf16(rng.standard_normal((tokens, 2, heads, 128)) * np.exp(rng.standard_normal((tokens, 1, heads, 1)) * 3))
    if tokens > 5:
        kv[0, :, :, 32:64] = -1.5                                                      # a group without spread
        kv[1, 0, 0, :32] = np.float32(1e-39)                                           # subnormal
        kv[2, 1, 0, 64:96] *= np.float32(2.0 ** 90)
        kv[3, 0, :, 5] = np.nan
        kv[4, 1, :, 99] = np.inf
        kv = ref.bf16(kv)
    slots = rng.permutation(pages * block)[:tokens].astype(np.int64)
    if tokens > 5:
        slots[5] = -1
    before = rng.integers(0, 256, (pages, pi.kv4_block_bytes), dtype=np.uint8)
    want = before.copy()
    for t in range(tokens):
        if slots[t] >= 0:
            ref.write_token(want, int(slots[t]), kv[t, 0], kv[t, 1], block)
    fused = bf(kv.reshape(tokens, -1))                                                 # K and V of a token side by side
    k, v = fused[:, :heads * 128].unflatten(1, (heads, 128)), fused[:, heads * 128:].unflatten(1, (heads, 128))
    store = dev(before)
    pi.kv4_store(k, v, store, dev(slots))
    clean(pi)
    got = store.cpu().numpy()
    if tokens > 5:                                                                     # NaN has many patterns: those rows' scales as values
        a, b = ref.unpack(got, heads, block), ref.unpack(want, heads, block)
        assert np.array_equal(a, b, equal_nan=True)
        for t in (3, 4):
            page, at = divmod(int(slots[t]), block)
            for x in (2048, 2304):
                for h in range(heads):
                    first = (h * (block // 16) + at // 16) * ref.TILE + x + at % 16 * 16
                    want[page, first:first + 16] = got[page, first:first + 16]
    assert np.array_equal(got, want)
    pi.close()


def test_store_of_runs_of_tokens_equals_store_token_by_token_and_a_pinned_store():
    pi = context(n_q_heads=4, n_kv_heads=4, block_tokens=32)
    rng = np.random.default_rng(5)
    kv = ref.bf16(rng.standard_normal((6, 4, 2, 32, 128)))
    want = ref.pack(kv, 32)
    blocks = bf(kv)
    rows = blocks.transpose(1, 3)                                                      # [block][token][K, V][head][128]
    out = torch.zeros((6, pi.kv4_block_bytes), dtype=torch.uint8, device=DEV)
    pi.kv4_store(rows[:, :, 0], rows[:, :, 1], out)
    pinned = torch.zeros((6, pi.kv4_block_bytes), dtype=torch.uint8).pin_memory()
    pi.kv4_store(rows[:, :, 0], rows[:, :, 1], pinned)
    clean(pi)
    assert np.array_equal(out.cpu().numpy(), want) and np.array_equal(pinned.numpy(), want)
    back = torch.zeros((6, 4, 2, 32, 128), dtype=torch.bfloat16, device=DEV)
    pi.kv4_load(pinned, back)
    clean(pi)
    assert np.array_equal(back.float().cpu().numpy(), ref.bf16(ref.unpack(want, 4, 32)))
    pi.kv4_store(rows[:0, :, 0], rows[:0, :, 1], out)                                  # no token at all
    clean(pi)
    pi.close()


def test_the_front_end_checks_devices_types_and_shapes():
    """Every tensor argument of the calls, one wrong at a time: refused before anything runs, and the call still works afterwards."""
    import paper_2609_34555_b200 as pkg
    pi = context()
    n, H, B, C, NB, K = 4, 2, 16, 24, 256, 16
    z = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype, device=DEV)          # noqa: E731
    bfz = lambda *shape: z(*shape, dtype=torch.bfloat16)                                       # noqa: E731
    pool, host = z(n, C, pi.kv4_block_bytes, dtype=torch.uint8), z(n, NB, pi.kv4_block_bytes, dtype=torch.uint8)
    calls = {
        "assign_pages": dict(old_len=z(n), new_len=z(n), page_table=z(n, NB), free_pages=z(50), free_state=torch.tensor([0, 50, 0, 0], device=DEV),
                             token_start=z(n + 1), slot_map=z(8, dtype=torch.int64), positions=z(8)),
        "qk_norm_rope": dict(q=bfz(n, 8, 128), k=bfz(n, H, 128), positions=z(n), inv_freq=z(64, dtype=torch.float32), q_out=bfz(n, 8, 128), k_out=bfz(n, H, 128),
                             q_weight=z(128, dtype=torch.float32), k_weight=z(128, dtype=torch.float32)),
        "kv4_store": dict(k=bfz(n, H, 128), v=bfz(n, H, 128), store=host, slot_map=z(n, dtype=torch.int64)),
        "kv4_load": dict(store=host, out=bfz(n, H, 2, B, 128), blocks=z(n)),
        "append_kv4": dict(layer=0, step=z(1) + 1, k_new=bfz(n, H, 128), v_new=bfz(n, H, 128), ctx_len=z(n), host_kv4=host, pool4=pool, block_table=z(n, NB) - 1,
                           slot_block=z(n, C) - 1, slot_stamp=z(n, C), digest=bfz(n, NB, 2, 128), page_table=z(n, NB)),
        "recall_kv4": dict(layer=0, host_kv4=host, pool4=pool, recall_list=z(n, K, 4), recall_count=z(n), page_table=z(n, NB)),
        "sparse_decode_attn_kv4": dict(layer=0, q=bfz(n, 8, 128), pool4=pool, sel_slots=z(n, K), sel_blocks=z(n, K), sel_count=z(n), ctx_len=z(n), out=bfz(n, 8, 128),
                                       lse=z(n, 8, dtype=torch.float32)),
    }
    for name, good in calls.items():
        call = getattr(pi, name)
        call(**good)
        clean(pi)
        for arg, t in good.items():
            if not isinstance(t, torch.Tensor):
                continue
            wrong = [t.to(torch.float64), t.cpu() if arg not in ("host_kv4", "store") else t[..., 16:], t.repeat_interleave(2, -1)[..., ::2]]
            if not (name, arg) in (("qk_norm_rope", "inv_freq"), ("kv4_load", "blocks"), ("assign_pages", "free_pages"), ("append_kv4", "step")):
                # (of the tables only the number of values is asked for)
                wrong.append(t[:1] if arg in ("block_table", "slot_block", "slot_stamp", "digest") else t[..., None].contiguous())
            if (name, arg) in (("kv4_store", "k"), ("kv4_store", "v"), ("qk_norm_rope", "q"), ("qk_norm_rope", "k")):
                wrong[2] = t.repeat_interleave(2, -1)[..., ::2]                                  # rows not contiguous
            for bad in wrong:
                if t.numel() == 1 and bad.is_cuda and bad.dtype == t.dtype:
                    continue
                with pytest.raises((TypeError, ValueError, pkg.PiError)):
                    call(**dict(good, **{arg: bad}))
        call(**good)
        clean(pi)
    with pytest.raises(pkg.PiError):
        pi.append_kv4(**dict(calls["append_kv4"], step=0))
    with pytest.raises(pkg.PiError):
        pi.append_kv4(**dict(calls["append_kv4"], layer=1))
    with pytest.raises(pkg.PiError):
        pi.qk_norm_rope(**dict(calls["qk_norm_rope"], k_weight=None))
    with pytest.raises(pkg.PiError) as e:
        pi.kv4_load(torch.zeros((n, pi.kv4_block_bytes), dtype=torch.uint8), calls["kv4_load"]["out"])
    assert e.value.code == -5                                                                    # not pinned
    pi.close()
    with pytest.raises(pkg.PiError):
        pi.kv4_load(**calls["kv4_load"])                                                         # a closed context


def test_store_skips_and_reports_a_slot_beyond_the_store():
    pi = context()
    rng = np.random.default_rng(6)
    kv = ref.bf16(rng.standard_normal((20, 2, 2, 128)))
    slots = np.arange(20, dtype=np.int64)
    slots[7], slots[8] = 32, (1 << 40)                                                 # the store has 32 slots
    want = np.zeros((2, pi.kv4_block_bytes), dtype=np.uint8)
    for t in range(20):
        if slots[t] < 32:
            ref.write_token(want, int(slots[t]), kv[t, 0], kv[t, 1], 16)
    whole = torch.zeros((4, pi.kv4_block_bytes), dtype=torch.uint8, device=DEV)
    pi.kv4_store(bf(kv[:, 0]), bf(kv[:, 1]), whole[1:3], dev(slots))
    got = clean(pi, -8)
    assert got[1] == 6 and got[2] in (7, 8)
    assert np.array_equal(whole[1:3].cpu().numpy(), want) and int(whole[0].sum()) == 0 and int(whole[3].sum()) == 0
    pi.close()


@pytest.mark.parametrize("heads,block", [(1, 16), (8, 16), (2, 64), (16, 32)])
def test_load_gives_the_values_rounded_once(heads, block):
    pi = context(n_q_heads=heads, n_kv_heads=heads, block_tokens=block)
    rng = np.random.default_rng(heads + block)
    packed = ref.pack(ref.bf16(rng.standard_normal((5, heads, 2, block, 128)) * 4), block)
    store = dev(packed)
    want = ref.bf16(ref.unpack(packed, heads, block))
    out = torch.zeros((5, heads, 2, block, 128), dtype=torch.bfloat16, device=DEV)
    pi.kv4_load(store, out)
    clean(pi)
    # scale * code + minimum is rounded to 32 bits and then to bf16: twice, so a value next to a border may go to its other side
    got = out.float().cpu().numpy()
    assert (np.abs(got - want) <= 2.0 ** -7 * np.abs(want)).all() and (got != want).mean() < 1e-3
    out = torch.full((4, heads, 2, block, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    pi.kv4_load(store, out, i32([4, 5, -1, 0]))
    got = clean(pi, -8)
    assert got[1] == 6 and got[2] in (1, 2)
    o = out.float().cpu().numpy()
    assert (np.abs(o[[0, 3]] - want[[4, 0]]) <= 2.0 ** -7 * np.abs(want[[4, 0]])).all() and (o[1:3] == 7).all()
    pi.close()


# ------------------------------------------------------------------ norm and rotation
ROPE_CASES = [(1, 8, 2, "bf16", 128, False, True), (5, 8, 2, "fp16", 128, True, True), (33, 32, 8, "fp32", 64, False, True), (3, 1, 1, "bf16", 2, False, False),
              (7, 5, 1, "bf16", 96, False, True), (7, 5, 1, "fp32", 96, True, False), (130, 12, 4, "fp16", 32, False, False), (4, 16, 16, "bf16", 128, False, False),
              (2, 8, 8, "bf16", 0, False, True), (700, 32, 8, "bf16", 128, False, True), (3000, 4, 1, "fp32", 128, True, True)]


@pytest.mark.parametrize("T,Hq,Hkv,dtype,rot,inter,norm", ROPE_CASES)
@pytest.mark.parametrize("fused", [False, True])
def test_norm_and_rotation(T, Hq, Hkv, dtype, rot, inter, norm, fused):
    pi = context(n_q_heads=Hq, n_kv_heads=Hkv)
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[dtype]
    g = torch.Generator().manual_seed(T + rot)
    x = (torch.randn((T, (Hq + 2 * Hkv) * 128), generator=g) * 2).to(dt)
    x[0, :128] *= 1e-3
    xd = x.to(DEV)
    q, k = xd[:, :Hq * 128].unflatten(1, (Hq, 128)), xd[:, Hq * 128:(Hq + Hkv) * 128].unflatten(1, (Hkv, 128))
    if not fused:
        q, k = q.contiguous(), k.contiguous()
    pos = np.random.default_rng(T).integers(0, 1 << 20, T).astype(np.int32)
    pos[0] = 2 ** 31 - 1 if T > 1 else 131071
    if T > 4:
        pos[3] = 0
        pos[T - 2:] = -1                                                               # padding
    freq = (500000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)
    wq, wk = (1 + 0.3 * np.random.default_rng(9).standard_normal((2, 128)).astype(np.float32)) if norm else (None, None)
    qo = torch.full((T + 1, Hq, 128), 5.0, dtype=torch.bfloat16, device=DEV)
    ko = torch.full((T + 1, Hkv, 128), 5.0, dtype=torch.bfloat16, device=DEV)
    pi.qk_norm_rope(q, k, i32(pos), dev(freq) if rot else None, qo[:T], ko[:T], q_weight=None if wq is None else dev(wq),
                    k_weight=None if wk is None else dev(wk), eps=1e-5, interleaved=inter)
    clean(pi)
    for got, src, w in ((qo, q, wq), (ko, k, wk)):
        got = got.float().cpu().numpy().astype(np.float64)
        want = ref.rope(src.double().cpu().numpy(), pos, freq, w, 1e-5, inter)
        assert (got[T] == 5).all()
        live = pos >= 0
        assert (got[:T][~live] == 5).all()
        # one rounding to bf16 (2^-8 of the value); in 32 bits before it: the norm (a sum of 128 squares, its root, two
        # products: under 2^-20 of the value) and the turn (angles off by 2^-23 of a turn: under 2^-20 of the pair's length)
        length = np.abs(want).max(-1, keepdims=True) * np.sqrt(2)
        tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * length + 1e-30
        bad = np.abs(got[:T] - want) > tol
        assert not bad[live].any()
    pi.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
def test_rotation_of_any_part_of_the_channels(dtype, inter):
    """Every even rot_dim; infinities and NaN behind the turned channels stay where they are."""
    pi = context(n_q_heads=6, n_kv_heads=2)
    g = torch.Generator().manual_seed(17)
    T = 9
    q, k = [(torch.randn((T, h, 128), generator=g) * 2).to(dtype).to(DEV) for h in (6, 2)]
    pos = np.random.default_rng(3).integers(0, 1 << 17, T).astype(np.int32)
    for rot in range(0, 129, 2):
        freq = (10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)
        a, b = q.clone(), k.clone()
        if rot < 128:
            a[1, :, rot:] = torch.inf
            a[2, :, 127] = torch.nan
            b[3, 0, rot] = -torch.inf
        qo, ko = torch.full_like(q, 5.0, dtype=torch.bfloat16), torch.full_like(k, 5.0, dtype=torch.bfloat16)
        pi.qk_norm_rope(a, b, i32(pos), dev(freq) if rot else None, qo, ko, interleaved=inter)
        clean(pi)
        for got, src, x in ((qo, a, q), (ko, b, k)):
            got, src = got.double().cpu().numpy(), src.double().cpu().numpy()
            want = ref.rope(x.double().cpu().numpy(), pos, freq, None, 0.0, inter)
            want[..., rot:] = src[..., rot:]
            # as above: one rounding to bf16, and under 2^-19 of the pair's length before it
            tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * np.abs(x.double().cpu().numpy()).max() * np.sqrt(2)
            same = (got == want) | (np.isnan(got) & np.isnan(want))
            with np.errstate(invalid="ignore"):
                assert (same | (np.abs(got - want) <= tol)).all(), rot
    pi.close()


def test_norm_and_rotation_in_place_and_far_rows_of_a_fused_projection():
    pi = context(n_q_heads=8, n_kv_heads=2)
    g = torch.Generator().manual_seed(3)
    q, k = torch.randn((50, 8, 128), generator=g).to(torch.bfloat16).to(DEV), torch.randn((50, 2, 128), generator=g).to(torch.bfloat16).to(DEV)
    pos, freq, w = i32(np.arange(50)), dev((1e4 ** (-np.arange(0, 128, 2) / 128)).astype(np.float32)), torch.ones(128, device=DEV)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    pi.qk_norm_rope(q, k, pos, freq, qo, ko, q_weight=w, k_weight=w)
    pi.qk_norm_rope(q, k, pos, freq, q, k, q_weight=w, k_weight=w)
    clean(pi)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    # rows more than 2^31 elements apart
    big = torch.zeros((3, (1 << 30) + 8), dtype=torch.bfloat16, device=DEV)
    big[:, :1280] = torch.randn((3, 1280), generator=g).to(torch.bfloat16).to(DEV)
    a, b = big[:, :1024].unflatten(1, (8, 128)), big[:, 1024:1280].unflatten(1, (2, 128))
    got, want = [torch.empty((3, 8, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    kk = torch.empty((3, 2, 128), dtype=torch.bfloat16, device=DEV)
    pi.qk_norm_rope(a, b, pos[:3].contiguous(), freq, got, kk)
    pi.qk_norm_rope(a.contiguous(), b.contiguous(), pos[:3].contiguous(), freq, want, kk)
    clean(pi)
    assert torch.equal(got, want)
    none = torch.empty((0, 8, 128), dtype=torch.bfloat16, device=DEV)
    pi.qk_norm_rope(none, none[:, :2], pos[:0], freq, none, none[:, :2])               # no token
    with pytest.raises(ValueError):
        pi.qk_norm_rope(q[:, :4], k, pos, freq, qo, ko)
    with pytest.raises(ValueError):
        pi.qk_norm_rope(q.transpose(0, 1).contiguous().transpose(0, 1), k, pos, freq, qo, ko)   # rows of a token apart
    with pytest.raises(TypeError):
        pi.qk_norm_rope(q.double(), k.double(), pos, freq, qo, ko)
    pi.close()


# ------------------------------------------------------------------ pages
def check_pages(pi, sim, state, old, new, capacity):
    """One call against the simulation; state = (table, ring, counters) on the device."""
    table, ring, counters = state
    batch = len(old)
    slots = torch.full((capacity,), 77, dtype=torch.int64, device=DEV)
    pos = torch.full((capacity,), 77, dtype=torch.int32, device=DEV)
    starts = torch.full((batch + 1,), 77, dtype=torch.int32, device=DEV)
    pi.assign_pages(i32(old), i32(new), table, ring, counters, starts, slots, pos)
    clean(pi)
    want_slots, want_pos, want_starts = sim.step(old, new)
    n = len(want_slots)
    assert np.array_equal(slots[:n].cpu().numpy(), want_slots) and (slots[n:] == -1).all()
    assert np.array_equal(pos[:n].cpu().numpy(), want_pos) and (pos[n:] == -1).all()
    assert np.array_equal(starts.cpu().numpy(), want_starts)
    assert np.array_equal(table.cpu().numpy(), sim.table)
    assert np.array_equal(ring.cpu().numpy(), sim.ring)
    assert counters.tolist()[:3] == sim.state[:2] + [0]


@pytest.mark.parametrize("batch,block,row,pages", [(1, 16, 5, 5), (3, 32, 40, 70), (8, 16, 256, 900), (5, 64, 7, 35), (300, 16, 16, 3000)])
def test_pages_over_many_steps_of_growing_and_shrinking_requests(batch, block, row, pages):
    pi = context(block_tokens=block, max_batch=max(8, batch), max_blocks=row)
    rng = np.random.default_rng(batch + block)
    order = rng.permutation(pages).astype(np.int32)
    table = np.full((batch, row + 3), -1, dtype=np.int32)                              # rows longer than the context's block count
    sim = ref.Pages(table, order, [0, pages, 0, 0], block)
    state = dev(table), dev(order), torch.tensor([0, pages, 0, 0], dtype=torch.int64, device=DEV)
    old = np.zeros(batch, dtype=np.int64)
    for step in range(12):
        new = old.copy()
        for s in range(batch):
            kind = rng.integers(0, 5)
            if kind == 0:
                new[s] = 0
            elif kind == 1:
                new[s] = rng.integers(0, old[s] + 1)
            elif kind == 2:
                new[s] = min(row * block, old[s] + 1)
            elif kind == 3:
                new[s] = rng.integers(old[s], row * block + 1)
        used = lambda x: int((-(-x // block)).sum())                                   # noqa: E731
        held = np.minimum(old, new)
        while used(held) + used(np.maximum(new, old)) - used(held) > pages:            # what is given back is free from the next call on
            s = int(np.argmax(new - old))
            new[s] = old[s]
        check_pages(pi, sim, state, old, new, int(np.maximum(new - old, 0).sum()) + int(rng.integers(0, 9)))
        old = new
    pi.close()


def test_pages_refuse_as_a_whole():
    pi = context(max_blocks=8)
    table = torch.full((3, 8), -1, dtype=torch.int32, device=DEV)
    ring, counters = pi.free_page_ring(10)
    zero = [0, 0, 0]
    check = (ring.clone(), counters.clone())

    def refused(old, new, code, first=None, capacity=400, counters=counters, ring=ring):
        slots = torch.full((capacity,), 77, dtype=torch.int64, device=DEV)
        starts = torch.full((4,), 77, dtype=torch.int32, device=DEV)
        was = counters.clone(), ring.clone(), table.clone()
        pi.assign_pages(i32(old), i32(new), table, ring, counters, starts, slots)
        got = clean(pi, code)
        assert got[1] == 7 and (first is None or got[2] == first)
        assert (slots == -1).all() and (starts == 0).all()
        assert torch.equal(table, was[2]) and torch.equal(ring, was[1]) and torch.equal(counters, was[0])

    refused(zero, [0, -1, 0], -8, 1)
    refused([0, 0, -5], zero, -8, 2)
    refused(zero, [129, 0, 0], -8, 0)                                                  # nine blocks in a row of eight
    refused(zero, [2 ** 31 - 1, 0, 0], -8, 0)
    refused(zero, [64, 64, 33], -4, -1)                                                # eleven pages of ten
    refused(zero, [64, 64, 0], -9, -2, capacity=127)                                   # more tokens than the maps hold
    refused([16, 0, 0], zero, -9, -1)                                                  # a page given back to a full ring
    for bad in ([-1, 10, 0, 0], [5, 4, 0, 0], [0, 11, 0, 0]):
        refused(zero, [1, 0, 0], -8, -1, counters=torch.tensor(bad, dtype=torch.int64, device=DEV))
    assert torch.equal(ring, check[0]) and torch.equal(counters, check[1])
    # a damaged ring: the page is not used
    broken = ring.clone()
    broken[1] = 10
    own = torch.tensor([0, 10, 0, 0], dtype=torch.int64, device=DEV)
    slots = torch.zeros(48, dtype=torch.int64, device=DEV)
    pi.assign_pages(i32(zero), i32([48, 0, 0]), table, broken, own, slot_map=slots)
    got = clean(pi, -8)
    assert got[1] == 7 and table[0].tolist()[:4] == [0, -1, 2, -1]
    assert slots[:16].tolist() == list(range(16)) and (slots[16:32] == -1).all() and slots[32:].tolist() == list(range(32, 48))
    pi.close()


def test_pages_with_maps_of_no_entries():
    """They hold nothing: new tokens are refused for them, and calls without new tokens run."""
    pi = context(max_blocks=8)
    table = torch.full((2, 8), -1, dtype=torch.int32, device=DEV)
    ring, counters = pi.free_page_ring(10)
    was = counters.clone(), table.clone()
    slots, positions = torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    for maps in (dict(slot_map=slots), dict(positions=positions), dict(slot_map=slots, positions=positions)):
        pi.assign_pages(i32([0, 0]), i32([0, 3]), table, ring, counters, **maps)
        assert clean(pi, -9)[2] == -2
        assert torch.equal(counters, was[0]) and torch.equal(table, was[1])
    pi.assign_pages(i32([0, 0]), i32([20, 3]), table, ring, counters)
    pi.assign_pages(i32([20, 3]), i32([16, 0]), table, ring, counters, slot_map=slots, positions=positions)
    clean(pi)
    assert counters.tolist()[:2] == [3, 12] and (table[0, 1:] == -1).all() and (table[1] == -1).all()
    pi.close()


def test_pages_of_the_largest_batch_and_a_long_prompt():
    pi = context(max_batch=4096, max_blocks=16384, block_tokens=16)
    batch = 4096
    rng = np.random.default_rng(2)
    new = rng.integers(0, 40, batch)
    new[17] = 262144
    new[4095] = 1
    need = int((-(-new // 16)).sum())
    table = np.full((batch, 16384), -1, dtype=np.int32)
    order = rng.permutation(need).astype(np.int32)
    sim = ref.Pages(table, order, [0, need, 0, 0], 16)
    state = dev(table), dev(order), torch.tensor([0, need, 0, 0], dtype=torch.int64, device=DEV)
    check_pages(pi, sim, state, np.zeros(batch, dtype=np.int64), new, int(new.sum()))
    pi.close()


def test_pages_in_a_replayed_graph():
    pi = context(max_blocks=16)
    table = np.full((2, 16), -1, dtype=np.int32)
    order = np.random.default_rng(0).permutation(32).astype(np.int32)
    sim = ref.Pages(table, order, [0, 32, 0, 0], 16)
    t, ring, counters = dev(table), dev(order), torch.tensor([0, 32, 0, 0], dtype=torch.int64, device=DEV)
    old, new = i32([0, 0]), i32([0, 0])
    slots, pos = torch.zeros(64, dtype=torch.int64, device=DEV), torch.zeros(64, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pi.assign_pages(old, new, t, ring, counters, slot_map=slots, positions=pos)
    a = np.zeros(2, dtype=np.int64)
    for b in ([20, 3], [21, 16], [21, 17], [0, 17], [31, 47], [5, 0]):
        old.copy_(i32(a)); new.copy_(i32(b))
        graph.replay()
        clean(pi)
        want, want_pos, _ = sim.step(a, np.asarray(b))
        assert np.array_equal(slots[:len(want)].cpu().numpy(), want) and (slots[len(want):] == -1).all()
        assert np.array_equal(pos[:len(want)].cpu().numpy(), want_pos)
        assert np.array_equal(t.cpu().numpy(), sim.table) and counters.tolist()[:2] == sim.state[:2]
        a = np.asarray(b)
    pi.close()


# ------------------------------------------------------------------ append and recall
@pytest.mark.parametrize("heads,block,paged,dev_step", [(2, 16, False, False), (8, 16, True, True), (1, 64, False, True), (4, 32, True, False)])
def test_append_over_block_borders(heads, block, paged, dev_step):
    pi = context(n_q_heads=heads, n_kv_heads=heads, block_tokens=block, pool_slots=20, max_blocks=40, solo_head=[heads - 1])
    rng = np.random.default_rng(heads + block)
    n, NB, C = 3, 40, 20
    ctx = np.asarray([12 * block + block - 2, 25 * block, 5 * block + 1])
    table = np.full((n, NB), -1, dtype=np.int32)
    slot_block = np.full((n, C), -1, dtype=np.int32)
    stamp = rng.integers(0, 50, (n, C)).astype(np.int32)
    for s in range(n):
        cur = -(-int(ctx[s]) // block)
        must = sorted({0} | set(range(max(0, cur - 2), cur)))
        other = [b for b in rng.permutation(cur) if b not in must][:C - len(must) - (2 if s == 0 else 0)]
        for slot, b in zip(rng.permutation(C), must + other):
            table[s, b], slot_block[s, slot] = slot, b
    digest = ref.bf16(np.stack((rng.standard_normal((n, NB, 128)) - 1, rng.standard_normal((n, NB, 128)) + 1), 2))
    pool = ref.pack(ref.bf16(rng.standard_normal((n * C, heads, 2, block, 128))), block).reshape(n, C, -1)
    pages = rng.permutation(n * NB).astype(np.int32).reshape(n, NB) if paged else None
    store = ref.pack(ref.bf16(rng.standard_normal((n * NB, heads, 2, block, 128))), block)
    if not paged:
        store = store.reshape(n, NB, -1)
    sim = ref.Appender(table, slot_block, stamp, digest, pool, store, pi.cfg, heads - 1)
    d = [dev(table), dev(slot_block), dev(stamp), bf(digest)]
    pool_d, store_d = dev(pool), torch.from_numpy(store.copy()).pin_memory()
    pt = dev(pages) if paged else None
    for step in range(100, 104):
        k, v = ref.bf16(rng.standard_normal((2, n, heads, 128)))
        st = i32([step]) if dev_step else step
        pi.append_kv4(0, st, bf(k), bf(v), i32(ctx), store_d, pool_d, d[0], d[1], d[2], d[3], page_table=pt)
        clean(pi)
        sim.step(ctx, k, v, step, pages)
        assert np.array_equal(d[0].cpu().numpy(), sim.table) and np.array_equal(d[1].cpu().numpy(), sim.slot_block)
        assert np.array_equal(d[2].cpu().numpy(), sim.stamp) and np.array_equal(d[3].float().cpu().numpy(), sim.digest)
        assert np.array_equal(pool_d.cpu().numpy(), sim.pool) and np.array_equal(store_d.numpy(), sim.store)
        ctx = ctx + 1
    pi.close()


def test_append_reports_what_cannot_be_appended():
    pi = context(pool_slots=16, max_blocks=10)
    store = torch.zeros((2, 10, pi.kv4_block_bytes), dtype=torch.uint8, device=DEV)
    pool = torch.zeros((2, 16, pi.kv4_block_bytes), dtype=torch.uint8, device=DEV)
    k = torch.ones((2, 2, 128), dtype=torch.bfloat16, device=DEV)

    def tables():
        return (torch.full((2, 10), -1, dtype=torch.int32, device=DEV), torch.full((2, 16), -1, dtype=torch.int32, device=DEV),
                torch.zeros((2, 16), dtype=torch.int32, device=DEV), torch.zeros((2, 10, 2, 128), dtype=torch.bfloat16, device=DEV))

    pi.append_kv4(0, 1, k, k, i32([160, 0]), store, pool, *tables())                   # block 10 of ten
    assert clean(pi, -9)[1] == 5
    pi.append_kv4(0, 1, k, k, i32([5, 0]), store, pool, *tables())                     # the block being filled is not resident
    assert clean(pi, -8)[1] == 5
    t, sb, st, dg = tables()
    sb.zero_()                                                                         # every slot holds the sink block
    pi.append_kv4(0, 1, k, k, i32([16, 16]), store, pool, t, sb, st, dg)
    assert clean(pi, -4)[1] == 5
    pages = torch.full((2, 10), 20, dtype=torch.int32, device=DEV)
    pi.append_kv4(0, 1, k, k, i32([0, 0]), store, pool, *tables(), page_table=pages)   # page 20 of twenty
    assert clean(pi, -8)[1] == 5
    assert int(store[:, 1:].sum()) == 0 and int(pool[:, 2:].sum()) == 0
    pi.close()


@pytest.mark.parametrize("heads,block,paged", [(1, 16, False), (2, 16, True), (8, 16, True), (8, 64, False)])
def test_recall_moves_whole_blocks_and_skips_what_leaves_the_pool(heads, block, paged):
    pi = context(n_q_heads=heads, n_kv_heads=heads, block_tokens=block, pool_slots=16, max_blocks=30)
    rng = np.random.default_rng(heads)
    n, NB, C = 3, 30, 16
    host = torch.from_numpy(rng.integers(0, 256, (n, NB, pi.kv4_block_bytes), dtype=np.uint8)).pin_memory()
    pages = rng.permutation(n * NB).astype(np.int32).reshape(n, NB) if paged else None
    logical = host.numpy() if not paged else host.numpy().reshape(n * NB, -1)[pages]
    lists = np.zeros((n, 16, 4), dtype=np.int32)
    lists[0, :3] = [[2, 0, 3, 0], [9, 5, 1, 3], [20, 12, 4, 4]]
    lists[2, :1] = [[29, 15, 1, 0]]
    pool = torch.full((n, C, pi.kv4_block_bytes), 3, dtype=torch.uint8, device=DEV)
    want = np.full((n, C, pi.kv4_block_bytes), 3, dtype=np.uint8)
    for s, cnt in ((0, 3), (2, 1)):
        for src, dst, m, _ in lists[s, :cnt]:
            want[s, dst:dst + m] = logical[s, src:src + m]
    pi.recall_kv4(0, host, pool, dev(lists), i32([3, 0, 1]), page_table=None if pages is None else dev(pages))
    clean(pi)
    assert np.array_equal(pool.cpu().numpy(), want)
    lists[1, :1] = [[0, 15, 2, 0]]                                                     # its second block would land behind the pool's sequence
    pi.recall_kv4(0, host, pool, dev(lists), i32([0, 1, 0]), page_table=None if pages is None else dev(pages))
    got = clean(pi, -8)
    want[1, 15] = logical[1, 0]
    assert got[1] == 3 and np.array_equal(pool.cpu().numpy(), want)
    lists[1, :1] = [[29, 2, 2, 0]]                                                     # and one that leaves the store
    pi.recall_kv4(0, host, pool, dev(lists), i32([0, 1, 0]), page_table=None if pages is None else dev(pages))
    got = clean(pi, -8)
    want[1, 2] = logical[1, 29]
    assert got[1] == 3 and np.array_equal(pool.cpu().numpy(), want)
    pi.close()


# ------------------------------------------------------------------ attention
def attention_case(pi, ctx, seed, spread=1.0, garbage=True):
    """Pool, lists and queries for the given lengths: the newest block and others, in scattered slots."""
    c = pi.cfg
    rng = np.random.default_rng(seed)
    n, K, C, B, H = len(ctx), c.budget_blocks, c.pool_slots, c.block_tokens, c.n_kv_heads
    kv = ref.bf16(rng.standard_normal((n * C, H, 2, B, 128)) * spread + rng.standard_normal((1, H, 2, 1, 128)))
    pool = ref.pack(kv, B).reshape(n, C, -1)
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
        if nb and last and garbage:                                                    # behind the last token: all ones, NaN scales
            b = pool[s, slots[s, count[s] - 1]]
            t = b[:H * B * 160].reshape(H, B // 16, ref.TILE)
            for r in range(last, B):
                for at, size in ((0, 64), (1024, 64), (2048, 16), (2304, 16)):
                    t[:, r // 16, at + r % 16 * size:at + r % 16 * size + size] = 255
            assert np.isnan(ref.unpack(b[None], H, B)[0, :, :, last:]).all()
    q = ref.bf16(rng.standard_normal((n, c.n_q_heads, 128)))
    return dict(pool=pool, blocks=blocks, slots=slots, count=count, ctx=np.asarray(ctx), q=q)


def check_attention(pi, case, out, lse):
    c = pi.cfg
    out, lse = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    for s in range(len(case["ctx"])):
        def kv_of(slot):
            return ref.unpack(case["pool"][s, slot][None], c.n_kv_heads, c.block_tokens)[0]
        want, want_lse, vmax, eps = ref.attention(case["q"][s].astype(np.float64), kv_of, case["blocks"][s], case["slots"][s], int(case["count"][s]),
                                                  int(case["ctx"][s]), c.block_tokens)
        # one rounding to bf16; weights off by the scores' rounding on both sides of the quotient.  Weight times scale is rounded
        # to 11 bits, by at most 2^-11 each; its codes are at most 15 where the value is at most scale * 15 + |minimum|, so the
        # sum over the tokens is off by at most 2^-11 of the largest |v| times two (scale * 15 <= 2 max|v|)
        G = c.n_q_heads // c.n_kv_heads
        v = np.repeat(np.broadcast_to(vmax, (c.n_kv_heads,)), G)
        tol = 2.0 ** -8 * np.abs(want) + ((2 * eps + 2.0 ** -10) * v)[:, None] + 1e-30
        assert (np.abs(out[s] - want) <= tol).all(), (s, np.abs(out[s] - want).max(), tol.min())
        if lse is not None:
            if np.isinf(want_lse).any():
                assert (lse[s] == -np.inf).all() and (out[s] == 0).all()
            else:
                assert (np.abs(lse[s] - want_lse) <= eps + 2.0 ** -20 * np.abs(want_lse) + 2.0 ** -18).all()


def run_attention(pi, case, lse=True, stream=None):
    n, c = len(case["ctx"]), pi.cfg
    out = torch.full((n + 1, c.n_q_heads, 128), 9.0, dtype=torch.bfloat16, device=DEV)
    l = torch.full((n + 1, c.n_q_heads), 9.0, dtype=torch.float32, device=DEV)
    pi.sparse_decode_attn_kv4(0, bf(case["q"]), dev(case["pool"]), dev(case["slots"]), dev(case["blocks"]), dev(case["count"]), i32(case["ctx"]),
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
    (32, 8, 16, 64, [8192]),                          # one sequence: eight CTAs an item
    (8, 8, 16, 3, [40] * 40),                         # many items: one CTA each
    (4, 1, 16, 300, [4795, 16, 4800]),                # more than 32 tiles a warp
])
def test_attention(Hq, Hkv, B, K, ctx):
    pi = context(n_q_heads=Hq, n_kv_heads=Hkv, block_tokens=B, budget_blocks=K, pool_slots=K + 3, max_batch=max(8, len(ctx)), n_sink_blocks=0, n_local_blocks=1)
    case = attention_case(pi, ctx, Hq * 100 + K)
    out, lse = run_attention(pi, case)
    check_attention(pi, case, out, lse)
    again, _ = run_attention(pi, case, lse=False)
    assert torch.equal(out, again)
    pi.close()


@pytest.mark.parametrize("Hq,Hkv,B,K", [(3, 1, 16, 256), (4, 1, 16, 300), (8, 2, 16, 257), (8, 1, 64, 70), (14, 2, 32, 150), (20, 2, 16, 300)])
def test_attention_over_long_lists_of_few_sequences(Hq, Hkv, B, K):
    """From 256 tiles on a few sequences take larger CTAs: lists of every length, empty ones among them."""
    pi = context(n_q_heads=Hq, n_kv_heads=Hkv, block_tokens=B, budget_blocks=K, pool_slots=K + 3, max_batch=4, max_blocks=2 * K)
    for ctx in ([K * B], [K * B - 3, 0], [37, 1, 2 * K * B - 9, 0], [B * K // 2, 17 * B + 1]):
        case = attention_case(pi, ctx, len(ctx))
        out, lse = run_attention(pi, case)
        check_attention(pi, case, out, lse)
    pi.close()


@pytest.mark.parametrize("Hq,Hkv", [(4, 1), (8, 1), (16, 1)])
def test_attention_over_a_long_list_of_one_sequence(Hq, Hkv):
    """4 096 blocks of 64 tokens, the largest budget: 2 048 tiles for each of eight CTAs."""
    pi = context(n_q_heads=Hq, n_kv_heads=Hkv, block_tokens=64, budget_blocks=4096, pool_slots=4096, max_batch=1, max_blocks=4096)
    rng = np.random.default_rng(0)
    small = ref.pack(ref.bf16(rng.standard_normal((64, Hkv, 2, 64, 128))), 64)
    pool = np.tile(small, (64, 1))[None]
    case = dict(pool=pool, blocks=np.arange(4096, dtype=np.int32)[None], slots=rng.permutation(4096).astype(np.int32)[None], count=np.asarray([4096], np.int32),
                ctx=np.asarray([4096 * 64 - 5]), q=ref.bf16(rng.standard_normal((1, Hq, 128))))
    out, lse = run_attention(pi, case)
    kept = {}

    def kv_of(slot):
        if slot % 64 not in kept:
            kept[slot % 64] = ref.unpack(small[slot % 64][None], Hkv, 64)[0]
        return kept[slot % 64]

    want, want_lse, vmax, eps = ref.attention(case["q"][0].astype(np.float64), kv_of, case["blocks"][0], case["slots"][0], 4096, int(case["ctx"][0]), 64)
    o, l = out[0].double().cpu().numpy(), lse[0].double().cpu().numpy()
    # a warp adds up to 512 tiles in 32 bits: 2^-23 of the sum of magnitudes for each of them; weight times scale as above
    tol = 2.0 ** -8 * np.abs(want) + ((2 * eps + 512 * 2.0 ** -23 + 2.0 ** -10) * np.repeat(vmax, Hq // Hkv))[:, None]
    assert (np.abs(o - want) <= tol).all()
    assert (np.abs(l - want_lse) <= eps + 512 * 2.0 ** -23).all()
    pi.close()


@pytest.mark.parametrize("spread", [1e-30, 1e-3, 60.0, 1e30])
def test_attention_with_small_and_large_values(spread):
    pi = context(budget_blocks=20)
    case = attention_case(pi, [300, 17], 3)
    rng = np.random.default_rng(1)
    kv = ref.bf16(rng.standard_normal((2 * pi.cfg.pool_slots, 2, 2, 16, 128)))
    kv[:, :, 1] = ref.bf16(kv[:, :, 1] * np.float32(spread))                          # V; scores stay ordinary
    case["pool"] = ref.pack(kv, 16).reshape(case["pool"].shape)
    out, lse = run_attention(pi, case)
    check_attention(pi, case, out, lse)
    kv[:, :, 0] = ref.bf16(kv[:, :, 0] * np.float32(40.0))                            # scores in the hundreds: weights of one and nothing
    kv[:, :, 1] = ref.bf16(rng.standard_normal(kv[:, :, 1].shape))
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
    key = float(ref.bf16(np.float32(1.37 * size ** 0.5)))
    kv[:, :, 0] = key                                                                 # a constant row is stored exactly
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
        want = np.repeat(v.mean(axis=1), 4, axis=0)
        # weights are all alike up to the rounding of weight times scale (as in check_attention); the score carries at
        # most nine cuts of 2^-23 in its one product that is not 0 and a few roundings of 2^-24 after it: below 2^-19 of itself
        assert (np.abs(out[s].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * np.abs(v).max()).all()
        want_lse = score + np.log(n)
        assert (np.abs(lse[s].double().cpu().numpy() - want_lse) <= 2.0 ** -19 * abs(score) + 2.0 ** -18).all()
        pick.append(v[:, 0])
    # the first token of each list half as far from 0 (scores below it) or twice as far (above it): the others' weights are nothing
    for s in range(2):
        kv.reshape(2, c.pool_slots, 2, 2, 16, 128)[s, case["slots"][s, 0], :, 0, 0] = key * (2.0 if sign > 0 else 0.5)
    case["pool"] = ref.pack(kv, 16).reshape(case["pool"].shape)
    out, lse = run_attention(pi, case)
    for s in range(2):
        want = np.repeat(pick[s], 4, axis=0)
        assert (np.abs(out[s].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * np.abs(want).max()).all()
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
    pi.sparse_decode_attn_kv4(0, bf(case["q"]), dev(case["pool"]), dev(case["slots"]), dev(case["blocks"]), dev(case["count"]), i32(case["ctx"]), out, lse)
    torch.cuda.synchronize()
    assert pi.status()[0] in (-8, -9) and pi.status()[1] == 4
    pi.clear_status()
    assert torch.equal(out[0], good[0]) and (out[1] == 0).all() and (lse[1] == -float("inf")).all()
    case["count"][1] = 0
    case["blocks"][2, 3] = -1                                                          # what the kernel skipped, the reference skips
    check_attention(pi, case, out, lse)
    # NaN in one sequence's cache stays in that sequence
    case = attention_case(pi, [250, 250], 9)
    case["pool"][1, case["slots"][1, 0], 2304:2306] = 255
    out, _ = run_attention(pi, case)
    assert torch.isnan(out[1]).any() and torch.isfinite(out[0].float()).all()
    pi.close()


def test_attention_takes_a_list_as_it_is():
    """Entries behind the count are not looked at, a block named twice counts twice, a block behind the context not at all;
    rows without any spread; a head whose query is not a number leaves the others alone."""
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
    kv = np.zeros((4 * pi.cfg.pool_slots, 2, 2, 16, 128), dtype=np.float32)
    kv += ref.bf16(np.random.default_rng(3).standard_normal((4 * pi.cfg.pool_slots, 2, 2, 16, 4))).repeat(32, -1)
    case["pool"] = ref.pack(kv, 16).reshape(case["pool"].shape)
    out, lse = run_attention(pi, case)
    check_attention(pi, case, out, lse)
    case["pool"][:] = 0                                                                # a pool that was never written: all values zero
    out, lse = run_attention(pi, case)
    check_attention(pi, case, out, lse)
    assert (out == 0).all()
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


def test_rotation_and_store_in_a_replayed_graph_and_on_a_side_stream():
    pi = context(n_q_heads=8, n_kv_heads=4, block_tokens=32)
    g = torch.Generator().manual_seed(5)
    T = 70
    qkv = torch.zeros((T, 16 * 128), dtype=torch.bfloat16, device=DEV)
    q, k, v = qkv[:, :1024].unflatten(1, (8, 128)), qkv[:, 1024:1536].unflatten(1, (4, 128)), qkv[:, 1536:].unflatten(1, (4, 128))
    pos, slots = torch.zeros(T, dtype=torch.int32, device=DEV), torch.zeros(T, dtype=torch.int64, device=DEV)
    freq = dev((1e4 ** (-np.arange(0, 128, 2) / 128)).astype(np.float32))
    store = torch.zeros((4, pi.kv4_block_bytes), dtype=torch.uint8, device=DEV)
    out = torch.zeros((4, 4, 2, 32, 128), dtype=torch.bfloat16, device=DEV)

    def step(qo, ko, store, out):
        pi.qk_norm_rope(q, k, pos, freq, qo, ko)
        pi.kv4_store(ko, v, store, slots)
        pi.kv4_load(store, out)

    def buffers():
        return torch.zeros((T, 8, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((T, 4, 128), dtype=torch.bfloat16, device=DEV), torch.zeros_like(store), torch.zeros_like(out)

    captured = buffers()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*captured)
    side = torch.cuda.Stream()
    for live in (70, 1, 33):
        qkv.copy_(torch.randn(qkv.shape, generator=g).to(torch.bfloat16))
        pos.copy_(torch.where(torch.arange(T) < live, torch.arange(T) * 7, -1).to(torch.int32))
        slots.copy_(torch.where(torch.arange(T) < live, torch.randperm(128, generator=g)[:T], -1))
        for t in captured:
            t.zero_()
        graph.replay()
        eager = buffers()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(*eager)
        clean(pi)
        for a, b in zip(captured, eager):
            assert torch.equal(a, b)
        assert (captured[0][live:] == 0).all()
    pi.close()


def test_attention_with_pool_offsets_beyond_32_bits():
    pi = context(n_q_heads=16, n_kv_heads=16, block_tokens=64, budget_blocks=4, pool_slots=8192, max_batch=4)
    small = attention_case(context(n_q_heads=16, n_kv_heads=16, block_tokens=64, budget_blocks=4, pool_slots=8, max_batch=4), [250, 3, 256, 200], 4)
    pool = torch.zeros((4, 8192, pi.kv4_block_bytes), dtype=torch.uint8, device=DEV)   # 5.4 GB
    far = np.asarray([8191, 5000, 8000, 1, 8190, 4096, 77, 3000])
    pool[:, torch.from_numpy(far).to(DEV)] = dev(small["pool"])
    slots = np.where(small["slots"] >= 0, far[np.maximum(small["slots"], 0)], -1).astype(np.int32)
    out, lse = torch.zeros((4, 16, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((4, 16), device=DEV)
    pi.sparse_decode_attn_kv4(0, bf(small["q"]), pool, dev(slots), dev(small["blocks"]), dev(small["count"]), i32(small["ctx"]), out, lse)
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
            pi.sparse_decode_attn_kv4(0, *a, o, stream=s)
    clean(pi)
    for o, w in zip(outs, want):
        assert torch.equal(o, w)
    static = [t.clone() for t in args[0]]
    out = torch.zeros_like(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pi.sparse_decode_attn_kv4(0, *static, out)
    for a, w in zip(args, want):
        for s, t in zip(static, a):
            s.copy_(t)
        graph.replay()
        clean(pi)
        assert torch.equal(out, w)
    pi.close()


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("paged", [False, True])
def test_a_session_in_4_bits_with_appends_eager_and_replayed(paged):
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
        sess = DecodeSession(pi, cfg.batch, cfg.n_layers, paged=paged, kv_bits=4)
        sess.ctx_len.copy_(i32(lens))
        for l in range(cfg.n_layers):
            res = np.stack([np.pad(gen.initial_resident(cfg.replace(ctx=n, batch=1), l)[0][:cfg.pool_slots],
                                   (0, max(0, cfg.pool_slots - len(gen.initial_resident(cfg.replace(ctx=n, batch=1), l)[0]))), constant_values=-1) for n in lens])
            sess.load_layer(l, gen.make_kv(cfg, l, device=torch.device(DEV)), i32(res))
        torch.cuda.synchronize()
        sessions.append((pi, sess))
    g = torch.Generator().manual_seed(1)
    qs = [torch.randn((2, 3, 16, 128), generator=g).to(torch.bfloat16).to(DEV) for _ in range(4)]
    new = [tuple(torch.randn((2, 3, 4, 128), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2)) for _ in range(4)]
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
        DecodeSession(pi, 3, 2, kv_bits=4, split_attention=True)
    with pytest.raises(TypeError):
        pi.sparse_decode_attn(0, qs[0][0], sess.bufs[0].pool, sess.bufs[0].sel_slots, sess.bufs[0].sel_blocks, sess.bufs[0].sel_count, sess.ctx_len, sess.out[0])
    pi.close()
    pi2.close()


def test_prompt_to_attention_through_pages_rotation_store_recall():
    """A ragged batch of prompts: pages, norm + rotation, store into an arena, recall into a pool, attention of the next
    token over everything, against the whole chain in 64 bits."""
    pi = context(n_q_heads=8, n_kv_heads=2, budget_blocks=16, pool_slots=16, max_blocks=16, max_batch=4, n_sink_blocks=1, n_local_blocks=1)
    lens = np.asarray([100, 1, 0, 256])
    rng = np.random.default_rng(12)
    T, cap = int(lens.sum()), int(lens.sum()) + 11
    table = torch.full((4, 16), -1, dtype=torch.int32, device=DEV)
    ring, counters = pi.free_page_ring(40)
    ring.copy_(dev(rng.permutation(40).astype(np.int32)))
    slots, pos = torch.empty(cap, dtype=torch.int64, device=DEV), torch.empty(cap, dtype=torch.int32, device=DEV)
    pi.assign_pages(i32([0] * 4), i32(lens), table, ring, counters, slot_map=slots, positions=pos)
    qkv = bf(rng.standard_normal((cap, 12 * 128)))
    q, k, v = qkv[:, :1024].unflatten(1, (8, 128)), qkv[:, 1024:1280].unflatten(1, (2, 128)), qkv[:, 1280:].unflatten(1, (2, 128))
    freq = (1e4 ** (-np.arange(0, 128, 2) / 128)).astype(np.float32)
    w = (1 + 0.1 * rng.standard_normal((2, 128))).astype(np.float32)
    qo, ko = torch.zeros((cap, 8, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((cap, 2, 128), dtype=torch.bfloat16, device=DEV)
    pi.qk_norm_rope(q, k, pos, dev(freq), qo, ko, q_weight=dev(w[0]), k_weight=dev(w[1]))
    arena = torch.zeros((40, pi.kv4_block_bytes), dtype=torch.uint8).pin_memory()
    pi.kv4_store(ko, v, arena, slots)
    # every block of every sequence into the pool, slot i <- block i
    nb = -(-lens // 16)
    lists = np.zeros((4, 16, 4), dtype=np.int32)
    for s in range(4):
        lists[s, 0] = [0, 0, nb[s], 0]
    pool = torch.zeros((4, 16, pi.kv4_block_bytes), dtype=torch.uint8, device=DEV)
    pi.recall_kv4(0, arena, pool, dev(lists), i32((nb > 0).astype(np.int32)), page_table=table)
    sel = np.where(np.arange(16)[None] < nb[:, None], np.arange(16)[None], -1).astype(np.int32)
    # the query: the last token's (the empty sequence: its own zeros)
    starts = np.concatenate(([0], np.cumsum(lens)))
    last = np.maximum(starts[1:] - 1, 0)
    qd = qo[torch.from_numpy(last).to(DEV)].contiguous()
    out, lse = torch.zeros((4, 8, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((4, 8), device=DEV)
    pi.sparse_decode_attn_kv4(0, qd, pool, dev(sel), dev(sel), i32(nb), i32(lens), out, lse)
    clean(pi)
    kw = ref.rope(k.double().cpu().numpy(), np.concatenate([np.arange(n) for n in lens] + [np.zeros(11)]).astype(np.int32), freq, w[1], 1e-6, False)
    assert (np.abs(ko[:T].double().cpu().numpy() - kw[:T]) <= 2.0 ** -8 * np.abs(kw[:T]) + 2.0 ** -19 * 8).all() and (ko[T:] == 0).all()
    kb, vb = ko.float().cpu().numpy(), v.float().cpu().numpy()
    pools = np.zeros((4, 16, pi.kv4_block_bytes), dtype=np.uint8)
    for s in range(4):
        for t in range(lens[s]):
            ref.write_token(pools[s], t, kb[starts[s] + t], vb[starts[s] + t], 16)
    assert np.array_equal(pool.cpu().numpy(), pools)
    check_attention(pi, dict(pool=pools, blocks=sel, slots=sel, count=nb, ctx=lens, q=qd.float().cpu().numpy()), out, lse)
    # retired: every page is free again
    pi.assign_pages(i32(lens), i32([0] * 4), table, ring, counters)
    clean(pi)
    head, tail = counters.tolist()[:2]
    assert tail - head == 40 and sorted(ring.tolist()) == list(range(40)) and (table == -1).all()
    pi.close()
