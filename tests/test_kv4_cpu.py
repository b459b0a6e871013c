"""The 4-bit format and the refusals of the calls around it, without a GPU.

The argument checks read nothing of a context but its configuration, with which it begins, so a zeroed buffer that
starts with one stands for a context in calls that must be refused."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_34555_b200 as pkg
from paper_2609_34555_b200.binding import PiConfig
from tests import kv4_reference as ref

P = 4096                                     # an aligned address that no refused call follows
INVALID, ALIGN, DIM, PINNED = -1, -2, -3, -5


def context(**kw):
    base = dict(n_layers=2, n_q_heads=32, n_kv_heads=8, head_dim=128, block_tokens=16, budget_blocks=64, n_sink_blocks=1,
                n_local_blocks=8, pool_slots=128, max_batch=4, max_blocks=512, recall_ctas=0, attn_ctas=0, attn_mode=0,
                wait_limit_us=0, test_hold_producer=0)
    base.update(kw)
    buf = ctypes.create_string_buffer(4096)
    cfg = PiConfig.from_buffer(buf)
    for name, value in base.items():
        setattr(cfg, name, value)
    return ctypes.cast(buf, ctypes.c_void_p), (buf, cfg)


@pytest.mark.parametrize("heads,block", [(1, 16), (2, 16), (4, 16), (8, 16), (16, 16), (8, 32), (1, 64), (16, 64)])
def test_block_bytes(heads, block):
    lib = pkg.load_library()
    ctx, keep = context(n_kv_heads=heads, n_q_heads=heads, block_tokens=block)
    n = lib.pi_kv4_block_bytes(ctx)
    assert n == ref.block_bytes(heads, block) and n % 4096 == 0 and heads * block * 160 <= n < heads * block * 160 + 4096
    assert lib.pi_kv4_block_bytes(None) == INVALID


@pytest.mark.parametrize("place", [ref.k_place, ref.v_place])
def test_every_nibble_of_a_row_holds_one_channel(place):
    assert sorted(place(d) for d in range(128)) == sorted((b, s) for b in range(64) for s in (0, 4))


def test_reference_rounding_is_half_a_step_at_most():
    rng = np.random.default_rng(0)
    x = ref.bf16(rng.standard_normal((50, 128)) * np.exp(rng.standard_normal((50, 1)) * 4))
    codes, s, lo = ref.round_rows(x)
    assert codes.max() == 15 and codes.min() == 0
    got = ref.values(codes, s, lo)
    step = np.repeat(s, 32, axis=1)
    # half a step; at the upper end the rounded scale may leave the maximum out of reach by 15 * 2^-8 of a step
    assert (np.abs(got - x) <= step * (0.5 + 15 * 2.0 ** -8) + 1e-30).all()
    kv = x[:48].reshape(1, 3, 2, 8, 128).repeat(2, axis=3)
    assert np.array_equal(ref.unpack(ref.pack(kv, 16), 3, 16), ref.values(*ref.round_rows(kv)))


def test_reference_token_writer_agrees_with_the_packer():
    rng = np.random.default_rng(1)
    kv = ref.bf16(rng.standard_normal((3, 2, 2, 32, 128)))
    blocks = np.zeros((3, ref.block_bytes(2, 32)), dtype=np.uint8)
    for b in range(3):
        for t in range(32):
            ref.write_token(blocks, b * 32 + t, kv[b, :, 0, t], kv[b, :, 1, t], 32)
    assert np.array_equal(blocks, ref.pack(kv, 32))


def test_special_rows():
    x = np.zeros((5, 128), dtype=np.float32)
    x[0] = 3.0                                                  # no spread
    x[1, 5] = np.nan
    x[2, 40] = np.inf
    x[3, 70] = -np.inf
    x[4, 96], x[4, 97] = 3e38, -3e38                            # the spread overflows
    with np.errstate(all="ignore"):
        got = ref.values(*ref.round_rows(ref.bf16(x)))
    assert (got[0] == 3).all()
    for row, group in ((1, 0), (2, 1), (3, 2), (4, 3)):
        bad = np.isnan(got[row]).reshape(4, 32).all(1)
        assert bad[group] and bad.sum() == 1


# ------------------------------------------------------------------ refusals
def refused(name, good, changes):
    lib = pkg.load_library()
    for change, code in changes:
        args = dict(good)
        args.update(change)
        got = getattr(lib, name)(*args.values())
        assert got == code, (name, change, got)


def test_assign_pages_refuses():
    ctx, keep = context()
    good = dict(ctx=ctx, batch=4, old=P, new=P, table=P, stride=512, ring=P, n_pages=100, state=P, starts=P, n_tokens=64, slots=P, pos=P, stream=None)
    refused("pi_assign_pages", good, [
        (dict(ctx=None), INVALID), (dict(batch=0), INVALID), (dict(batch=5), INVALID), (dict(old=None), INVALID), (dict(new=None), INVALID),
        (dict(table=None), INVALID), (dict(ring=None), INVALID), (dict(state=None), INVALID), (dict(stride=0), INVALID), (dict(n_pages=0), INVALID),
        (dict(n_tokens=-1), INVALID), (dict(n_tokens=1 << 31), INVALID), (dict(slots=P + 8), ALIGN), (dict(pos=P + 4), ALIGN), (dict(state=P + 4), ALIGN)])


def test_qk_norm_rope_refuses():
    ctx, keep = context()
    good = dict(ctx=ctx, n=4, dtype=0, q=P, qs=6144, k=P, ks=6144, pos=P, wq=P, wk=P, eps=1e-6, freq=P, rot=128, inter=0, qo=P, ko=P, stream=None)
    refused("pi_qk_norm_rope", good, [
        (dict(ctx=None), INVALID), (dict(n=-1), INVALID), (dict(n=1 << 31), INVALID), (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID),
        (dict(rot=130), DIM), (dict(rot=63), DIM), (dict(rot=-2), DIM), (dict(inter=2), INVALID), (dict(freq=None), INVALID), (dict(wq=None), INVALID),
        (dict(wk=None), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(q=None), INVALID),
        (dict(k=None), INVALID), (dict(pos=None), INVALID), (dict(qo=None), INVALID), (dict(ko=None), INVALID), (dict(qs=4088), INVALID),
        (dict(ks=1016), INVALID), (dict(qs=6148), ALIGN), (dict(dtype=2, qs=6146), ALIGN), (dict(q=P + 8), ALIGN), (dict(ko=P + 2), ALIGN), (dict(wq=P + 4), ALIGN),
        (dict(n=0, q=None), 0)])


def test_kv4_store_and_load_refuse():
    ctx, keep = context()
    good = dict(ctx=ctx, n=40, k=P, kt=1024, kh=128, ko=0, v=P, vt=1024, vh=128, vo=0, inner=0, slots=P, store=P, n_blocks=4, stream=None)
    refused("pi_kv4_store", good, [
        (dict(ctx=None), INVALID), (dict(n=-1), INVALID), (dict(n=1 << 31), INVALID), (dict(inner=-1), INVALID), (dict(n_blocks=0), INVALID),
        (dict(n_blocks=1 << 31), INVALID), (dict(kt=-8), INVALID), (dict(vh=-128), INVALID), (dict(kt=1020), ALIGN), (dict(vo=4), ALIGN), (dict(k=None), INVALID),
        (dict(v=None), INVALID), (dict(store=None), INVALID), (dict(slots=None, n=65), INVALID), (dict(k=P + 8), ALIGN), (dict(v=P + 2), ALIGN),
        (dict(store=P + 4), ALIGN), (dict(n=0, k=None), 0)])
    good = dict(ctx=ctx, n=4, store=P, n_blocks=4, blocks=P, out=P, stream=None)
    refused("pi_kv4_load", good, [
        (dict(ctx=None), INVALID), (dict(n=-1), INVALID), (dict(n_blocks=0), INVALID), (dict(n=1 << 30), DIM), (dict(store=None), INVALID), (dict(out=None), INVALID),
        (dict(blocks=None, n=5), INVALID), (dict(store=P + 8), ALIGN), (dict(out=P + 8), ALIGN), (dict(n=0, store=None), 0)])


def test_append_recall_and_attention_refuse():
    ctx, keep = context()
    good = dict(ctx=ctx, layer=1, batch=4, step=3, step_dev=None, k=P, v=P, ctx_len=P, host=P, hs=0, pt=None, ps=0, pages=0, pool=P, table=P, sb=P,
                stamp=P, digest=P, stream=None)
    refused("pi_append_kv4", good, [
        (dict(ctx=None), INVALID), (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(batch=0), INVALID), (dict(batch=5), INVALID), (dict(step=0), INVALID),
        (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(ctx_len=None), INVALID), (dict(host=None), INVALID), (dict(pool=None), INVALID),
        (dict(table=None), INVALID), (dict(sb=None), INVALID), (dict(stamp=None), INVALID), (dict(digest=None), INVALID), (dict(hs=-16), INVALID),
        (dict(hs=8), ALIGN), (dict(pt=P, ps=0, pages=5), INVALID), (dict(pt=P, ps=5, pages=0), INVALID), (dict(k=P + 8), ALIGN), (dict(pool=P + 8), ALIGN)])
    no_window, keep2 = context(n_local_blocks=0)
    refused("pi_append_kv4", good, [(dict(ctx=no_window), INVALID)])
    good = dict(ctx=ctx, layer=0, batch=4, host=P, hs=0, pt=None, ps=0, pages=0, pool=P, lists=P, cap=64, count=P, stream=None)
    refused("pi_recall_kv4", good, [
        (dict(ctx=None), INVALID), (dict(layer=2), INVALID), (dict(batch=5), INVALID), (dict(host=None), INVALID), (dict(pool=None), INVALID), (dict(lists=None), INVALID),
        (dict(count=None), INVALID), (dict(cap=0), INVALID), (dict(hs=-16), ALIGN), (dict(pt=P, ps=5, pages=0), INVALID), (dict(lists=P + 8), ALIGN), (dict(pool=P + 8), ALIGN)])
    good = dict(ctx=ctx, layer=0, batch=4, q=P, pool=P, slots=P, blocks=P, count=P, ctx_len=P, out=P, lse=None, stream=None)
    refused("pi_sparse_decode_attn_kv4", good, [
        (dict(ctx=None), INVALID), (dict(layer=2), INVALID), (dict(batch=0), INVALID), (dict(batch=5), INVALID), (dict(q=None), INVALID), (dict(pool=None), INVALID),
        (dict(slots=None), INVALID), (dict(blocks=None), INVALID), (dict(count=None), INVALID), (dict(ctx_len=None), INVALID), (dict(out=None), INVALID),
        (dict(q=P + 8), ALIGN), (dict(pool=P + 8), ALIGN), (dict(out=P + 8), ALIGN)])


def test_the_front_end_refuses_what_is_not_on_the_gpu():
    ctx, keep = context()
    pi = object.__new__(pkg.PulseInfer)
    pi._lib, pi._ctx, pi.cfg, pi.device, pi.kv4_block_bytes = pkg.load_library(), ctx, keep[1], torch.device("cuda", 0), 20480
    pi._remember_shape()
    pi.close = lambda: None                                     # (nothing was created)
    i32, bf = torch.zeros(4, dtype=torch.int32), torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    blocks = torch.zeros((4, 20480), dtype=torch.uint8)
    here = dict(stream=0)                                       # (the current stream of a device that is not there cannot be asked for)
    with pytest.raises(TypeError, match="old_len"):
        pi.assign_pages(i32, i32, torch.zeros((4, 512), dtype=torch.int32), i32, torch.zeros(4, dtype=torch.int64), **here)
    with pytest.raises(TypeError, match="q: expected a CUDA tensor"):
        pi.qk_norm_rope(torch.zeros((4, 32, 128), dtype=torch.bfloat16), bf, i32, None, bf, bf, **here)
    with pytest.raises(TypeError, match="expected a tensor"):
        pi.qk_norm_rope(None, bf, i32, None, bf, bf, **here)
    with pytest.raises(TypeError, match="k: expected a CUDA tensor"):
        pi.kv4_store(bf, bf, blocks, **here)
    with pytest.raises(TypeError):
        pi.kv4_load(blocks.view(4, 2, 10240), bf, **here)       # not whole blocks
    with pytest.raises(TypeError, match="out"):
        pi.kv4_load(blocks, bf, **here)
    with pytest.raises(TypeError):
        pi.append_kv4(0, 1, bf, bf, i32, blocks, blocks, i32, i32, i32, bf, **here)
    with pytest.raises(TypeError):
        pi.recall_kv4(0, blocks, blocks, torch.zeros((4, 8, 4), dtype=torch.int32), i32, **here)
    with pytest.raises(TypeError, match="q"):
        pi.sparse_decode_attn_kv4(0, torch.zeros((4, 32, 128), dtype=torch.bfloat16), blocks, i32, i32, i32, i32, bf, **here)
    with pytest.raises(TypeError):
        pi._front.kv4_load(pi._shape, blocks)                   # wrong number of arguments
    with pytest.raises(ValueError):
        pi._front.kv4_load(pi._ctx, blocks, bf, None, 0)        # not a shape
    pi._ctx = ctypes.c_void_p()


def a_front_end(**kw):
    """A PulseInfer whose context is a zeroed buffer, for calls that must be refused; keep what it returns beside it."""
    ctx, keep = context(**kw)
    pi = object.__new__(pkg.PulseInfer)
    pi._lib, pi._ctx, pi.cfg, pi.device = pkg.load_library(), ctx, keep[1], torch.device("cuda", 0)
    pi.close = lambda: None                                     # (nothing was created)
    pi.kv4_block_bytes = int(pi._lib.pi_kv4_block_bytes(ctx))
    pi.block_bytes = pi.cfg.n_kv_heads * pi.cfg.block_tokens * 512
    return pi, keep


@pytest.mark.parametrize("heads,block", [(1, 16), (2, 16), (8, 32)])
def test_calls_on_bf16_blocks_refuse_4_bit_blocks(heads, block):
    """They address blocks 2 to 3.2 times as large, and would write or read behind the tensor.  Told by the last axis or by the size;
    byte views of whole bf16 stores are taken, and fail here only for not being on a GPU or pinned."""
    pi, keep = a_front_end(n_q_heads=heads, n_kv_heads=heads, block_tokens=block, max_blocks=12, pool_slots=6, budget_blocks=4, n_local_blocks=1, max_batch=2)
    pool4, host4 = torch.zeros((2, 6, pi.kv4_block_bytes), dtype=torch.uint8), torch.zeros((2, 12, pi.kv4_block_bytes), dtype=torch.uint8)
    pool, host = torch.zeros((2, 6, pi.block_bytes // 2), dtype=torch.bfloat16), torch.zeros((2, 12, pi.block_bytes // 2), dtype=torch.bfloat16)
    i32, bf = torch.zeros((2, 4), dtype=torch.int32), torch.zeros((2, heads, 128), dtype=torch.bfloat16)
    lists, count, table = torch.zeros((2, 4, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros((2, 12), dtype=torch.int32)

    def attention(p):
        return [lambda: pi.sparse_decode_attn(0, bf, p, i32, i32, count, count, bf),
                lambda: pi.sparse_decode_attn_resident(0, bf, p, i32, i32, count, count, lists, count, pool),
                lambda: pi.sparse_decode_attn_recalled(0, bf, p, i32, i32, count, count, lists, count, pool, bf)]

    def writing(h, p):
        calls = []
        for kw in (dict(), dict(page_table=table), dict(page_table=table, n_pages=24)):
            calls.append(lambda kw=kw: pi.recall_gather_scatter(0, h, p, lists, count, **kw))
            calls += [lambda kw=kw, step=step: pi.append_kv(0, step, bf, bf, count, h, p, i32, i32, i32, bf, **kw) for step in (1, count[:1])]
        return calls

    for make in (lambda t: t, lambda t: t.view(2, -1), lambda t: t.view(2, t.shape[1], 2, -1)):
        small_pool, small_host = make(pool4), make(host4)
        for call in attention(small_pool) + writing(host, small_pool):
            with pytest.raises(TypeError, match="pool: expected blocks of bf16"):
                call()
        for i, call in enumerate(writing(small_host, pool)):
            if 3 <= i < 6 and small_host is not host4:
                continue                                        # (an arena of so many bytes, read as fewer pages: nothing to tell it by)
            with pytest.raises(TypeError, match="host_kv: expected blocks of bf16"):
                call()
        with pytest.raises(TypeError, match="kv: expected blocks of bf16"):
            pi.build_digests(0, small_host, count, bf)
        with pytest.raises(TypeError, match="kv: expected blocks of bf16"):
            pi.build_digests_all(small_host, count, bf)
    for view in (lambda t: t, lambda t: t.view(torch.uint8), lambda t: t.view(torch.uint8).view(2, -1)):
        for call in attention(view(pool)):
            with pytest.raises(TypeError, match="contiguous CUDA tensor"):
                call()
        for call in writing(view(host), view(pool)):
            with pytest.raises(pkg.PiError) as e:
                call()
            assert e.value.code == PINNED
    frag = block * 512                                          # units of one KV head: any rows, of as many bytes
    if heads == 2:
        assert frag == pi.kv4_block_bytes
    with pytest.raises(pkg.PiError):
        pi.recall_gather_scatter(0, host.view(torch.uint8).view(-1, frag), pool.view(torch.uint8).view(-1, frag), lists.repeat(heads, 1, 1), count.repeat(heads), lists_per_seq=heads,
                                 unit_bytes=frag, unit_stride=frag, host_seq_stride=12 * pi.block_bytes, pool_seq_stride=6 * pi.block_bytes)
    pi._ctx = ctypes.c_void_p()


def test_a_flag_without_a_truth_value_is_an_error():
    """Whatever asking for it raises is raised; it does not count as true."""
    pi, keep = a_front_end()
    bf, i32 = torch.zeros((4, 8, 128), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)

    class Neither:
        def __bool__(self):
            raise ZeroDivisionError("neither")

    with pytest.raises(ZeroDivisionError):
        pi.qk_norm_rope(torch.zeros((4, 32, 128), dtype=torch.bfloat16), bf, i32, None, bf, bf, interleaved=Neither(), stream=0)
    with pytest.raises(TypeError, match="CUDA tensor"):
        pi.qk_norm_rope(torch.zeros((4, 32, 128), dtype=torch.bfloat16), bf, i32, None, bf, bf, interleaved=1, stream=0)
    pi._ctx = ctypes.c_void_p()
