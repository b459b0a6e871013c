"""The 8-bit format and the prompt attention's reference without a GPU: what the tests on the GPU rest on, and what is refused before any launch."""
import math
import types

import numpy as np
import pytest
import torch

import paper_2609_34555_b200 as pkg
from paper_2609_34555_b200 import binding
from paper_2609_34555_b200.irq import CudaNormal
from paper_2609_34555_b200.runner import DecodeSession, LayerBuffers, RecallPath
from tests import kv8_reference as ref
from tests import prompt_reference
from tests.test_kv4_cpu import ALIGN, INVALID, P, context, refused
from tests.test_runner_cpu import Calls, buffers


def test_the_table_and_its_rounding_are_those_of_the_type():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(want, ref.TABLE, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate((rng.standard_normal(20000) * np.exp(4 * rng.standard_normal(20000)), (ref.SIZES[1:] + ref.SIZES[:-1]) / 2, ref.SIZES, [0.0, -0.0])).astype(np.float32)
    x = np.clip(np.concatenate((x, -x)), -448, 448)
    assert np.array_equal(torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), ref.round_numbers(x.astype(np.float64)))
    assert (ref.round_numbers(np.asarray([np.nan, np.inf, -np.inf])) == 127).all()


@pytest.mark.parametrize("heads,block", [(1, 16), (8, 16), (4, 32), (16, 64)])
def test_a_blocks_bytes_and_what_a_value_is_off_by(heads, block):
    rng = np.random.default_rng(heads)
    kv = ref.bf16(rng.standard_normal((3, heads, 2, block, 128)) * np.exp(rng.standard_normal((3, heads, 2, 1, 1)) * 5))
    kv[0, 0, 0] = 0
    kv[1, 0, 1] = np.float32(1e-38)
    got = ref.unpack(ref.pack(kv, block), heads, block)
    top = np.abs(kv).max((-1, -2), keepdims=True)
    off = np.abs(got - kv)
    assert (off <= np.maximum(np.abs(kv) * 2.0 ** -4, np.maximum(top * 2.0 ** -17, 2.0 ** -127))).all()
    cfg = types.SimpleNamespace(n_kv_heads=heads, block_tokens=block, head_dim=128)
    assert binding.PulseInfer.kv8_block_bytes.fget(types.SimpleNamespace(cfg=cfg)) == ref.block_bytes(heads, block) == len(ref.pack(kv, block)[0])


def test_tokens_that_join_one_by_one_are_what_one_store_makes_of_them_but_for_the_smallest():
    """Rounding again under a scale that is a power of two larger changes nothing above the numbers without a full fraction."""
    rng = np.random.default_rng(4)
    k, v = ref.bf16(rng.standard_normal((2, 16, 2, 128)) * np.exp(rng.standard_normal((2, 16, 2, 1))))
    one, many = (np.zeros((1, ref.block_bytes(2, 16)), dtype=np.uint8) for _ in range(2))
    ref.store(one, k, v, range(16), 16)
    for t in range(16):
        ref.write_token(many, t, k[t], v[t], 16)
    a, b = ref.unpack(one, 2, 16), ref.unpack(many, 2, 16)
    scale = ref.parts(one[0], 2, 16)[1].astype(np.float64)[None, :, :, None, None]
    assert np.array_equal(ref.parts(one[0], 2, 16)[1], ref.parts(many[0], 2, 16)[1])
    full = np.abs(a) >= 2.0 ** -6 * scale
    assert np.array_equal(a[full], b[full]) and (np.abs(a - b) <= 2.0 ** -9 * scale).all()


def test_the_attentions_allowance_tells_a_lost_weight():
    rng = np.random.default_rng(5)
    kv = ref.unpack(ref.pack(ref.bf16(rng.standard_normal((4, 1, 2, 16, 128))), 16), 1, 16)
    q = rng.standard_normal((2, 128))
    out, lse, tol, eps = ref.attention(q, lambda s: kv[s], [0, 1, 2, 3], [0, 1, 2, 3], 4, 60, 16)
    less = ref.attention(q, lambda s: kv[s], [0, 1, 2, 3], [0, 1, 2, 3], 4, 59, 16)
    assert (np.abs(less[0] - out) > tol).any() and (np.abs(less[1] - lse) > eps + 2.0 ** -18).all()
    assert ref.attention(q, None, [-1], [0], 1, 60, 16)[1].tolist() == [-math.inf] * 2


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_the_prompt_reference_is_plain_attention_and_its_check_tells_a_wrong_mask(dtype):
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((t, h, 128), generator=g).to(dtype) for t, h in ((50, 4), (90, 2), (90, 2)))
    qs, ks = [0, 20, 20, 48], [0, 20, 31, 90]
    made = prompt_reference.reference(q, k, v, qs, ks)
    for s in (0, 2):
        a, b, c, d = qs[s], qs[s + 1], ks[s], ks[s + 1]
        mask = torch.arange(d - c)[None] <= torch.arange(b - a)[:, None] + (d - c) - (b - a)
        want = torch.nn.functional.scaled_dot_product_attention(q[a:b].double().transpose(0, 1), k[c:d].double().repeat_interleave(2, 1).transpose(0, 1),
                                                                v[c:d].double().repeat_interleave(2, 1).transpose(0, 1), attn_mask=mask).transpose(0, 1)
        assert torch.allclose(want, made[0][a:b], atol=1e-12)
    prompt_reference.check(dtype, made[0].to(dtype), made[1].float(), made)
    with pytest.raises(AssertionError):
        wrong = prompt_reference.reference(q, k, v, qs, [0, 20, 30, 90])
        prompt_reference.check(dtype, wrong[0].to(dtype), None, made)


@pytest.mark.parametrize("name", ["pi_prompt_attn", "pi_kv8_store", "pi_kv8_load", "pi_append_kv8", "pi_recall_kv8", "pi_sparse_decode_attn_kv8"])
def test_calls_without_a_context_are_refused(name):
    call = getattr(pkg.load_library(), name)
    kinds = call.argtypes
    assert call(*[0.0 if "float" in k.__name__ else None if "void" in k.__name__ or "P" in k.__name__ else 1 for k in kinds]) == -1
    assert pkg.load_library().pi_kv8_block_bytes(None) == -1


def test_calls_by_the_form_of_the_blocks():
    path = object.__new__(RecallPath)
    path.pi = Calls()
    buf = buffers(kv_bits=8)
    path.recall(0, buf, None, None, None)
    path.append(0, 1, buf, None, None, None, None)
    path.attention(0, buf, None, None, None)
    assert path.pi.made == ["recall_kv8", "append_kv8", "sparse_decode_attn_kv8"]
    normal = object.__new__(CudaNormal)
    normal.pi, normal.buf, normal.q, normal.ctx, normal.out, normal.stream = Calls(), buf, None, None, None, None
    normal.torch = types.SimpleNamespace(cuda=types.SimpleNamespace(Event=lambda: types.SimpleNamespace(record=lambda stream: None)))
    normal.enqueue_attention(0)
    assert normal.pi.made == ["sparse_decode_attn_kv8"]
    with pytest.raises(ValueError):
        LayerBuffers(types.SimpleNamespace(cfg=None), 1, kv_bits=5)
    with pytest.raises(ValueError):
        DecodeSession(types.SimpleNamespace(cfg=None), 1, 1, kv_bits=8, split_attention=True)
    with pytest.raises(ValueError):
        path.prepare_layer(0, buf, None, None, None)                                   # digests are built from keys in bf16


def test_prompt_attn_refuses():
    ctx, keep = context()
    good = dict(ctx=ctx, seqs=4, dtype=0, n_q=40, q=P, qt=4096, qh=128, n_k=60, k=P, kt=1024, kh=128, v=P, vt=1024, vh=128, q_start=P, k_start=P, out=P, lse=P, stream=None)
    refused("pi_prompt_attn", good, [
        (dict(ctx=None), INVALID), (dict(seqs=0), INVALID), (dict(seqs=5), INVALID), (dict(seqs=-1), INVALID), (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID),
        (dict(n_q=-1), INVALID), (dict(n_k=-1), INVALID), (dict(n_q=(1 << 31) - 100), INVALID), (dict(n_k=1 << 31), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID),
        (dict(v=None), INVALID), (dict(q_start=None), INVALID), (dict(out=None), INVALID), (dict(qt=0), INVALID), (dict(qh=-128), INVALID), (dict(kt=0), INVALID),
        (dict(vh=0), INVALID), (dict(vt=1 << 40), INVALID), (dict(qt=4100), ALIGN), (dict(kh=132), ALIGN), (dict(vt=1028), ALIGN), (dict(q=P + 8), ALIGN),
        (dict(k=P + 8), ALIGN), (dict(v=P + 2), ALIGN), (dict(out=P + 4), ALIGN), (dict(n_q=0, q=None, out=None), 0)])


def test_the_8_bit_calls_refuse_what_the_4_bit_calls_refuse():
    ctx, keep = context()
    good = dict(ctx=ctx, n=40, k=P, kt=1024, kh=128, ko=0, v=P, vt=1024, vh=128, vo=0, inner=0, slots=P, store=P, n_blocks=4, stream=None)
    refused("pi_kv8_store", good, [
        (dict(ctx=None), INVALID), (dict(n=-1), INVALID), (dict(n=1 << 31), INVALID), (dict(inner=-1), INVALID), (dict(n_blocks=0), INVALID), (dict(kt=-8), INVALID),
        (dict(kt=1020), ALIGN), (dict(vo=4), ALIGN), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(store=None), INVALID), (dict(slots=None, n=65), INVALID),
        (dict(k=P + 8), ALIGN), (dict(store=P + 4), ALIGN), (dict(n=0, k=None), 0)])
    refused("pi_kv8_load", dict(ctx=ctx, n=4, store=P, n_blocks=4, blocks=P, out=P, stream=None), [
        (dict(ctx=None), INVALID), (dict(n=-1), INVALID), (dict(n_blocks=0), INVALID), (dict(n=1 << 30), -3), (dict(store=None), INVALID), (dict(out=None), INVALID),
        (dict(blocks=None, n=5), INVALID), (dict(store=P + 8), ALIGN), (dict(out=P + 8), ALIGN), (dict(n=0, store=None), 0)])
    good = dict(ctx=ctx, layer=1, batch=4, step=3, step_dev=None, k=P, v=P, ctx_len=P, host=P, hs=0, pt=None, ps=0, pages=0, pool=P, table=P, sb=P,
                stamp=P, digest=P, stream=None)
    refused("pi_append_kv8", good, [
        (dict(ctx=None), INVALID), (dict(layer=2), INVALID), (dict(batch=5), INVALID), (dict(step=0), INVALID), (dict(k=None), INVALID), (dict(host=None), INVALID),
        (dict(digest=None), INVALID), (dict(hs=-16), INVALID), (dict(hs=8), ALIGN), (dict(pt=P, ps=0, pages=5), INVALID), (dict(k=P + 8), ALIGN), (dict(pool=P + 8), ALIGN)])
    good = dict(ctx=ctx, layer=0, batch=4, host=P, hs=0, pt=None, ps=0, pages=0, pool=P, lists=P, cap=64, count=P, stream=None)
    refused("pi_recall_kv8", good, [
        (dict(ctx=None), INVALID), (dict(layer=2), INVALID), (dict(batch=5), INVALID), (dict(host=None), INVALID), (dict(count=None), INVALID), (dict(cap=0), INVALID),
        (dict(hs=-16), ALIGN), (dict(pt=P, ps=5, pages=0), INVALID), (dict(lists=P + 8), ALIGN), (dict(pool=P + 8), ALIGN)])
    good = dict(ctx=ctx, layer=0, batch=4, q=P, pool=P, slots=P, blocks=P, count=P, ctx_len=P, out=P, lse=None, stream=None)
    refused("pi_sparse_decode_attn_kv8", good, [
        (dict(ctx=None), INVALID), (dict(layer=2), INVALID), (dict(batch=0), INVALID), (dict(q=None), INVALID), (dict(pool=None), INVALID), (dict(slots=None), INVALID),
        (dict(out=None), INVALID), (dict(q=P + 8), ALIGN), (dict(pool=P + 8), ALIGN), (dict(out=P + 8), ALIGN)])


def test_the_front_end_refuses_what_is_not_on_the_gpu():
    ctx, keep = context()
    pi = object.__new__(pkg.PulseInfer)
    pi._lib, pi._ctx, pi.cfg, pi.device, pi.kv4_block_bytes = pkg.load_library(), ctx, keep[1], torch.device("cuda", 0), 20480
    pi._remember_shape()
    pi.close = lambda: None                                     # (nothing was created)
    i32, bf = torch.zeros(5, dtype=torch.int32), torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    blocks = torch.zeros((4, pi.kv8_block_bytes), dtype=torch.uint8)
    here = dict(stream=0)                                       # (the current stream of a device that is not there cannot be asked for)
    with pytest.raises(TypeError, match="q: expected a CUDA tensor of bfloat16 or float16"):
        pi.prompt_attn(torch.zeros((4, 32, 128), dtype=torch.bfloat16), bf, bf, i32, bf, **here)
    with pytest.raises(TypeError, match="k: expected a CUDA tensor"):
        pi.kv8_store(bf, bf, blocks, **here)
    with pytest.raises(TypeError, match="out"):
        pi.kv8_load(blocks, bf, **here)
    with pytest.raises(TypeError):
        pi.append_kv8(0, 1, bf, bf, i32[:4], blocks, blocks, i32, i32, i32, bf, **here)
    with pytest.raises(TypeError):
        pi.recall_kv8(0, blocks, blocks, torch.zeros((4, 8, 4), dtype=torch.int32), i32[:4], **here)
    with pytest.raises(TypeError, match="q"):
        pi.sparse_decode_attn_kv8(0, bf, blocks, i32, i32, i32, i32, bf, **here)


def test_prompts_that_do_not_fit_are_refused_before_anything_is_written():
    sess = object.__new__(DecodeSession)
    made = []
    sess.pi = types.SimpleNamespace(cfg=types.SimpleNamespace(max_blocks=4, block_tokens=16, pool_slots=4), prompt_attn=lambda *a, **k: made.append(a))
    sess.batch, sess.kv_bits, sess.device, sess.ctx_len = 2, 8, torch.device("cpu"), torch.full((2,), 9, dtype=torch.int32)
    q, k, starts = torch.zeros((20, 4, 128), dtype=torch.bfloat16), torch.zeros((20, 2, 128), dtype=torch.bfloat16), torch.tensor([0, 5, 20], dtype=torch.int32)
    for args, kw, error in (((q[:19], k, k, starts), {}, ValueError), ((q, k[:19], k[:19], starts), {}, ValueError), ((q, k, k[:19], starts), {}, ValueError),
                            ((q.half(), k.half(), k.half(), starts), {}, TypeError), ((q, k, k.float(), starts), {}, TypeError), ((q, k, k, starts[:2]), {}, ValueError),
                            ((q, k, k, starts.flip(0)), {}, ValueError), ((q, k, k, starts), dict(resident=torch.zeros((2, 3), dtype=torch.int32)), ValueError)):
        with pytest.raises(error, match="load_prompts"):
            sess.load_prompts(0, *args, torch.zeros_like(args[0]), **kw)
    assert made == [] and sess.ctx_len.tolist() == [9, 9]
