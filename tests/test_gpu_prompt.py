"""Attention over packed prompts against the definition in 64 bits."""
import pytest
import torch

import paper_2609_34555_b200 as pkg
from tests.prompt_reference import check, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")


def context(Hq=8, Hkv=2, max_batch=64, **kw):
    return pkg.PulseInfer(**dict(dict(n_layers=1, n_q_heads=Hq, n_kv_heads=Hkv, block_tokens=16, budget_blocks=8, n_sink_blocks=1, n_local_blocks=1,
                                      pool_slots=8, max_batch=max_batch, max_blocks=8, solo_head=[0]), **kw))


def starts(lens):
    got = [0]
    for n in lens:
        got.append(got[-1] + n)
    return got


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def case(Hq, Hkv, n, m, dtype=torch.bfloat16, seed=0, pad=3, scale=1.0):
    """q, k, v with `pad` tokens behind the last sequence, and the bounds of the sequences."""
    g = torch.Generator().manual_seed(seed)
    qs, ks = starts(n), starts(m)
    q, k, v = (torch.randn((t + pad, h, 128), generator=g).to(dtype).cuda() for t, h in ((qs[-1], Hq), (ks[-1], Hkv), (ks[-1], Hkv)))
    return q * scale, k, v, qs, ks


def run(pi, q, k, v, qs, ks, lse=True, stream=None):
    out = torch.full_like(q, 7.0).contiguous()
    l = torch.full(q.shape[:2], 7.0, device="cuda") if lse else None
    pi.prompt_attn(q, k, v, i32(qs), out, k_start=None if ks is None else i32(ks), lse=l, stream=stream)
    torch.cuda.synchronize()
    assert pi.status()[0] == 0, pi.status()
    return out, l


def untouched(out, lse, qs):
    rest = torch.ones(out.shape[0], dtype=torch.bool)
    rest[qs[0]:qs[-1]] = False
    assert bool((out.cpu()[rest] == 7).all()) and (lse is None or bool((lse.cpu()[rest] == 7).all()))


LENGTHS = [([1], [1]), ([128], [128]), ([129], [129]), ([77], [77]), ([300], [300]), ([1, 5, 0, 200, 33], [1, 5, 0, 200, 33]), ([1, 1, 1], [700, 1, 128]),
           ([40, 3], [1000, 131]), ([0, 0], [5, 0]), ([50], [7]), ([300, 20], [100, 0]), ([257, 64], [640, 129])]


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 1), (8, 2), (6, 2), (5, 1), (16, 1), (7, 1), (32, 8)])
@pytest.mark.parametrize("n,m", LENGTHS)
def test_lengths_and_head_groups(Hq, Hkv, n, m):
    pi = context(Hq, Hkv)
    q, k, v, qs, ks = case(Hq, Hkv, n, m)
    out, lse = run(pi, q, k, v, qs, ks)
    check(q.dtype, out, lse, reference(q, k, v, qs, ks))
    untouched(out, lse, qs)


@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (8, 1), (12, 4)])
@pytest.mark.parametrize("n,m", [([3, 150, 1], [3, 150, 900]), ([260], [900])])
def test_fp16(Hq, Hkv, n, m):
    pi = context(Hq, Hkv)
    q, k, v, qs, ks = case(Hq, Hkv, n, m, torch.float16)
    out, lse = run(pi, q, k, v, qs, ks)
    check(q.dtype, out, lse, reference(q, k, v, qs, ks))
    untouched(out, lse, qs)
