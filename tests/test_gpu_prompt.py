"""Attention over packed prompts against the definition in 64 bits."""
import random

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


@pytest.mark.parametrize("Hq,Hkv,n,m", [(8, 1, 1, 9000), (8, 2, 5, 4200), (32, 8, 40, 2300), (4, 4, 130, 3000), (16, 1, 17, 1030), (2, 1, 1, 130000)])
def test_few_queries_over_many_keys(Hq, Hkv, n, m):
    """Keys shared out over clusters and over both softmax groups."""
    pi = context(Hq, Hkv)
    for batch in (1, 3):
        if batch * m > 140000:
            continue
        q, k, v, qs, ks = case(Hq, Hkv, [n] * batch, [m - 37 * i for i in range(batch)], seed=n)
        out, lse = run(pi, q, k, v, qs, ks)
        check(q.dtype, out, lse, reference(q, k, v, qs, ks))
        untouched(out, lse, qs)


# so many sequences of one token beside the others that the items are of two query tiles, whatever the GPU's SMs
ONES = [1] * 250


@pytest.mark.parametrize("Hq,Hkv,dtype", [(1, 1, torch.bfloat16), (4, 1, torch.float16), (8, 2, torch.bfloat16), (10, 2, torch.bfloat16), (16, 1, torch.bfloat16), (7, 1, torch.float16)])
@pytest.mark.parametrize("n,m", LENGTHS + [([64, 65, 63], [64, 192, 255]), ([256, 129], [320, 130])])
def test_two_query_tiles_an_item(Hq, Hkv, dtype, n, m):
    pi = context(Hq, Hkv, max_batch=300)
    n, m = n + ONES, m + ONES
    q, k, v, qs, ks = case(Hq, Hkv, n, m, dtype, seed=sum(n) + Hq)
    out, lse = run(pi, q, k, v, qs, ks)
    check(q.dtype, out, lse, reference(q, k, v, qs, ks))
    untouched(out, lse, qs)


@pytest.mark.parametrize("Hq,Hkv,batch,n,m,dtype", [(8, 8, 10, 200, 5000, torch.bfloat16), (16, 4, 20, 50, 4400, torch.float16), (12, 4, 20, 70, 4300, torch.bfloat16)])
def test_two_ctas_share_items_of_two_query_tiles(Hq, Hkv, batch, n, m, dtype):
    r = random.Random(batch + n)
    lens = [n] + [r.randrange(n // 2, n + 1) for _ in range(batch - 3)] + [0, 1]
    keys = [m + 700 + r.randrange(0, 600) for _ in range(batch - 2)] + [9, 300]
    q, k, v, qs, ks = case(Hq, Hkv, lens, keys, dtype, seed=n)
    pi = context(Hq, Hkv)
    out, lse = run(pi, q, k, v, qs, ks)
    check(q.dtype, out, lse, reference(q, k, v, qs, ks))
    untouched(out, lse, qs)


def test_a_prompt_of_many_blocks_and_a_large_batch():
    pi = context(4, 1, max_batch=300)
    for lens in ([1900], [1 + 7 * (i % 29) for i in range(300)]):
        q, k, v, qs, ks = case(4, 1, lens, lens, seed=len(lens))
        out, lse = run(pi, q, k, v, qs, None)
        check(q.dtype, out, lse, reference(q, k, v, qs, ks))
        untouched(out, lse, qs)


def test_random_shapes():
    r = torch.Generator().manual_seed(11)
    pick = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=r))  # noqa: E731
    for i in range(40):
        Hkv = (1, 2, 4, 8, 16)[pick(0, 4)]
        Hq = Hkv * pick(1, 16)
        batch = pick(1, 9)
        n = [pick(0, (3, 70, 300)[pick(0, 2)]) for _ in range(batch)]
        m = [max(0, a + (pick(0, 500) if pick(0, 1) else pick(-40, 10))) for a in n]
        dtype = torch.bfloat16 if pick(0, 2) else torch.float16
        pi = context(Hq, Hkv)
        q, k, v, qs, ks = case(Hq, Hkv, n, m, dtype, seed=i, pad=pick(1, 5))
        out, lse = run(pi, q, k, v, qs, ks)
        check(dtype, out, lse, reference(q, k, v, qs, ks))
        untouched(out, lse, qs)
        pi.close()


def test_strides_and_no_lse():
    """Slices of a fused projection, heads before tokens, every second token; the first sequence not at the first token."""
    pi = context(8, 2)
    g = torch.Generator().manual_seed(3)
    qs = [5, 90, 200]
    want = None
    x = torch.randn((220, 12 * 128), generator=g).to(torch.bfloat16).cuda()
    q, k, v = x[:, :1024].unflatten(1, (8, 128)), x[:, 1024:1280].unflatten(1, (2, 128)), x[:, 1280:].unflatten(1, (2, 128))
    heads_first = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    spaced = lambda t: t.repeat_interleave(2, 0)[::2]  # noqa: E731
    for form in (lambda t: t, lambda t: t.contiguous(), heads_first, spaced):
        out, lse = torch.full((220, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda"), None
        pi.prompt_attn(form(q), form(k), form(v), i32(qs), out)
        torch.cuda.synchronize()
        assert pi.status()[0] == 0
        if want is None:
            check(out.dtype, out, lse, reference(q, k, v, qs, qs))
            untouched(out, None, qs)
            want = out
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,m", [([200, 61, 3], [200, 61, 3]), ([2, 70], [300, 1000]), ([200, 61, 3] + ONES, [200, 61, 3] + ONES), ([2, 70] + ONES, [300, 1000] + ONES)])
def test_what_is_not_seen_does_not_reach_a_row(dtype, n, m):
    """Infinities and NaN in keys and values: rows that see them are what the sums make of them, all others are as without them.  In the
    tokens behind a sequence, in its neighbours, and in its own future."""
    pi = context(8, 2, max_batch=300)
    q, k, v, qs, ks = case(8, 2, n, m, dtype, seed=5, pad=40)
    base, base_lse = run(pi, q, k, v, qs, ks)
    bad_v = [(ks[1] - 1, 0, 3, float("nan")), (ks[1] - min(m[0], 30), 1, 9, float("inf")), (ks[1], 0, 70, float("-inf")), (ks[-1] + 2, 0, 5, float("nan")), (ks[-1] + 39, 1, 127, float("inf"))]
    bad_k = [(ks[-1] - 1, 1, 2, float("nan")), (ks[-1] + 1, 0, 0, float("inf"))]
    for t, h, d, x in bad_v:
        v[t, h, d] = x
    for t, h, d, x in bad_k:
        k[t, h, d] = x
    out, lse = run(pi, q, k, v, qs, ks)
    for s in range(len(n)):
        for i in range(n[s]):
            row, seen = qs[s] + i, ks[s] + i + m[s] - n[s] + 1
            for h in range(2):
                heads = slice(4 * h, 4 * h + 4)
                if any(kh == h and ks[s] <= t < seen for t, kh, _, _ in bad_k):
                    assert torch.isnan(out[row, heads].float()).all()
                    continue
                assert torch.equal(lse[row, heads], base_lse[row, heads])
                hit = {d: x for t, vh, d, x in bad_v if vh == h and ks[s] <= t < seen}
                for d in range(128):
                    got = out[row, heads, d].float()
                    if d in hit:
                        assert torch.equal(got, torch.full_like(got, hit[d])) or (hit[d] != hit[d] and torch.isnan(got).all()), (s, i, h, d)
                keep = [d for d in range(128) if d not in hit]
                assert torch.equal(out[row, heads][:, keep], base[row, heads][:, keep]), (s, i, h)


@pytest.mark.parametrize("dtype,scale", [(torch.bfloat16, 30.0), (torch.bfloat16, 1e5), (torch.bfloat16, 1e9), (torch.bfloat16, 1e15), (torch.float16, 100.0)])
def test_scores_of_any_size(dtype, scale):
    """Queries and keys so large that one key takes all the weight: the output is its value, the log-sum-exp its score."""
    pi = context(4, 2)
    q, k, v, qs, ks = case(4, 2, [150, 7], [400, 7], dtype, seed=9, scale=scale if dtype == torch.bfloat16 else 1.0)
    k = (k * scale).to(dtype)
    out, lse = run(pi, q, k, v, qs, ks)
    o, l, _, _, owned = reference(q, k, v, qs, ks)
    out, lse = out.cpu().double(), lse.cpu().double()
    # a score is a sum of 128 products in 32 bits, off by at most 128 cuts of 2^-23 of the sum of magnitudes
    size = (q.abs().float().amax(-1).cpu().double() * k.abs().float().amax().cpu().double() * 128 / 128 ** 0.5)
    off = 128 * 2.0 ** -23 * size
    assert bool(((lse - l).abs() <= off + 2.0 ** -16 * (1 + l.abs()))[owned].all())
    # rows whose two largest scores are further apart than that: the weights are known
    for s in range(2):
        for i in range(qs[s], qs[s + 1]):
            for h in range(4):
                seen = ks[s + 1] - (qs[s + 1] - 1 - i)
                z = k[ks[s]:seen, h // 2].cpu().double() @ q[i, h].cpu().double() / 128 ** 0.5
                top = torch.topk(z, min(2, len(z)))
                if len(z) == 1 or float(top.values[0] - top.values[1]) > 2 * float(off[i, h]) + 20:
                    want = v[ks[s] + int(top.indices[0]), h // 2].cpu().double()
                    assert bool(((out[i, h] - want).abs() <= torch.finfo(dtype).eps * want.abs() + 2.0 ** -20).all())


@pytest.mark.parametrize("others", [[], ONES])
def test_scores_that_rise_from_key_to_key(others):
    """Every tile's largest score is above the last one's by more than a factor of 2^8 after the exponential: the reference moves each time."""
    pi = context(4, 1, max_batch=300)
    n = 700
    q, k, v, qs, ks = case(4, 1, [n] + others, [n] + others, seed=2)
    q[:], k[:] = 0, 0
    q[..., 0] = 1.0
    k[..., 0] = (torch.arange(k.shape[0]) * 0.5).to(torch.bfloat16).cuda()[:, None]
    k[:, :, 1:] = torch.randn(k[:, :, 1:].shape, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    q[..., 1:] = 0.1
    out, lse = run(pi, q, k, v, qs, ks)
    check(q.dtype, out, lse, reference(q, k, v, qs, ks))


def test_heads_whose_query_is_no_number_leave_the_others_alone():
    pi = context(8, 2)
    q, k, v, qs, ks = case(8, 2, [90, 1], [90, 500], seed=4)
    base, base_lse = run(pi, q, k, v, qs, ks)
    q[17, 5, 3] = float("nan")
    q[60, 0] = float("inf")
    q[90, 7, 127] = float("nan")
    out, lse = run(pi, q, k, v, qs, ks)
    hit = torch.zeros(q.shape[:2], dtype=torch.bool)
    hit[17, 5] = hit[60, 0] = hit[90, 7] = True
    assert torch.equal(out.cpu()[~hit], base.cpu()[~hit]) and torch.equal(lse.cpu()[~hit], base_lse.cpu()[~hit])
    assert bool(torch.isnan(out.cpu()[hit].float()).all())


def test_bounds_that_make_no_sense_are_reported_and_left_out():
    pi = context(8, 2)
    q, k, v, qs, ks = case(8, 2, [20, 30, 10], [50, 30, 60], pad=0)
    good, good_lse = run(pi, q, k, v, qs, ks)
    for bad_q, bad_k, which in (([0, 20, 10, 60], ks, 1), (qs, [0, 50, 80, 141], 2), ([-1, 20, 50, 60], ks, 0), (qs, [0, 50, 40, 140], 1)):
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        pi.prompt_attn(q, k, v, i32(bad_q), out, k_start=i32(bad_k), lse=lse)
        torch.cuda.synchronize()
        got = pi.status()
        assert got[0] == -8 and got[1] == 8 and got[2] == which, got
        pi.clear_status()
        # (the sequence behind one whose bounds decrease may name tokens of an earlier one too: those rows are either's)
        spans = [range(x, y) for x, y in zip(bad_q, bad_q[1:]) if 0 <= x <= y <= 60]
        for s in range(3):
            if bad_q[s:s + 2] == qs[s:s + 2] and bad_k[s:s + 2] == ks[s:s + 2]:
                rows = [t for t in range(qs[s], qs[s + 1]) if sum(t in x for x in spans) == 1]
                assert len(rows) >= 10 and torch.equal(out[rows], good[rows]) and torch.equal(lse[rows], good_lse[rows])


def test_no_queries_no_keys():
    pi = context(8, 2)
    q, k, v, qs, ks = case(8, 2, [3, 4], [0, 0], pad=0)
    assert k.shape[0] == 0
    out, lse = run(pi, q, k, v, qs, ks)
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all())
    out, lse = torch.zeros((0, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((0, 8), device="cuda")
    pi.prompt_attn(q[:0], k, v, i32([0, 0]), out, lse=lse)
    torch.cuda.synchronize()
    assert pi.status()[0] == 0


def test_the_front_end_checks_devices_types_and_shapes():
    pi = context(8, 2, max_batch=2)
    q, k, v, qs, ks = case(8, 2, [9], [9], pad=0)
    out, s = torch.zeros_like(q), i32([0, 9])
    for change, error in (
            (lambda: pi.prompt_attn(q.float(), k, v, s, out), TypeError), (lambda: pi.prompt_attn(q, k.half(), v, s, out), TypeError),
            (lambda: pi.prompt_attn(q.cpu(), k, v, s, out), TypeError), (lambda: pi.prompt_attn(q, k, v[:5], s, out), ValueError),
            (lambda: pi.prompt_attn(q[:, :6], k, v, s, out), ValueError), (lambda: pi.prompt_attn(q, k, v, s.long(), out), TypeError),
            (lambda: pi.prompt_attn(q, k, v, s[:1], out), ValueError), (lambda: pi.prompt_attn(q, k, v, s, out.half()), TypeError),
            (lambda: pi.prompt_attn(q, k, v, s, out[:5]), ValueError), (lambda: pi.prompt_attn(q, k, v, s, out, k_start=i32([0, 1, 9])), ValueError),
            (lambda: pi.prompt_attn(q, k, v, s, out, lse=torch.zeros((9, 2), device="cuda")), ValueError),
            (lambda: pi.prompt_attn(q.transpose(1, 2).contiguous().transpose(1, 2), k, v, s, out), ValueError)):
        with pytest.raises(error):
            change()
    x = torch.zeros((9, 12 * 128 + 4), dtype=torch.bfloat16, device="cuda")
    for change, code in ((lambda: pi.prompt_attn(q, k, v, i32([0, 3, 6, 9]), out), -1),                      # more sequences than the context has
                         (lambda: pi.prompt_attn(x[:, :1024].unflatten(1, (8, 128)), k, v, s, out), -2),     # tokens 8 bytes off
                         (lambda: pi.prompt_attn(q, k[:1].expand(9, 2, 128), v, s, out), -1)):               # one key for all tokens
        with pytest.raises(pkg.binding.PiError) as e:
            change()
        assert e.value.code == code
    torch.cuda.synchronize()
    assert pi.status()[0] == 0 and bool((out == 0).all())


def test_on_two_streams_at_once_and_in_a_replayed_graph():
    pi = context(32, 8)
    cases = [case(32, 8, [100, 1, 300], [100, 700, 900], seed=s) for s in (1, 2)]
    want = [run(pi, *c) for c in cases]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    bounds = [(i32(c[3]), i32(c[4])) for c in cases]
    outs = [(torch.full_like(c[0], 7.0), torch.full(c[0].shape[:2], 7.0, device="cuda")) for c in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        for (q, k, v, *_), (qs, ks), (o, l), st in zip(cases, bounds, outs, streams):
            pi.prompt_attn(q, k, v, qs, o, k_start=ks, lse=l, stream=st)
    torch.cuda.synchronize()
    for (o, l), (wo, wl) in zip(outs, want):
        assert torch.equal(o, wo) and torch.equal(l, wl)
    # captured once for a capacity; replayed for other sequences, among them fewer tokens than the capacity
    q, k, v = torch.zeros((500, 32, 128), dtype=torch.bfloat16, device="cuda"), *(torch.zeros((2000, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    qs, ks = i32([0] * 4), i32([0] * 4)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        pi.prompt_attn(q, k, v, qs, out, k_start=ks, lse=lse)
    for n, m in (([100, 1, 300], [100, 700, 900]), ([0, 0, 0], [0, 0, 0]), ([5, 495, 0], [5, 600, 3])):
        cq, ck, cv, a, b = case(32, 8, n, m, seed=sum(n), pad=0)
        q[:a[-1]], k[:b[-1]], v[:b[-1]] = cq, ck, cv
        q[a[-1]:], k[b[-1]:], v[b[-1]:] = float("nan"), float("nan"), float("nan")
        qs.copy_(i32(a)); ks.copy_(i32(b))
        out.fill_(7.0); lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert pi.status()[0] == 0
        check(q.dtype, out[:a[-1]], lse[:a[-1]], reference(cq, ck, cv, a, b))
        untouched(out, lse, a)


@pytest.mark.parametrize("n,m", [([1], [2000]), ([40, 9], [900, 2500]), ([77], [77]), ([300] * 9, [300] * 9)])
def test_the_first_call_of_a_context_may_be_captured(n, m):
    pi = context(32, 8)
    q, k, v, a, b = case(32, 8, n, m, seed=9)
    qs, ks, out, lse = i32(a), i32(b), torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        pi.prompt_attn(q, k, v, qs, out, k_start=ks, lse=lse)
    graph.replay()
    torch.cuda.synchronize()
    assert pi.status()[0] == 0
    check(q.dtype, out, lse, reference(q, k, v, a, b))
    untouched(out, lse, a)


def test_a_wait_that_runs_out_is_reported_and_the_next_call_works():
    """The last values of every piece of work never arrive (a test's switch): every CTA gives up after a millisecond, says so and ends."""
    held = context(8, 2, wait_limit_us=1000, test_hold_producer=1)
    q, k, v, qs, ks = case(8, 2, [300, 2], [300, 1000])
    out = torch.zeros_like(q)
    held.prompt_attn(q, k, v, i32(qs), out, k_start=i32(ks))
    torch.cuda.synchronize()
    assert held.status()[0] == -7 and held.status()[1] == 8
    held.close()
    pi = context(8, 2)
    out, lse = run(pi, q, k, v, qs, ks)
    check(q.dtype, out, lse, reference(q, k, v, qs, ks))


@pytest.mark.parametrize("n,longest", [(1, 3000), (1, 7000), (3, 500), (90, 2000)])
def test_call_after_call_gives_the_same_bits(n, longest):
    """Hundreds of calls without a pause, of uneven sequences, more of them than fit the GPU at once or few that are shared."""
    r = random.Random(n * longest)
    for batch in (21, 5):
        lens = [r.randrange(1, n + 1) for _ in range(batch)]
        q, k, v, qs, ks = case(32, 8, lens, [a + r.randrange(0, longest) for a in lens], seed=n)
        pi = context(32, 8, wait_limit_us=100000)
        out, lse = run(pi, q, k, v, qs, ks)
        check(q.dtype, out, lse, reference(q, k, v, qs, ks))
        a, b, others = i32(qs), i32(ks), [(torch.full_like(out, 7.0), torch.full_like(lse, 7.0)) for _ in range(3)]
        for i in range(300):
            pi.prompt_attn(q, k, v, a, others[i % 3][0], k_start=b, lse=others[i % 3][1])
        torch.cuda.synchronize()
        assert pi.status()[0] == 0, pi.status()
        for o, l in others:
            assert torch.equal(o, out) and torch.equal(l, lse)


def test_keys_beyond_32_bits_of_an_address():
    """Keys 5 GB apart in one tensor: the sequences at its two ends."""
    pi = context(16, 16)
    q, k, v, qs, ks = case(16, 16, [30, 40], [300, 70], pad=0)
    rows = 1300000                                                                     # x 16 heads x 256 bytes
    far = [torch.zeros((rows, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for f, x in zip(far, (k, v)):
        f[:300], f[rows - 70:] = x[:300], x[300:]
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    pi.prompt_attn(q, *far, i32([0, 30, 30, 70]), out, k_start=i32([0, 300, rows - 70, rows]), lse=lse)
    torch.cuda.synchronize()
    assert pi.status()[0] == 0
    check(q.dtype, out, lse, reference(q, k, v, qs, ks))


# ------------------------------------------------------------------ clusters that share items, and many sequences
MANY = [(4, 1, [1] * 256, [4500] * 256),
        (8, 8, [0] * 2016 + [1] * 32, [0] * 2016 + [8000] * 32),
        (8, 8, ([0] * 31 + [1]) * 32, ([0] * 31 + [8000]) * 32)]


@pytest.mark.parametrize("Hq,Hkv,n,m", MANY, ids=["256 of one token", "the last 32 of 2048", "every 32nd of 1024"])
def test_shared_items_of_few_rows_among_many_sequences(Hq, Hkv, n, m):
    """Three items and more a cluster, each of which is told late: the looking through hundreds of sequences comes before it."""
    pi = context(Hq, Hkv, max_batch=2048, wait_limit_us=20000)
    q, k, v, qs, ks = case(Hq, Hkv, n, m, seed=len(n), pad=0)
    out, lse = run(pi, q, k, v, qs, ks)
    check(q.dtype, out, lse, reference(q, k, v, qs, ks))
    a, b, o, l = i32(qs), i32(ks), torch.empty_like(out), torch.empty_like(lse)
    for _ in range(20):
        pi.prompt_attn(q, k, v, a, o, k_start=b, lse=l)
    torch.cuda.synchronize()
    assert pi.status()[0] == 0 and torch.equal(o, out) and torch.equal(l, lse)


def test_shared_items_with_and_without_rows_of_the_second_tile_and_with_empty_ranges():
    """Clusters whose items follow each other in every order: few rows and many, one query tile and two, keys for every CTA, for one, for none."""
    r = random.Random(8)
    n = [r.choice([0, 1, 1, 30, 70, 128, 140, 250]) for _ in range(100)]
    m = [r.choice([0, 1, 9, 128, 129, 300]) if i % 5 == 1 else 5600 + r.randrange(0, 900) for i in range(100)]
    pi = context(2, 2, max_batch=100, wait_limit_us=20000)
    q, k, v, qs, ks = case(2, 2, n, m, seed=8)
    assert 2 * (q.shape[0] + 100 * 255) // 256 <= 296 and sum(m) // 100 > 33 * 128       # up to two items an SM, keys enough: two CTAs each
    out, lse = run(pi, q, k, v, qs, ks)
    check(q.dtype, out, lse, reference(q, k, v, qs, ks))
    untouched(out, lse, qs)
    a, b, o, l = i32(qs), i32(ks), torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    for _ in range(20):
        pi.prompt_attn(q, k, v, a, o, k_start=b, lse=l)
    torch.cuda.synchronize()
    assert pi.status()[0] == 0 and torch.equal(o, out) and torch.equal(l, lse)


@pytest.mark.parametrize("Hq,Hkv,batch", [(8, 8, 24), (4, 1, 12), (8, 1, 3)])
def test_tiles_that_take_long_to_look_through_between_others(Hq, Hkv, batch):
    """Prompts whose last tiles are full of infinities, so that each is rewritten, between sequences that see all of theirs: every load of either
    kind is followed, and the result is there within a short limit of the waits."""
    n = [1 if i % 2 else 129 for i in range(batch)]
    m = [1280 if i % 2 else 900 + 128 * (i % 3) for i in range(batch)]
    q, k, v, qs, ks = case(Hq, Hkv, n, m, seed=batch)
    pi = context(Hq, Hkv, wait_limit_us=20000)
    want, want_lse = run(pi, q, k, v, qs, ks)
    check(q.dtype, want, want_lse, reference(q, k, v, qs, ks))
    for i in range(0, batch, 2):
        v[ks[i + 1] - 128:ks[i + 1], :, ::3] = float("inf")                            # seen by all rows but the first, from one key on
    a, b, out, lse = i32(qs), i32(ks), torch.full_like(want, 7.0), torch.full_like(want_lse, 7.0)
    for _ in range(50):
        pi.prompt_attn(q, k, v, a, out, k_start=b, lse=lse)
    torch.cuda.synchronize()
    assert pi.status()[0] == 0, pi.status()
    assert torch.equal(lse, want_lse)
    keep = [d for d in range(128) if d % 3]
    assert torch.equal(out[..., keep], want[..., keep])
    for i in range(batch):
        rows = out[qs[i]:qs[i + 1], :, ::3].float()
        if i % 2:
            assert torch.equal(rows, want[qs[i]:qs[i + 1], :, ::3].float())
        else:
            assert torch.equal(rows[0], want[qs[i], :, ::3].float()) and bool((rows[1:] == float("inf")).all())


@pytest.mark.parametrize("Hq,Hkv,n,m", [(4, 4, [50], [70]), (8, 1, [5], [2500]), (4, 4, [40, 129] + [1] * 80, [60, 300] + [1] * 80), (2, 2, [30] * 30, [4700] * 30)])
def test_rows_of_a_warp_that_see_different_numbers_of_infinite_values(Hq, Hkv, n, m):
    """Every key of the last ones has an infinity of its own: a warp's rows look at different numbers of them, and some of its rows are of no query."""
    q, k, v, qs, ks = case(Hq, Hkv, n, m, seed=3)
    pi = context(Hq, Hkv, max_batch=100, wait_limit_us=20000)
    want, want_lse = run(pi, q, k, v, qs, ks)
    put = []
    for s, e in enumerate(ks[1:]):
        for x in range(min(n[s], 40)):                                                 # key e - 1 - x: channel 3 x + 1 of every head
            v[e - 1 - x, :, 3 * x + 1] = float("inf") if x % 2 else -float("inf")
            put.append((s, x))
    out, lse = run(pi, q, k, v, qs, ks)
    assert torch.equal(lse, want_lse)
    expect = want.float()
    for s, x in put:                                                                   # the last x + 1 queries see it
        expect[qs[s + 1] - 1 - x:qs[s + 1], :, 3 * x + 1] = float("inf") if x % 2 else -float("inf")
    got = out.float()
    assert torch.equal(torch.isinf(got), torch.isinf(expect)) and torch.equal(got[torch.isinf(got)], expect[torch.isinf(expect)])
    assert torch.equal(got[~torch.isinf(got)], expect[~torch.isinf(expect)])
    untouched(out, lse, qs)


@pytest.mark.parametrize("nats", [5.0, 14.0, 17.0])
@pytest.mark.parametrize("Hq,Hkv,n,m,at", [(4, 1, 1, 65537, 0), (4, 1, 1, 65537, 40000), (2, 2, 40, 20000, 0), (16, 16, 1200, 6000, 3), (16, 16, 1200, 6000, 5000)])
def test_a_long_tail_under_one_large_score_in_fp16(Hq, Hkv, n, m, at, nats):
    """One key far above all others, of value 0: the result is what the others' small weights make of it.  Weights are counted 2^7 times as
    large as under the reference, which the largest is never below, so they are off by half a step (2^-11 of themselves) or by 2^-25-7
    of the largest."""
    q, k, v, qs, ks = case(Hq, Hkv, [n], [m], torch.float16, seed=m, pad=0)
    q[..., 0] = 128 ** 0.5
    k *= 0.1
    k[..., 0] = 0
    k[at, :, 0] = nats
    v += 2
    v[at] = 0
    pi = context(Hq, Hkv)
    out, lse = run(pi, q, k, v, qs, ks)
    ref = reference(q, k, v, qs, ks)
    check(q.dtype, out, lse, ref)
    want, want_lse, spread, thin, _ = ref
    tol = 2.0 ** -11 * want.abs() + (2.0 ** -11 + 2.0 ** -15) * spread + 2.0 ** -32 * thin + 2.0 ** -25
    over = float(((out.cpu().double() - want).abs() / tol).max())
    assert over <= 1.0, over


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,m", [([90], [400]), ([90] + ONES, [400] + ONES), ([3], [3000])])
def test_a_row_with_scores_far_from_zero_leaves_the_bits_of_its_neighbours(dtype, n, m):
    pi = context(8, 2, max_batch=300)
    q, k, v, qs, ks = case(8, 2, n, m, dtype, seed=6)
    base, base_lse = run(pi, q, k, v, qs, ks)
    large = torch.zeros(q.shape[:2], dtype=torch.bool)
    for row, head in ((0, 5), (n[0] // 2, 0), (n[0] - 1, 7)):
        large[row, head] = True
    q[large.cuda()] *= 2000.0
    out, lse = run(pi, q, k, v, qs, ks)
    assert torch.equal(out.cpu()[~large], base.cpu()[~large]) and torch.equal(lse.cpu()[~large], base_lse.cpu()[~large])
    assert bool((lse.cpu()[large].abs() > 1024).all())


# two scores a step of fp32 apart, whose logarithms under base 2 round to the same number although the weights differ by 2^16 and 2^261
@pytest.mark.parametrize("dtype,q0,k0,step", [(torch.float16, 32768.0, 64288.0, 128.0), (torch.bfloat16, 221184.0, 153600.0, 2048.0)])
@pytest.mark.parametrize("others", [[], ONES])
def test_scores_so_large_that_a_step_is_more_than_a_weights_range(dtype, q0, k0, step, others):
    pi = context(4, 1, max_batch=300)
    q, k, v, qs, ks = case(4, 1, [1] + others, [700] + others, dtype, seed=13)
    q[0], k[:700] = 0, 0
    q[0, :, 0], q[0, :, 1] = q0, 1.0
    k[5, 0, 0] = k0
    k[300, 0, 0], k[300, 0, 1] = k0, step
    out, lse = run(pi, q, k, v, qs, ks)
    a, b = v[5, 0].double().cpu(), v[300, 0].double().cpu()
    # (a score is off by more than the two differ, so the result may be either value or any in between)
    got = out[0].double().cpu()
    slack = torch.finfo(dtype).eps * torch.maximum(a.abs(), b.abs()) + 2.0 ** -14
    assert bool(((got >= torch.minimum(a, b) - slack) & (got <= torch.maximum(a, b) + slack)).all())
    assert bool(((lse[0].double().cpu() - q0 * k0 / 128 ** 0.5).abs() <= 2.0 ** -20 * q0 * k0 / 128 ** 0.5).all())
    for s in range(1, len(qs) - 1):
        assert torch.allclose(out[qs[s]].float(), v[ks[s]].float().expand(4, 128))


@pytest.mark.parametrize("batch,longest", [(33, 300), (64, 200), (1024, 9), (1025, 40), (1057, 3), (4096, 5)])
def test_many_sequences_of_any_length(batch, longest):
    """More sequences than are looked at at once, some without queries, some without keys, among them a few long ones."""
    r = random.Random(batch)
    n = [r.choice([0, 0, 1, r.randrange(longest + 1)]) for _ in range(batch)]
    m = [max(0, a + r.choice([0, 0, 7, 130, -2])) for a in n]
    for s in (0, 31, 32, batch // 2, batch - 1):
        n[s], m[s] = 270 + s % 7, 500
    pi = context(2, 2, max_batch=4096)
    q, k, v, qs, ks = case(2, 2, n, m, seed=batch)
    out, lse = run(pi, q, k, v, qs, ks)
    check(q.dtype, out, lse, reference(q, k, v, qs, ks))
    untouched(out, lse, qs)


@pytest.mark.parametrize("batch,at", [(40, 35), (1500, 1499), (1500, 700), (4096, 1024)])
def test_bounds_that_make_no_sense_among_many_sequences(batch, at):
    n = [3] * batch
    pi = context(2, 2, max_batch=4096)
    q, k, v, qs, ks = case(2, 2, n, n, seed=1, pad=0)
    good, good_lse = run(pi, q, k, v, qs, ks)
    bad = list(ks)
    bad[at + 1] = ks[-1] + 1 if at + 1 == batch else ks[at] - 1                        # behind the tensor, or falling
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    pi.prompt_attn(q, k, v, i32(qs), out, k_start=i32(bad), lse=lse)
    torch.cuda.synchronize()
    got = pi.status()
    assert got[0] == -8 and got[1] == 8 and got[2] == at, got
    rows = torch.ones(q.shape[0], dtype=torch.bool)
    rows[qs[at]:qs[at + 1]] = False
    assert bool((out.cpu()[~rows] == 7).all())
    if at + 1 < batch:
        rows[qs[at + 1]:qs[at + 2]] = False                                            # the next one has other keys than before
    assert torch.equal(out.cpu()[rows], good.cpu()[rows]) and torch.equal(lse.cpu()[rows], good_lse.cpu()[rows])


def test_a_short_limit_of_the_waits_does_not_end_a_long_item():
    """Items of 938 K/V tiles, which take longer than the limit of a single wait: nothing stands still, so nothing is given up."""
    pi, short = context(16, 16), context(16, 16, wait_limit_us=500)
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn((t, 16, 128), generator=g, device="cuda", dtype=torch.bfloat16) for t in (1200, 120000, 120000))
    want, want_lse = run(pi, q, k, v, [0, 1200], [0, 120000])
    out, lse = run(short, q, k, v, [0, 1200], [0, 120000])
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    heads = [0, 15]
    check(q.dtype, out[-3:, heads], lse[-3:, heads], reference(q[-3:, heads], k[:, heads], v[:, heads], [0, 3], [0, 120000]))
