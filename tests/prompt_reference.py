"""Attention over packed prompts in 64 bits, sequence by sequence, with what its rounding may be off by."""
import math

import torch


def reference(q, k, v, q_start, k_start):
    """out, lse and the allowances' sizes, as float64 / numbers of q's rows: out [T][Hq][D], lse [T][Hq], and of each row and channel the weighted
    sum of |v| (`spread`), and of each row the number of keys over the sum of weights under the largest (`thin`)."""
    q, k, v = q.cpu().double(), k.cpu().double(), v.cpu().double()
    T, Hq, D = q.shape
    G = Hq // k.shape[1]
    out, lse = torch.zeros((T, Hq, D), dtype=torch.float64), torch.zeros((T, Hq), dtype=torch.float64)
    spread, thin, owned = torch.zeros_like(out), torch.zeros_like(out), torch.zeros(T, dtype=torch.bool)
    for s in range(len(q_start) - 1):
        a, b, c, d = q_start[s], q_start[s + 1], k_start[s], k_start[s + 1]
        n, m = b - a, d - c
        owned[a:b] = True
        seen = torch.arange(m)[None] <= torch.arange(n)[:, None] + m - n
        for h in range(Hq):
            kk, vv = k[c:d, h // G], v[c:d, h // G]
            z = (q[a:b, h] @ kk.T / math.sqrt(D)).masked_fill(~seen, -math.inf)
            if m == 0 or n == 0:
                lse[a:b, h] = -math.inf
                continue
            top = z.amax(-1, keepdim=True)
            p = torch.where(seen, torch.exp(z - top.clamp(min=-1e300)), 0.0)
            l = p.sum(-1, keepdim=True)
            some = l > 0
            lse[a:b, h] = torch.where(some, top + torch.log(l), -math.inf)[:, 0]
            w = torch.where(some, p / l.clamp(min=1e-300), 0.0)
            out[a:b, h] = w @ vv
            spread[a:b, h] = w @ vv.abs()
            thin[a:b, h] = torch.where(some, seen.sum(-1, keepdim=True) / l.clamp(min=1e-300), 0.0) * vv.abs().amax()
    return out, lse, spread, thin, owned


def allowance(dtype, out, spread, thin):
    """Half a step of the output's rounding; half a step of every weight's (weights below fp16's normal numbers: 2^-25 of the largest);
    and 2^-15 of the weighted sum of |v| for scores, exponentials and sums in 32 bits."""
    half = torch.finfo(dtype).eps / 2
    got = half * out.abs() + half * spread + 2.0 ** -15 * spread + 1e-30
    if dtype == torch.float16:
        got = got + 2.0 ** -25 * thin + 2.0 ** -25       # the output itself may be below its normal numbers
    return got


def check(dtype, got, lse, ref):
    out, want, spread, thin, owned = ref
    got = got.cpu().double()
    off = (got - out).abs()
    over = off[owned] / allowance(dtype, out, spread, thin)[owned]
    assert owned.sum() == 0 or float(over.max()) <= 1.0, float(over.max())
    if lse is not None:
        lse = lse.cpu().double()[owned]
        want = want[owned]
        none = torch.isinf(want)
        assert torch.equal(none, torch.isinf(lse)) and bool((lse[none] < 0).all())
        assert bool(((lse - want)[~none].abs() <= 2.0 ** -18 * (1 + want[~none].abs())).all())
