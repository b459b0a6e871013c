"""The mean-square check of kv4_accuracy on models of the kernel: it passes the arithmetic that the kernel has and fails less of it."""
import numpy as np
import pytest

from tests import kv4_accuracy as acc
from tests import kv4_reference as ref


def bits(x, n):
    """x rounded to n significant bits."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(np.ldexp(m, n)), e - n)


def model(kind, p, codes, s, lo):
    scale, low = np.repeat(s, 32, -1), np.repeat(lo, 32, -1)
    w = p * 37.3                                                     # unnormalised, as the kernel's are
    if kind == "zero":
        return np.zeros((p.shape[0], 128))
    if kind == "weights of 8 bits":
        w = bits(w, 8)
        return w @ (codes * scale + low) / w.sum(1, keepdims=True)
    if kind == "minima with weights of 8 bits":
        return (w @ (codes * scale) + bits(w, 8) @ low) / 37.3
    if kind == "half of the tokens twice":
        w = w * (1 + (np.arange(w.shape[1]) % 2 * 2 - 1) * 0.05)
        return w @ (codes * scale + low) / w.sum(1, keepdims=True)
    ws = np.stack([bits(w * s[:, j], 11) for j in range(4)])         # [group][G][tokens]
    middle = {"codes from 0": 0, "codes from the middle": 8}[kind]
    out = np.concatenate([ws[j] @ (codes[:, 32 * j:32 * j + 32] - middle) for j in range(4)], 1)
    return (out + bits(w, 16) @ (low + middle * scale)) / 37.3


@pytest.mark.parametrize("kind,passes", [("codes from the middle", True), ("codes from 0", False), ("zero", False), ("weights of 8 bits", False),
                                         ("minima with weights of 8 bits", False), ("half of the tokens twice", False)])
@pytest.mark.parametrize("n", [250, 1024, 4800])
def test_the_check_tells_the_kernels_arithmetic_from_less(kind, passes, n):
    rng = np.random.default_rng(n)
    got, want, before = [], [], []
    for _ in range(64):                                              # KV heads, of 8 query heads
        kv = ref.bf16(rng.standard_normal((2, n, 128)))
        (ck, sk, lk), (cv, sv, lv) = [[a.astype(np.float64) for a in ref.round_rows(kv[i])] for i in (0, 1)]
        p, _ = acc.softmax(ref.bf16(rng.standard_normal((8, 128))).astype(np.float64), ck, sk, lk)
        w, b = acc.allowed(p, cv, sv, lv)
        got.append(ref.bf16(model(kind, p, cv, sv, lv).astype(np.float32))), want.append(w), before.append(b)
    got, want, before = [np.stack(x) for x in (got, want, before)]
    if passes:
        acc.check(got, want, before)
    else:
        with pytest.raises(AssertionError):
            acc.check(got, want, before)


def test_parts_are_what_unpack_says():
    rng = np.random.default_rng(0)
    pool = ref.pack(ref.bf16(rng.standard_normal((5, 2, 2, 32, 128))), 32)
    c, s, lo = acc.parts(pool, 2, 32)
    assert np.array_equal(c * np.repeat(s, 32, -1) + np.repeat(lo, 32, -1), ref.unpack(pool, 2, 32))
    c, s, lo = acc.tokens(pool, [4, 0, 1], [0, 2, -1], 3, 70, 2, 32)
    assert c.shape == (2, 2, 38, 128) and s.shape == (2, 2, 38, 4)
    assert np.array_equal((c * np.repeat(s, 32, -1) + np.repeat(lo, 32, -1))[:, :, :32], ref.unpack(pool[4:5], 2, 32)[0])
