"""The arithmetic of sample's weights, replayed in 32 bits with the kernel's own table and numbers, against the weights'
definition: within the 2^-30 that the operator promises (host side; no GPU needed)."""
import os
import re

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
f32, long = np.float32, np.longdouble


def numbers():
    """(table's fp32 numbers, what log2 of them is short of, MAGIC, the series' coefficients from r^3 down)."""
    src = open(os.path.join(ROOT, "paper_2601_08670_gb300", "csrc", "sample.cuh")).read()
    table = re.search(r"kExp2Table\[SMP_EXP2\] = \{(.*?)\};", src, re.S).group(1)
    rows = re.findall(r"\{0x([0-9A-F]{8})u, (\S+?)f\}", table)
    of = re.search(r"void of\(.*?\n  \}\n", src, re.S).group(0)
    magic = float(re.search(r"MAGIC = ([0-9.]+)f", of).group(1))
    series = [f32(x) for x in re.findall(r"([0-9.]+e-[0-9]+)f", of)]
    assert len(rows) == 64 and magic == 1.5 * 2 ** 17 and len(series) == 3
    return (np.array([int(r[0], 16) for r in rows], np.uint32).view(f32), np.array([r[1] for r in rows], f32), f32(magic),
            series)


def fma(a, b, c):
    return (a.astype(long) * np.asarray(b, f32).astype(long) + np.asarray(c, f32).astype(long)).astype(f32)


def weights(x, t):
    hi, rest, magic, (c3, c2, c1) = numbers()
    lh, ll = f32(1.44269502), f32(1.92596303e-08)
    ch = lh / t
    cl = (fma(-ch[None], t, lh)[0] + ll) / t
    p = x * ch
    low = fma(x, cl, fma(x, ch, -p))
    whole = (p + magic) - magic
    q = np.rint(whole.astype(np.float64) * 64).astype(np.int64)
    r = (p - whole) + (low + rest[q % 64])
    g = r * fma(r, fma(r, c3, c2), c1)
    return hi[q % 64].astype(long) * np.exp2((q // 64).astype(long)) * (1 + g.astype(long))


def test_the_table():
    hi, rest, _, _ = numbers()
    want = np.exp2(np.arange(64, dtype=long) / 64)
    assert np.array_equal(hi, want.astype(f32))
    assert np.abs(np.log2(want / hi.astype(long)) - rest.astype(long)).max() < 2.0 ** -47


@pytest.mark.parametrize("t", [1.0, 0.37, 0.7, 1.3, 0.01, 30.0])
@pytest.mark.parametrize("size", [1.0, 4.0, 60.0])
def test_weights(t, size):
    t = f32(t)
    x = np.random.default_rng(int(size)).normal(0, size, 300_000).astype(f32)
    x = x[np.abs(x) / t < 5000]  # (2^y as a long double has no larger y; |y| counts up to 8192)
    y = x.astype(long) / long(t)
    assert float(np.abs(weights(x, t) / np.exp(y) - 1).max()) <= 2.0 ** -30
