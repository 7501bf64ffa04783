"""Codes of values in the middle between two integers, and what a pass from rows to results makes of them.  Half of a row's
largest value is such a middle, 63.5, and common among bf16 values: the even integer is 64.  A quotient formed as
x * (127 / top) misses it, in 64 bits too, so the values here are whole numbers and fractions."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2304_09590_amd import pnn

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def code(x, top):
    """The integer nearest to 127 x / top, ties to even."""
    return round(127 * Fraction(x) / Fraction(top))


def rows(width, seed=0):
    """A row for each of bf16's 128 numbers from 1 to 2: the largest value that number, a third of the others its half."""
    g = np.random.default_rng(seed)
    top = 1 + np.arange(128) / 128
    x = np.trunc(g.random((128, width)) * 128) / 128 * g.choice([-1, 1], (128, width))  # (8 bits, at most 1)
    half = g.random((128, width)) < 1 / 3
    x = np.where(half, np.sign(x + 0.5 ** 20) * top[:, None] / 2, x)
    x[:, g.integers(width)] = top
    scale = 2.0 ** g.integers(-40, 40, 128)
    return x * scale[:, None]


def test_the_middle_is_a_middle():
    """127 (top / 2) / top is 63.5 for every top, and a product with the rounded 127 / top is not."""
    assert all(code(Fraction(128 + t, 256), Fraction(128 + t, 128)) == 64 for t in range(128))
    top = 1 + np.arange(128) / 128
    missed = np.rint((top / 2) * (127 / top)) != 64
    assert 0 < missed.sum() < 128


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [3, 48, 500, 1500, 3000, 5000])
def test_codes_of_middles(width, dtype):
    x = rows(width)
    t = torch.from_numpy(x).to(dtype)
    assert torch.equal(t.double(), torch.from_numpy(x))
    q, _ = pnn.quantize_rows(t.cuda())
    top = np.abs(x).max(1)
    near = {}
    want = np.array([[near.setdefault((v, m), code(v, m)) for v in r] for r, m in zip(x.tolist(), top.tolist())])
    assert np.array_equal(q.cpu().numpy()[:, :width], want) and (q[:, width:] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k,K,I,O", [(1, 64, 48, 33), (2, 3, 48, 70), (2, 2, 2048, 40), (1, 1, 1024, 513)])
def test_results_of_middles(k, K, I, O, dtype):
    """The whole pass against 64 bits: a code that went to the wrong side would show, 2^-24 of a result does not."""
    x = rows(I, seed=1)
    g = np.random.default_rng(2)
    w = g.integers(-127, 128, (K, O, I)).astype(np.int8)
    ws = (g.random((K, O)) * 0.01).astype(np.float32)
    ids = g.integers(0, K, (128, k)).astype(np.int32)
    q, s = pnn.quantize_rows(torch.from_numpy(x).to(dtype).cuda())
    got = pnn.grouped_forward_int8(pnn.group_rows(torch.from_numpy(ids).cuda(), K), q, s, torch.from_numpy(w).cuda(), torch.from_numpy(ws).cuda())
    top = np.abs(x).max(1)
    near = {}
    codes = np.array([[near.setdefault((v, m), code(v, m)) for v in r] for r, m in zip(x.tolist(), top.tolist())], dtype=np.int64)
    e, r = ids.reshape(-1), np.arange(128 * k) // k
    want = np.stack([w[a].astype(np.int64) @ codes[b] for a, b in zip(e, r)]) * (top / 127)[r][:, None] * ws[e].astype(np.float64)
    # the scale's rounding, the sum's, two products
    assert (np.abs(got.double().cpu().numpy() - want) <= 4 * U * np.abs(want)).all()
