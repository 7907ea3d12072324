"""Sums over the rows in which the errors of single terms cannot cancel: equal probabilities, few large ones, very many rows.

Tolerances, in H = 2^-24, relative to sum p |row|.  The reference takes the same float32 log-sum-exp, so its rounding does not count.
p: an exponential (2 H), a factor for what float32 does not hold of the exponent's parts, its exponential and its product (2 + 1 H).
The exponent itself is off by its rounding, H |s - lse| (with a bias twice, and its unit by H / 2 of it).  Three pieces of p are exact.  An instruction
adds 16 rows of one piece and is off by 2 H of the sum at most, one after the other in a part of the rows: 6 H / 16 a row.  Up to three
sums of waves are joined (3 H); parts are added in 64 bits.  Together T = 8 H + 3 H |s - lse| + 6 H ceil(rows / 16).
"""
import math

import numpy as np
import pytest
import torch

import paper_2003_05622_amd as hps
import mx4_reference as ref
from test_gpu_mx4 import dev, make

pytestmark = pytest.mark.gpu
H = 2.0 ** -24


def alike(n, dim):
    """n times the same row, and its values."""
    codes, scales, v = ref.quantize(np.random.default_rng(0).normal(size=(1, dim)).astype(np.float32))
    return hps.Mx4Rows(dev(np.repeat(codes, n, axis=0)), dev(np.repeat(scales, n, axis=0)), dim), v[0]


def zeros(m, dim):
    codes, scales, _ = ref.quantize(np.zeros((m, dim), dtype=np.float32))
    return hps.Mx4Rows(dev(codes), dev(scales), dim)


def rows_of_a_part(m, n, dim):
    """At most so many rows are added up one after the other in 32 bits: those of a part, of which the workspace has one sum for every query's value."""
    parts = hps.lib().hps_mx4_logprobs_backward_bytes(m, n, dim) // (4 * m * dim)
    return min(n, -(-(-(-n // parts)) // 128) * 128)


@pytest.mark.parametrize("m,dim", [(1, 16), (1, 64), (40, 128), (70, 300), (300, 64), (3, 1024)])
@pytest.mark.parametrize("biased", [False, True])
def test_equal_probabilities_add_up(m, dim, biased):
    """A query of zeros (no known keys) has p = 1 / n throughout: the gradient of a row's log probability is that row less the mean of all."""
    given, u = torch.zeros((m, 1), dtype=torch.int32, device="cuda"), torch.ones((m, 1), device="cuda")
    for n in list(range(2, 20)) + list(range(20, 400, 9)) + [1000, 1023, 1025, 4099]:
        rows, v = alike(n, dim)
        lse = np.float32(math.log(n))
        d = hps.mx4_logprobs_backward(zeros(m, dim), rows, given, u, torch.full((m,), float(lse), device="cuda"),
                                      bias=torch.zeros(n, device="cuda") if biased else None).cpu().numpy()
        want = v * (1 - n * math.exp(-float(lse)))
        t = H * (8 + 3 * math.log(n) + 6 * math.ceil(rows_of_a_part(m, n, dim) / 16))
        assert np.all(np.abs(d - want) <= t * np.abs(v) + 2 * H * np.abs(want)), (n, np.abs(d - want).max() / H)


@pytest.mark.parametrize("n", [2, 3, 7, 13, 24, 32, 47])
@pytest.mark.parametrize("dim", [8, 64, 260])
def test_few_rows_with_large_probabilities(n, dim):
    """Where every p is above 2^-6 all of its bits count."""
    rng = np.random.default_rng(n)
    for m in (1, 33, 70):
        (q, qv), (r, rv) = make(rng, m, dim, 0.3, 0.0), make(rng, n, dim, 0.3, 0.0)
        scale = np.float32(0.5 / math.sqrt(dim))
        s = ref.scores(qv, rv, scale)
        lse = np.log(np.exp(s).sum(axis=1)).astype(np.float32)
        p = np.exp(s - lse.astype(np.float64)[:, None])
        assert p.min() > 2.0 ** -7
        given = rng.integers(0, n, size=(m, 1)).astype(np.int32)
        u = np.ones((m, 1), dtype=np.float32)
        d = hps.mx4_logprobs_backward(q, r, dev(given), dev(u), dev(lse), scale=float(scale)).cpu().numpy()
        want = float(scale) * (rv[given[:, 0]] - p @ rv)
        deep = np.abs(s - lse[:, None]).max() + np.abs(s).max()           # (the product's unit: H of the score)
        t = H * (8 + 3 * deep + 6 * math.ceil(n / 16))
        assert np.all(np.abs(d - want) <= float(scale) * t * (p @ np.abs(rv)) + 2 * H * np.abs(want)), n


def test_two_probabilities_add_up():
    """Half of the rows have one bias, half another."""
    for n in range(70, 400, 11):
        rows, v = alike(n, 64)
        bias = np.where(np.arange(n) < n // 2, 0.0, 0.3).astype(np.float32)
        lse = np.float32(math.log(np.exp(bias.astype(np.float64)).sum()))
        p = np.exp(bias.astype(np.float64) - float(lse))
        d = hps.mx4_logprobs_backward(zeros(2, 64), rows, torch.full((2, 1), n - 1, dtype=torch.int32, device="cuda"), torch.ones((2, 1), device="cuda"),
                                      torch.full((2,), float(lse), device="cuda"), bias=dev(bias)).cpu().numpy()
        want = v * (1 - p.sum())
        t = H * (8 + 3 * (float(lse) + 0.3) + 6 * math.ceil(rows_of_a_part(2, n, 64) / 16))
        assert np.all(np.abs(d - want) <= t * np.abs(v) + 2 * H * np.abs(want)), (n, np.abs(d - want).max() / H)
