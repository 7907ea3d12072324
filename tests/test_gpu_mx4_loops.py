"""The operators on frozen rows at sizes where a workgroup goes round its loops several times: buffers in LDS change places, rows are loaded
ahead over the end of a stage, running maxima rise, and the last turn is short.  Against the definition in 64 bits, with the
tolerances of test_gpu_mx4.py; the sizes of the workspaces say how long the parts are, so that a retuned division shows here."""
import math

import numpy as np
import pytest
import torch

import paper_2003_05622_amd as hps
import mx4_reference as ref
from test_gpu_mx4 import check_gradient, check_logprobs, dev, make

pytestmark = pytest.mark.gpu


def held(rng, n, dim, spread=2):
    """Random codes with scales 2^0 to 2^spread: (Mx4Rows, values).  (Quantising many wide rows on the CPU takes too long.)"""
    codes = rng.integers(0, 256, size=(n, ref.row_bytes(dim)), dtype=np.uint8)
    codes[:, dim // 2:] = 0
    scales = rng.integers(124, 125 + spread, size=(n, -(-dim // 32)), dtype=np.uint8)
    return hps.Mx4Rows(dev(codes), dev(scales), dim), ref.values(codes, scales, dim)


def a_bias(rng, n):
    bias = rng.normal(size=n).astype(np.float32)
    bias[rng.random(n) < 0.1] = -np.inf
    return bias


def a_scale(dim, sign=1):
    """Scores of a standard deviation of about 2.5: codes have a mean square of 8.6 (scales not counted)."""
    return sign * 2.5 / (8.6 * math.sqrt(dim) * 0.25 * 0.25 * 2.5)


# (queries, rows, dim, parts, at least so many rows each): every kernel of the gradient, at several stages of 128 rows (64 where the
# waves share the rows): waves that split a stage four and two ways, four of them with a query tile each, with two
GRAD = [(1, 400003, 64, 300), (2, 300001, 16, 256), (40, 200003, 100, 300), (50, 140001, 36, 130), (130, 70001, 128, 200), (300, 70001, 64, 200),
        (260, 60001, 16, 200), (130, 40001, 256, 200), (100, 20011, 512, 128), (70, 20003, 1000, 128), (3, 20011, 1024, 128)]


@pytest.mark.parametrize("m,n,dim,rows_of_a_part", GRAD)
@pytest.mark.parametrize("biased,with_entropy", [(False, False), (True, True)])
def test_gradient_of_several_stages(m, n, dim, rows_of_a_part, biased, with_entropy):
    parts = hps.lib().hps_mx4_logprobs_backward_bytes(m, n, dim) // (4 * m * dim)
    assert n / parts >= rows_of_a_part
    rng = np.random.default_rng(m + n + dim)
    (q, qv), (r, rv) = held(rng, m, dim), held(rng, n, dim)
    given = rng.integers(-1, n + 1, size=(m, 3)).astype(np.int32)
    check_gradient(q, qv, r, rv, a_scale(dim), a_bias(rng, n) if biased else None, given, rng.normal(size=(m, 3)).astype(np.float32),
                   rng.normal(size=m).astype(np.float32) if with_entropy else None)


# (and the other two of the four kinds, for every width that has a kernel of its own)
@pytest.mark.parametrize("m,n,dim", [(5, 700, 8), (33, 900, 16), (300, 1500, 12), (3, 1000, 20), (300, 2000, 32), (40, 1100, 64), (300, 900, 64), (70, 700, 128),
                                     (70, 900, 256), (40, 700, 260), (70, 900, 512), (8, 500, 1000), (130, 700, 1024)])
@pytest.mark.parametrize("biased,with_entropy", [(True, False), (False, True)])
def test_gradient_of_a_bias_or_the_entropy_alone(m, n, dim, biased, with_entropy):
    rng = np.random.default_rng(m + n + dim)
    (q, qv), (r, rv) = held(rng, m, dim), held(rng, n, dim)
    given = rng.integers(-1, n + 1, size=(m, 3)).astype(np.int32)
    check_gradient(q, qv, r, rv, a_scale(dim, -1), a_bias(rng, n) if biased else None, given, rng.normal(size=(m, 3)).astype(np.float32),
                   rng.normal(size=m).astype(np.float32) if with_entropy else None)


# one and two query tiles a wave at several tiles of 32 rows, and waves that share them
LOG = [(1, 1500001, 8, 0, 250), (3, 1200007, 20, 5, 250), (33, 600011, 64, 3, 120), (70, 400003, 36, 0, 250), (300, 90001, 100, 8, 100),
       (130, 70001, 260, 0, 120), (130, 40001, 512, 4, 64), (100, 40003, 1024, 0, 36)]


@pytest.mark.parametrize("m,n,dim,top,rows_of_a_part", LOG)
@pytest.mark.parametrize("biased", [False, True])
def test_log_probabilities_of_several_tiles(m, n, dim, top, rows_of_a_part, biased):
    parts = hps.lib().hps_mx4_logprobs_bytes(m, n, dim, 0) // (12 * m)
    assert n / parts >= rows_of_a_part
    rng = np.random.default_rng(m + n + dim)
    (q, qv), (r, rv) = held(rng, m, dim), held(rng, n, dim)
    given = rng.integers(-1, n + 1, size=(m, 2)).astype(np.int32)
    check_logprobs(q, qv, r, rv, a_scale(dim, -1), a_bias(rng, n) if biased else None, given, top)


@pytest.mark.parametrize("dim", [64, 1024])
def test_maxima_that_rise_all_the_time(dim):
    """Rows in the order of their scores, either way: the running maximum rises with every tile, or never after the first."""
    rng = np.random.default_rng(dim)
    n = 40001
    q = rng.integers(0, 256, size=(1, ref.row_bytes(dim)), dtype=np.uint8)
    (r, rv) = held(rng, n, dim)
    scales = np.full((1, dim // 32), 126, dtype=np.uint8)
    qv = ref.values(q, scales, dim)
    order = np.argsort((qv @ rv.T)[0], kind="stable")
    for m in (1, 130):
        queries = hps.Mx4Rows(dev(np.repeat(q, m, axis=0)), dev(np.repeat(scales, m, axis=0)), dim)
        for way in (order, order[::-1]):
            rows = hps.Mx4Rows(dev(r.codes.cpu().numpy()[way]), dev(r.scales.cpu().numpy()[way]), dim)
            check_logprobs(queries, np.repeat(qv, m, axis=0), rows, rv[way], 2 * a_scale(dim), None, None, 5)


@pytest.mark.parametrize("m,n,dim", [(200, 100003, 260), (330, 60001, 1024), (500, 200003, 64), (70, 300001, 100)])
def test_scores_of_several_tiles_of_queries(m, n, dim):
    """A part of the queries alone gives the same bits, and these were compared with 64 bits elsewhere."""
    rng = np.random.default_rng(m + n)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m)
    q = hps.mx4_quantize(torch.randn((m, dim), generator=gen, device="cuda"))
    r = hps.mx4_quantize(torch.randn((n, dim), generator=gen, device="cuda"))
    bias = dev(a_bias(rng, n))
    for b in (None, bias):
        out = hps.mx4_scores(q, r, 0.3, b)
        narrow = hps.mx4_scores(q, r, 0.3, b, dtype=torch.bfloat16)
        for first in range(0, m, 23):
            part = q[first:first + 23]
            want = hps.mx4_scores(part, r, 0.3, b)
            assert torch.equal(out[first:first + 23], want) and torch.equal(narrow[first:first + 23], want.bfloat16())
        want = ref.scores(q.dequantize().double().cpu().numpy()[-9:], r.dequantize().double().cpu().numpy()[:2000], 0.3,
                          None if b is None else b.cpu().numpy()[:2000])
        got = out[-9:, :2000].double().cpu().numpy()
        near = np.isfinite(want)
        size = 0.3 * (np.abs(q.dequantize().double().cpu().numpy()[-9:]) @ np.abs(r.dequantize().double().cpu().numpy()[:2000]).T)
        assert np.array_equal(np.isfinite(got), near)
        assert np.all(np.abs(got[near] - want[near]) <= 2.0 ** -24 * (64 * size[near] + 2 * np.abs(want[near])))


# ---- sums that float32 does not hold ------------------------------------------------------------------
@pytest.mark.parametrize("m,n,dim,top", [(1, 3000, 64, 10), (5, 20000, 128, 64), (40, 5000, 260, 7), (70, 4000, 512, 20), (300, 3000, 96, 16), (130, 2500, 1024, 33),
                                         (3, 100001, 1000, 5)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("biased", [False, True])
def test_best_rows_where_sums_are_rounded(m, n, dim, top, sign, biased):
    """Scales that differ by 2^40 within a row: a score depends on the order in which its sum is rounded, and the scores that the groups are chosen by,
    those that the rows are chosen by and those of mx4_scores have to be the same numbers all the same."""
    rng = np.random.default_rng(m + n + dim)

    def wild(k):
        codes = rng.integers(0, 256, size=(k, ref.row_bytes(dim)), dtype=np.uint8)
        codes[:, dim // 2:] = 0
        return hps.Mx4Rows(dev(codes), dev(rng.integers(107, 128, size=(k, -(-dim // 32)), dtype=np.uint8)), dim)
    q, r = wild(m), wild(n)
    qv, rv = q.dequantize().double().cpu().numpy(), r.dequantize().double().cpu().numpy()
    exact = (qv[:5] @ rv[:2000].T)
    assert (exact != exact.astype(np.float32)).mean() > 0.1          # (that is what this is about: with two blocks few sums, with more nearly all)
    bias = a_bias(rng, n) if biased else None
    scale = sign * 0.05
    check_logprobs(q, qv, r, rv, scale, bias, rng.integers(0, n, size=(m, 2)).astype(np.int32), top)
    s = hps.mx4_scores(q, r, scale, None if bias is None else dev(bias))
    left = torch.isfinite(s).sum(1)
    got = hps.mx4_logprobs(q, r, None, top, scale, None if bias is None else dev(bias))
    assert ((got.top_index >= 0).sum(1) == torch.clamp(left, max=top)).all()


def test_gradient_with_a_very_large_scale():
    """Scores up to some millions: one row has all of the probability (where the next score is near, p depends on how lse was rounded)."""
    rng = np.random.default_rng(12)
    (q, qv), (r, rv) = make(rng, 40, 64), make(rng, 900, 64, 0.1)
    given = rng.integers(-1, 900, size=(40, 2)).astype(np.int32)
    u, h = rng.normal(size=(40, 2)).astype(np.float32), rng.normal(size=40).astype(np.float32)
    check_gradient(q, qv, r, rv, 1e6, None, given, u, None)
    check_gradient(q, qv, r, rv, -1e6, None, given, u, h)
    check_gradient(q, qv, r, rv, 1e6, np.zeros(900, dtype=np.float32), given, u, h)
