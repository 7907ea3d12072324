"""Sums over the rows in which the errors of single terms cannot cancel: equal probabilities, few large ones, very many rows.

Tolerances, in H = 2^-24, relative to sum p |row|.  The reference takes the same float32 log-sum-exp, so its rounding does not count.
p: an exponential (2 H), a factor for what float32 does not hold of the exponent's parts, its exponential and its product (2 + 1 H).
The exponent itself is off by its rounding, H |s - lse| (with a bias twice, and its unit by H / 2 of it).  Three pieces of p are exact.  An instruction
adds 16 rows of one piece and is off by 2 H of the sum at most, one after the other in a part of the rows: 6 H / 16 a row.  Up to three
sums of waves are joined (3 H); parts are added in 64 bits, and so is what a long part has for every 4096 rows.  Together T = 8 H + 3 H |s - lse| + 6 H ceil(rows / 16).

Log-sum-exp and entropy: exponentials are off by 3 H |s - m| + 2 H; a lane adds up its 16 rows of a tile (9 additions), 128 tiles
one after the other (the rest in 64 bits), and some 40 sums of lanes, waves and parts follow: R = 180 H + 3 H |s - m|, and the roundings of lse's own size.
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
    return min(n, 4096, -(-(-(-n // parts)) // 128) * 128)


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


@pytest.mark.parametrize("scale", [2.0 ** -60, 1e-20, -1e-12])
def test_equal_probabilities_of_different_products(scale):
    """A scale next to nothing: the rows differ, their probabilities do not.  (The gradient has the scale as a factor, which is divided out.)"""
    for n in list(range(66, 400, 13)) + [1025]:
        rng = np.random.default_rng(n)
        (q, _), (r, rv) = make(rng, 2, 64), make(rng, n, 64, 0.1, 0.0)
        rv = np.abs(rv)
        r.codes.bitwise_and_(0x77)    # (no signs: the mean of the rows is as large as they are)
        lse = np.float32(math.log(n))
        d = hps.mx4_logprobs_backward(q, r, torch.zeros((2, 1), dtype=torch.int32, device="cuda"), torch.ones((2, 1), device="cuda"),
                                      torch.full((2,), float(lse), device="cuda"), scale=scale).cpu().numpy().astype(np.float64)
        held = float(np.float32(scale))
        p = math.exp(-float(lse))
        want = rv[0] - p * rv.sum(axis=0)
        t = H * (8 + 3 * math.log(n) + 6 * math.ceil(rows_of_a_part(2, n, 64) / 16))
        assert np.all(np.abs(d / held - want) <= t * p * rv.sum(axis=0) + 3 * H * np.abs(want)), n


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


# (queries, rows, dim): so many queries that one part holds all of the rows, or nearly; waves that hold two query tiles and one, and waves that share the rows
LONG = [(131072, 300007, 16), (131077, 70001, 64), (65540, 40001, 128), (32768, 20011, 300), (8200, 16385, 1024), (8200, 20480, 1000)]


@pytest.mark.parametrize("m,n,dim", LONG)
@pytest.mark.parametrize("biased", [False, True])
def test_very_many_rows_in_one_part(m, n, dim, biased):
    # (8 bytes of workspace for each value of a query: one part, in 64 bits)
    assert hps.lib().hps_mx4_logprobs_backward_bytes(m, n, dim) <= 8 * m * dim + 256
    given, u = torch.zeros((m, 1), dtype=torch.int32, device="cuda"), torch.ones((m, 1), device="cuda")
    rows, v = alike(n, dim)
    lse = np.float32(math.log(n))
    q = zeros(1, dim)
    q = hps.Mx4Rows(q.codes.repeat(m, 1), q.scales.repeat(m, 1), dim)
    d = hps.mx4_logprobs_backward(q, rows, given, u, torch.full((m,), float(lse), device="cuda"),
                                  bias=torch.zeros(n, device="cuda") if biased else None)
    assert torch.equal(d, d[:1].expand(m, dim))
    d = d[0].cpu().numpy()
    want = v * (1 - n * math.exp(-float(lse)))
    t = H * (8 + 3 * math.log(n) + 6 * 4096 / 16)
    assert np.all(np.abs(d - want) <= t * np.abs(v) + 2 * H * np.abs(want)), np.abs(d - want).max() / H


@pytest.mark.parametrize("m,n,dim", [(65600, 40011, 64), (33000, 20011, 260), (65536, 4097, 16)])
@pytest.mark.parametrize("kind", ["plain", "entropy", "biased"])
def test_long_parts_give_what_short_ones_give(m, n, dim, kind):
    """Some of many queries against the same ones alone, whose parts are short."""
    rng = np.random.default_rng(n)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    q = hps.mx4_quantize(torch.randn((m, dim), generator=gen, device="cuda"))
    r = hps.mx4_quantize(0.1 * torch.randn((n, dim), generator=gen, device="cuda"))
    scale = 20 / math.sqrt(dim)
    bias = None
    if kind == "biased":
        bias = torch.randn(n, generator=gen, device="cuda")
        bias[dev(rng.random(n) < 0.2)] = float("-inf")
    given = torch.randint(-1, n, (m, 2), generator=gen, device="cuda", dtype=torch.int32)
    u = torch.randn((m, 2), generator=gen, device="cuda")
    h = None if kind == "plain" else torch.randn(m, generator=gen, device="cuda")
    parts = [(0, 40), (m // 2 - 5, m // 2 + 30), (m - 33, m)]
    outs = [hps.mx4_logprobs(q[a:b], r, given[a:b], 0, scale, bias) for a, b in parts]
    lse, entropy = torch.zeros(m, device="cuda"), torch.zeros(m, device="cuda")
    for (a, b), out in zip(parts, outs):
        lse[a:b], entropy[a:b] = out.lse, out.entropy
    d = hps.mx4_logprobs_backward(q, r, given, u, lse, entropy, h, scale, bias)
    most = r.dequantize().abs().max().item()
    for (a, b), out in zip(parts, outs):
        want = hps.mx4_logprobs_backward(q[a:b], r, given[a:b], u[a:b], out.lse, out.entropy, None if h is None else h[a:b], scale, bias)
        # |c| sums up to |U| + |h| sum p |log p + H| <= |U| + 2 |h| H; sums of 4096 rows are off by 6 H / 16 a row, of pieces 2^-17 may be left out
        size = u[a:b].abs().sum(1) + (2 * h[a:b].abs() * out.entropy if h is not None else 0.0)
        off = abs(scale) * most * size * (2 * 6 * H * 4096 / 16 + 2 * 2.0 ** -17)
        assert ((d[a:b] - want).abs() <= off[:, None]).all()


def test_very_many_given_rows():
    """Their gradients are added up in 64 bits, with a gradient of the entropy as without."""
    m, n, dim, g = 3, 40, 64, 300001
    rng = np.random.default_rng(5)
    (q, qv), (r, rv) = make(rng, m, dim, 0.3, 0.0), make(rng, n, dim, 0.3, 0.0)
    out = hps.mx4_logprobs(q, r, scale=0.1)
    given = rng.integers(0, n, size=(m, g)).astype(np.int32)
    u = np.full((m, g), 0.1, dtype=np.float32)
    s = ref.scores(qv, rv, 0.1)
    p = np.exp(s - out.lse.cpu().numpy().astype(np.float64)[:, None])
    total = g * float(np.float32(0.1))
    c = -total * p
    for i in range(m):
        np.add.at(c[i], given[i], float(np.float32(0.1)))
    want = float(np.float32(0.1)) * (c @ rv)
    t = H * (8 + 3 * (np.abs(s).max() + math.log(n)) + 6 * math.ceil(n / 16) + 2)
    off = 0.1 * total * t * (p @ np.abs(rv)) + 2 * H * np.abs(want)
    for h in (None, torch.zeros(m, device="cuda")):
        d = hps.mx4_logprobs_backward(q, r, dev(given), dev(u), out.lse, out.entropy, h, scale=0.1).cpu().numpy()
        assert np.all(np.abs(d - want) <= off), np.max(np.abs(d - want) / off)


@pytest.mark.parametrize("m,n,dim", [(32800, (1 << 24) + 77, 8), (16500, (1 << 24) + 33, 260)])
@pytest.mark.parametrize("biased", [False, True])
def test_log_probabilities_of_very_many_rows(m, n, dim, biased):
    """Eight parts of two million rows: one term's worth of sums after the other that never is a whole number of anything."""
    rows = hps.Mx4Rows.empty(n, dim, "cuda")
    rows.codes.zero_()
    rows.scales.fill_(127)
    queries = hps.Mx4Rows.empty(m, dim, "cuda")
    queries.codes.fill_(0x22)
    queries.scales.fill_(127)
    scale = 0.28
    # (8 parts, 12 bytes a query each)
    assert hps.lib().hps_mx4_logprobs_bytes(m, n, dim, 0) <= 8 * 12 * m + 256
    for every in (64, 1000):
        # the first two values of a row are a half, of every so many rows 1
        rows.codes[:, 0] = 0x11
        rows.codes[::every, 0] = 0x22
        out = hps.mx4_logprobs(queries, rows, None, 0, scale, torch.zeros(n, device="cuda") if biased else None)
        assert (out.lse == out.lse[0]).all() and (out.entropy == out.entropy[0]).all()
        low = float(np.float32(scale))
        high, k = 2 * low, -(-n // every)
        l = k * math.exp(high) + (n - k) * math.exp(low)
        lse, entropy = math.log(l), math.log(l) - (k * math.exp(high) * high + (n - k) * math.exp(low) * low) / l
        r = H * (180 + 3 * low)
        assert abs(float(out.lse[0]) - lse) <= r + 4 * H * lse
        assert abs(float(out.entropy[0]) - entropy) <= 2 * r * (1 + low) + 8 * H * entropy


def test_long_parts_captured_and_on_two_streams():
    """Several launches add up in one workspace: replays with new inputs, and two such calls at once, give what a call alone gives."""
    m, n, dim = 66000, 70001, 32
    gen = torch.Generator(device="cuda")

    def inputs(seed):
        gen.manual_seed(seed)
        q = hps.mx4_quantize(torch.randn((m, dim), generator=gen, device="cuda"))
        r = hps.mx4_quantize(torch.randn((n, dim), generator=gen, device="cuda"))
        given = torch.randint(0, n, (m, 1), generator=gen, device="cuda", dtype=torch.int32)
        return q, r, given, torch.randn((m, 1), generator=gen, device="cuda")

    def both(q, r, given, u):
        out = hps.mx4_logprobs(q, r, given, 0, 0.3)
        return out.lse, hps.mx4_logprobs_backward(q, r, given, u, out.lse, out.entropy, scale=0.3)
    assert hps.lib().hps_mx4_logprobs_backward_bytes(m, n, dim) <= 8 * m * dim + 256
    held = inputs(0)
    other = inputs(100)
    want_other = both(*other)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both(*held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(*held)
    for turn in range(3):
        for to, of in zip(held, inputs(turn + 1)):
            if isinstance(to, hps.Mx4Rows):
                to.codes.copy_(of.codes)
                to.scales.copy_(of.scales)
            else:
                to.copy_(of)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            at_once = both(*other)
        torch.cuda.synchronize()
        want = both(*held)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(at_once[0], want_other[0]) and torch.equal(at_once[1], want_other[1])
