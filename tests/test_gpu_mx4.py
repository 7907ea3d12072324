"""The operators on frozen rows (include/hps_mx4.h) on the GPU, against their definition in 64 bits.

Tolerances.  A float32 operation is off by at most H = 2^-24 of its result.  A product of a query with a row is a sum
over at most 32 blocks, so it is off by at most 64 H of the sum of the products' magnitudes A (twice the number of
additions of blocks); a score adds one rounding: E = H (64 |scale| A + 2 |score|).  A sum of exponentials: the exponent
is off by E and three roundings of its size, the exponential by 2 H, and at most 256 additions and
joins follow: R = max E + 3 H max|s - m| + 300 H, relative.  lse is off by R, and by the roundings of its own size.
"""
import ctypes

import numpy as np
import pytest
import torch

import paper_2003_05622_amd as hps
import mx4_reference as ref

pytestmark = pytest.mark.gpu
H = 2.0 ** -24


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def make(rng, n, dim, size=1.0, spread=0.5):
    """Held rows: (Mx4Rows, the float64 values they stand for)."""
    x = (rng.normal(size=(n, dim)) * size * np.exp(spread * rng.normal(size=(n, 1)))).astype(np.float32)
    codes, scales, v = ref.quantize(x)
    return hps.Mx4Rows(dev(codes), dev(scales), dim), v


def score_error(q, r, scale, s):
    with np.errstate(all="ignore"):
        return H * (64 * abs(scale) * (np.abs(q) @ np.abs(r).T) + 2 * np.where(np.isfinite(s), np.abs(s), 0.0))


# ---- the form ------------------------------------------------------------------------------------
DIMS = [4, 8, 12, 16, 20, 28, 32, 36, 60, 64, 96, 100, 260, 1000, 1024]


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("bf16", [False, True])
def test_quantize_gives_the_nearest_codes(dim, bf16):
    rng = np.random.default_rng(dim)
    for n in (1, 2, 63, 257):
        x = (rng.normal(size=(n, dim)) * np.exp(3 * rng.normal(size=(n, 1)))).astype(np.float32)
        x[rng.random(x.shape) < 0.1] = 0.0
        x[n // 2] = 0.0
        wide = dim + 4 * int(rng.integers(0, 3))
        t = torch.zeros((n, wide), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
        t[:, :dim] = dev(x)
        codes, scales, v = ref.quantize(t[:, :dim].float().cpu().numpy())
        rows, rounded = hps.mx4_quantize(t[:, :dim], values=True)
        assert np.array_equal(rows.scales.cpu().numpy(), scales)
        assert np.array_equal(rows.codes.cpu().numpy(), codes)
        assert np.array_equal(rounded.cpu().numpy(), v.astype(np.float32))
        assert np.array_equal(rows.dequantize().cpu().numpy(), v.astype(np.float32))
        again = hps.mx4_quantize(t[:, :dim])
        assert torch.equal(again.codes, rows.codes) and torch.equal(again.scales, rows.scales)


def test_quantize_at_the_borders():
    """Values on and next to the borders between codes, the smallest and largest magnitudes, what is not finite."""
    borders = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7], dtype=np.float32)
    near = np.concatenate([borders, np.nextafter(borders, np.float32(9)), np.nextafter(borders, np.float32(-9))])
    near = np.concatenate([near, -near])
    near = near[np.abs(near) < 8]
    x = []
    for e in (-149, -140, -130, -127, -126, -125, -60, 0, 60, 124, 125):
        for i in range(0, near.size, 31):
            part = np.zeros(32)
            got = near[i:i + 31].astype(np.float64)
            part[:got.size] = got
            part[31] = 4.0                     # the largest power of two in the block
            part[np.abs(part) >= 8] = 0
            with np.errstate(over="ignore"):
                x.append((part * 2.0 ** e).astype(np.float32))
    x = np.array(x)
    x = np.concatenate([x, np.zeros((4, 32), np.float32)])
    x[-1, 3], x[-2, 5], x[-3, 31] = np.nan, np.inf, -np.inf
    assert np.isfinite(x[:-3]).all()
    codes, scales, v = ref.quantize(x)
    rows, rounded = hps.mx4_quantize(dev(x), values=True)
    assert np.array_equal(rows.scales.cpu().numpy(), scales)
    assert np.array_equal(rows.codes.cpu().numpy(), codes)
    assert np.array_equal(rounded.cpu().numpy(), v.astype(np.float32), equal_nan=True)
    assert np.array_equal(rows.dequantize().cpu().numpy(), v.astype(np.float32), equal_nan=True)


def test_quantize_leaves_the_rest_alone():
    """Nothing is written behind the last row, and nothing between rows that lie apart is read as a value."""
    dim, n = 36, 33
    rng = np.random.default_rng(1)
    x = torch.full((n, 44), float("nan"), device="cuda")
    x[:, :dim] = dev(rng.normal(size=(n, dim)).astype(np.float32))
    codes = torch.full((n + 1, 32), 0xAB, dtype=torch.uint8, device="cuda")
    scales = torch.full((n * 2 + 3,), 0xCD, dtype=torch.uint8, device="cuda")
    rounded = torch.full((n * dim + 4,), 7.0, device="cuda")
    st = hps.lib().hps_mx4_quantize(x.data_ptr(), 0, n, dim, 44, codes.data_ptr(), scales.data_ptr(), rounded.data_ptr(),
                                    torch.cuda.current_stream().cuda_stream)
    assert st == hps.OK
    want = ref.quantize(x[:, :dim].cpu().numpy())
    assert np.array_equal(codes[:n].cpu().numpy(), want[0]) and (codes[n] == 0xAB).all()
    assert np.array_equal(scales[:2 * n].cpu().numpy().reshape(n, 2), want[1]) and (scales[2 * n:] == 0xCD).all()
    assert np.array_equal(rounded[:n * dim].cpu().numpy().reshape(n, dim), want[2].astype(np.float32)) and (rounded[n * dim:] == 7).all()


@pytest.mark.parametrize("dim", [4, 8, 16, 20, 32, 64, 100, 260])
@pytest.mark.parametrize("row_format", [hps.ROWS_F32, hps.ROWS_BF16, hps.ROWS_F32_WIDE])
def test_get_is_get_followed_by_quantize(dim, row_format):
    rng = np.random.default_rng(dim)
    t = hps.HpsTable(4000, dim, 4096, 4096, row_format=row_format, init_seed=3)
    keys = dev(rng.permutation(6000).astype(np.int64) * 977 + 5)
    t.insert(keys[:3000])
    t.insert(keys[:100], dev((rng.normal(size=(100, dim)) * 10).astype(np.float32)))
    for n in (0, 1, 63, 64, 65, 1000):
        asked = keys[torch.from_numpy(rng.integers(0, 6000, n)).cuda()].contiguous()
        rows, found = t.get_mx4(asked)
        w, _, f = t.get(asked)
        want = hps.mx4_quantize(w)
        assert torch.equal(found, f)
        assert torch.equal(rows.codes, want.codes) and torch.equal(rows.scales, want.scales)
    assert t.stats().size == 3000            # nothing was created


def test_get_gives_zeros_while_the_status_is_set():
    t = hps.HpsTable(100, 16, 64, 64)
    t.insert(dev(np.arange(1, 51, dtype=np.int64)))
    t.insert(dev(np.array([-1], dtype=np.int64)))        # the reserved key
    rows, found = t.get_mx4(dev(np.arange(1, 11, dtype=np.int64)))
    assert not found.any() and (rows.codes == 0).all() and (rows.scales == 0).all()
    t.clear_error()
    _, found = t.get_mx4(dev(np.arange(1, 11, dtype=np.int64)))
    assert found.all()


# ---- scores --------------------------------------------------------------------------------------
SHAPES = [(1, 1, 4), (1, 1000, 8), (3, 33, 12), (33, 31, 16), (32, 32, 20), (5, 4097, 32), (65, 129, 36), (31, 500, 64), (64, 256, 64),
          (100, 63, 100), (17, 300, 128), (7, 65, 260), (40, 96, 512), (2, 200, 1000), (130, 140, 1024), (1, 70000, 64), (300, 2, 64),
          (257, 1025, 96)]


@pytest.mark.parametrize("m,n,dim", SHAPES)
@pytest.mark.parametrize("biased", [False, True])
def test_scores(m, n, dim, biased):
    rng = np.random.default_rng(m * 7 + n + dim)
    (q, qv), (r, rv) = make(rng, m, dim), make(rng, n, dim, 0.1)
    scale = float(rng.choice([1.0, -0.37, 3.0, 0.1]))
    bias = None
    if biased:
        bias = rng.normal(size=n).astype(np.float32)
        bias[rng.random(n) < 0.2] = rng.choice([-np.inf, np.inf, np.nan])
        bias[rng.random(n) < 0.1] = np.finfo(np.float32).min
    want = ref.scores(qv, rv, scale, bias)
    off = score_error(qv, rv, scale, want)
    got = hps.mx4_scores(q, r, scale, None if bias is None else dev(bias)).cpu().numpy()
    out = np.isneginf(want)
    assert np.array_equal(np.isneginf(got), out)
    assert np.all(np.abs(np.where(out, 0, got.astype(np.float64) - np.where(out, 0, want))) <= off)
    # bfloat16 is the float32 score rounded once more, to the nearest; wider rows keep what lies between them
    wide = torch.full((m, n + 3), 5.0, dtype=torch.bfloat16, device="cuda")
    hps.mx4_scores(q, r, scale, None if bias is None else dev(bias), out=wide[:, :n])
    assert torch.equal(wide[:, :n], torch.from_numpy(got).cuda().bfloat16())
    assert (wide[:, n:] == 5).all()


def test_scores_are_exact_where_sums_are():
    """Scales of one size: every product and sum fits float32, whatever the order of the additions."""
    rng = np.random.default_rng(0)
    for dim in (4, 16, 64, 100, 1024):
        q = ref.quantize(rng.integers(-6, 7, size=(40, dim)).astype(np.float32))
        r = ref.quantize(rng.integers(-6, 7, size=(333, dim)).astype(np.float32))
        got = hps.mx4_scores(hps.Mx4Rows(dev(q[0]), dev(q[1]), dim), hps.Mx4Rows(dev(r[0]), dev(r[1]), dim))
        assert np.array_equal(got.cpu().numpy(), (q[2] @ r[2].T).astype(np.float32))


def test_parts_of_rows_and_nan_blocks():
    """A range of a catalogue starts at any row (scales at any byte); a block that stands for NaN reaches its row's scores alone."""
    rng = np.random.default_rng(2)
    for dim in (4, 12, 36, 100):
        (q, qv), (r, rv) = make(rng, 9, dim), make(rng, 200, dim)
        for first, last in ((1, 200), (3, 130), (37, 38), (5, 5)):
            got = hps.mx4_scores(q[1:8], r[first:last]).cpu().numpy()
            want = ref.scores(qv[1:8], rv[first:last], 1.0)
            assert got.shape == want.shape and np.all(np.abs(got - want) <= score_error(qv[1:8], rv[first:last], 1.0, want))
        r.scales[50, 0] = 255
        got = hps.mx4_scores(q, r)
        assert torch.isnan(got[:, 50]).all() and torch.isnan(got).sum() == 9
        bias = torch.zeros(200, device="cuda")
        bias[50] = float("-inf")
        assert (hps.mx4_scores(q, r, bias=bias)[:, 50] == float("-inf")).all()


# ---- log probabilities ---------------------------------------------------------------------------
def check_logprobs(q, qv, r, rv, scale, bias, given, top):
    got = hps.mx4_logprobs(q, r, None if given is None else dev(given), top, scale, None if bias is None else dev(bias))
    want = ref.log_probs(qv, rv, scale, bias, given=given)
    s = want["scores"]
    m, n = s.shape
    e = np.where(np.isneginf(s), 0, score_error(qv, rv, scale, s)).max(axis=1, initial=0)
    with np.errstate(all="ignore"):
        # how far a score that counts (by more than 2^-40) lies below the highest
        deep = np.where(s - s.max(axis=1, initial=-np.inf, keepdims=True) > -30, s.max(axis=1, initial=-np.inf, keepdims=True) - s, 0)
        deep = np.nan_to_num(deep).max(axis=1, initial=0)
        empty = np.isneginf(want["lse"])
        off = e + 3 * H * deep + 300 * H
        lse, entropy = got.lse.cpu().numpy().astype(np.float64), got.entropy.cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isneginf(lse), empty)
        lse_off = off + 4 * H * np.abs(want["lse"])
        assert np.all(np.where(empty, 0, np.abs(lse - want["lse"]) <= lse_off) + empty)
        # entropy = log l - e / l: each of the two is as far off as lse, the second times how deep its terms lie
        assert np.all(np.abs(entropy - want["entropy"]) <= 2 * off * (1 + deep) + 8 * H * (1 + np.log(max(n, 1))))
        if given is not None:
            logp, w = got.logp.cpu().numpy().astype(np.float64), want["logp"]
            assert np.array_equal(np.isnan(logp), np.isnan(w)) and np.array_equal(np.isneginf(logp), np.isneginf(w))
            near = np.isfinite(w)
            assert np.all(np.abs(logp - w)[near] <= (lse_off[:, None] + e[:, None] + 4 * H * np.abs(w))[near])
    if top:
        # the order is that of the scores as float32, which hps_mx4_scores gives too
        f = hps.mx4_scores(q, r, scale, None if bias is None else dev(bias)).cpu().numpy()
        order = np.argsort(-f, axis=1, kind="stable")[:, :top]
        v = np.take_along_axis(f, order, axis=1)
        left = ~np.isneginf(v)
        index = np.full((m, top), -1)
        index[:, :order.shape[1]][left] = order[left]
        assert np.array_equal(got.top_index.cpu().numpy(), index)
        best = got.top_logp.cpu().numpy().astype(np.float64)
        w = np.full((m, top), -np.inf)
        w[:, :order.shape[1]] = np.where(left, v - np.where(empty, 0, want["lse"])[:, None], -np.inf)
        assert np.array_equal(np.isneginf(best), np.isneginf(w))
        near = np.isfinite(w)
        assert np.all(np.abs(best - np.where(near, w, 0))[near] <= (lse_off[:, None] + 4 * H * np.abs(np.where(near, w, 0)))[near])
    return got


LOG_SHAPES = [(1, 1, 4, 1), (1, 2, 8, 3), (2, 31, 16, 64), (33, 32, 12, 8), (1, 33, 64, 1), (5, 1000, 64, 10), (32, 4097, 20, 16), (65, 700, 100, 64),
              (3, 65, 260, 5), (9, 3000, 128, 0), (1, 60000, 64, 16), (1, 50000, 8, 64), (2, 40001, 32, 50), (8, 30000, 1024, 8), (40, 5000, 36, 33),
              (200, 513, 16, 2), (1, 200000, 16, 64), (4, 99999, 64, 7), (129, 20000, 64, 16)]


@pytest.mark.parametrize("m,n,dim,top", LOG_SHAPES)
@pytest.mark.parametrize("biased", [False, True])
def test_logprobs(m, n, dim, top, biased):
    rng = np.random.default_rng(m + n + dim + top)
    (q, qv), (r, rv) = make(rng, m, dim), make(rng, n, dim, 0.1)
    scale = float(rng.choice([10, -20, 50])) / np.sqrt(dim)
    bias = None
    if biased:
        bias = rng.normal(size=n).astype(np.float32)
        bias[rng.random(n) < 0.3] = rng.choice([-np.inf, np.inf, np.nan])
        bias[rng.random(n) < 0.1] = np.finfo(np.float32).min
    given = rng.integers(-1, n + 1, size=(m, int(rng.choice([1, 2, 65])))).astype(np.int32)
    check_logprobs(q, qv, r, rv, scale, bias, given, top)


@pytest.mark.parametrize("scale", [1e-30, 0.0, 1.0, -1.0, 100.0])
def test_logprobs_of_equal_and_far_scores(scale):
    """Ties of all kinds: rows that come several times, and scores that differ by hundreds."""
    rng = np.random.default_rng(5)
    few = ref.quantize(rng.integers(-3, 4, size=(7, 32)).astype(np.float32))
    pick = rng.integers(0, 7, size=5000)
    r = hps.Mx4Rows(dev(few[0][pick]), dev(few[1][pick]), 32)
    q, qv = make(rng, 35, 32)
    q.codes[3] = 0                              # a query that is zero
    qv[3] = 0
    given = rng.integers(0, 5000, size=(35, 3)).astype(np.int32)
    check_logprobs(q, qv, r, few[2][pick], scale, None, given, 64)


@pytest.mark.parametrize("dim", [8, 64])
def test_logprobs_where_nothing_or_little_is_left(dim):
    rng = np.random.default_rng(6)
    (q, qv), (r, rv) = make(rng, 34, dim), make(rng, 3000, dim)
    low = np.finfo(np.float32).min
    for kind in ("none", "one", "last", "lowest", "lowest and one"):
        bias = np.full(3000, -np.inf, dtype=np.float32)
        bias[::3], bias[1::3] = np.nan, np.inf
        if kind == "one":
            bias[1234] = 0.5
        elif kind == "last":
            bias[2990:] = 0.0
        elif kind != "none":
            bias[100:2000] = low
            if kind == "lowest and one":
                bias[1500] = 1.0
        given = np.tile(np.array([0, 1234, 1500, 2999, 3000, -1, -2 ** 31, 2 ** 31 - 1], dtype=np.int32), (34, 1))
        check_logprobs(q, qv, r, rv, 0.5, bias, given, 20)
    # no rows, no queries
    got = hps.mx4_logprobs(q, r[5:5], dev(np.tile(np.array([[-1, 0]], dtype=np.int32), (34, 1))), 3)
    assert (got.lse == float("-inf")).all() and (got.entropy == 0).all() and (got.top_index == -1).all()
    assert (got.top_logp == float("-inf")).all() and (got.logp[:, 0] == 0).all() and torch.isnan(got.logp[:, 1]).all()
    got = hps.mx4_logprobs(q[3:3], r, torch.empty((0, 2), dtype=torch.int32, device="cuda"), 3)
    assert got.lse.shape == (0,) and got.top_index.shape == (0, 3)


def test_logprobs_with_a_nan_score():
    rng = np.random.default_rng(7)
    (q, _), (r, _) = make(rng, 40, 64), make(rng, 5000, 64)
    clean = hps.mx4_logprobs(q, r, top=8)
    at = int(clean.top_index[0, 0])
    r.scales[at, 1] = 255
    got = hps.mx4_logprobs(q, r, torch.full((40, 1), 3, dtype=torch.int32, device="cuda"), top=8)
    assert torch.isnan(got.lse).all() and torch.isnan(got.entropy).all() and torch.isnan(got.logp).all() and torch.isnan(got.top_logp).all()
    assert torch.equal(got.top_index[0, :7], clean.top_index[0, 1:])
    bias = torch.zeros(5000, device="cuda")
    bias[at] = float("nan")
    got = hps.mx4_logprobs(q, r, top=8, bias=bias)
    assert torch.isfinite(got.lse).all() and torch.equal(got.top_index[0, :7], clean.top_index[0, 1:])


# ---- gradient ------------------------------------------------------------------------------------
def check_gradient(q, qv, r, rv, scale, bias, given, u, h):
    b = None if bias is None else dev(bias)
    out = hps.mx4_logprobs(q, r, None if given is None else dev(given), 0, scale, b)
    got = hps.mx4_logprobs_backward(q, r, None if given is None else dev(given), None if u is None else dev(u), out.lse, out.entropy,
                                    None if h is None else dev(h), scale, b).cpu().numpy()
    want = ref.query_gradient(qv, rv, scale, bias, given, u, h)
    s = ref.scores(qv, rv, scale, bias)
    with np.errstate(all="ignore"):
        lse = ref.log_probs(qv, rv, scale, bias)["lse"]
        # (of all rows whose p float32 holds: a column in which the likely rows have zeros is made of the others)
        deep = np.where(s - lse[:, None] > -88, np.abs(s - lse[:, None]), 0)
        deep = np.nan_to_num(deep).max(axis=1, initial=0)
        e = np.where(np.isneginf(s), 0, score_error(qv, rv, scale, s)).max(axis=1, initial=0)
        p = np.where(np.isneginf(s), 0, np.exp(s - lse[:, None]))
    kept = rv if bias is None else np.where(np.isfinite(np.asarray(bias, dtype=np.float64))[:, None], rv, 0.0)
    # p is off by R and lse's own error, relative; what multiplies it, U + h (log p + H), likewise; then one sum over
    # the rows, at most 1024 additions one after the other in a part and some hundred parts: 1200 H of the sum of magnitudes
    rel = 2 * (e + 3 * H * deep + 300 * H + 4 * H * np.abs(np.nan_to_num(lse, neginf=0))) + 1200 * H
    size = np.abs(np.asarray(u, np.float64)).sum(axis=1) if u is not None else np.zeros(len(qv))
    given_part = np.zeros_like(want)
    if given is not None:
        for i in range(len(qv)):
            for j, g in enumerate(given[i]):
                if 0 <= g < len(rv):
                    given_part[i] += abs(float(u[i, j])) * np.abs(kept[g])
    if h is not None:
        size = size + np.abs(np.asarray(h, np.float64)) * (2 * deep + 2 + np.log(max(len(rv), 1)))
    off = abs(scale) * (rel[:, None] * size[:, None] * (p @ np.abs(kept)) + 80 * H * given_part) + 4 * H * np.abs(want)
    # a p below float32's smallest normal number 2^-126 may be held as 0: it is then off by itself, which is below 2^-126, and what
    # it adds to a column by at most 2^-126 |row| (U + |h| |log p + H|), |log p| <= |s - lse|.  (Seen: 0 for -5e-46.)
    with np.errstate(invalid="ignore"):
        gone = np.nan_to_num(np.where(np.isneginf(s), 0, np.abs(s - lse[:, None])), posinf=0, neginf=0) + np.log(max(len(rv), 1)) + 1
    weight = np.abs(np.asarray(u, np.float64)).sum(axis=1) if u is not None else np.zeros(len(qv))
    weight = weight[:, None] + (np.abs(np.asarray(h, np.float64))[:, None] * gone if h is not None else 0.0)
    off = off + abs(scale) * 2.0 ** -126 * (weight * np.ones_like(s) @ np.abs(kept)) + 2.0 ** -149
    assert np.all(np.abs(got - want) <= off), np.max(np.abs(got - want) / np.maximum(off, 1e-300))
    return got


GRAD_SHAPES = [(1, 1, 4, 1), (2, 3, 8, 2), (1, 1000, 16, 1), (33, 31, 12, 3), (32, 64, 20, 1), (5, 4097, 32, 16), (65, 700, 100, 4), (3, 65, 260, 65),
               (40, 300, 512, 2), (130, 500, 64, 1), (2, 200, 1000, 3), (7, 1500, 1024, 1), (64, 20000, 16, 1), (34, 9999, 36, 2)]


@pytest.mark.parametrize("m,n,dim,g", GRAD_SHAPES)
@pytest.mark.parametrize("kind", ["plain", "entropy", "biased"])
def test_gradient(m, n, dim, g, kind):
    rng = np.random.default_rng(m + n + dim + g)
    (q, qv), (r, rv) = make(rng, m, dim), make(rng, n, dim, 0.1)
    scale = float(rng.choice([10, -20, 50])) / np.sqrt(dim)
    bias = h = None
    if kind == "biased":
        bias = rng.normal(size=n).astype(np.float32)
        bias[rng.random(n) < 0.3] = rng.choice([-np.inf, np.inf, np.nan])
        bias[rng.random(n) < 0.1] = np.finfo(np.float32).min
    if kind != "plain":
        h = rng.normal(size=m).astype(np.float32)
    given = rng.integers(-1, n + 1, size=(m, g)).astype(np.int32)
    if g > 2:
        given[:, 2] = given[:, 1]              # the same row twice
    check_gradient(q, qv, r, rv, scale, bias, given, rng.normal(size=(m, g)).astype(np.float32), h)


def test_gradient_of_the_entropy_alone_and_of_nothing():
    rng = np.random.default_rng(9)
    (q, qv), (r, rv) = make(rng, 6, 64), make(rng, 200, 64, 0.1)
    check_gradient(q, qv, r, rv, 2.0, None, None, None, rng.normal(size=6).astype(np.float32))
    lse = hps.mx4_logprobs(q, r).lse
    assert (hps.mx4_logprobs_backward(q, r, None, None, lse) == 0).all()
    none = hps.mx4_logprobs(q, r[3:3])
    assert (hps.mx4_logprobs_backward(q, r[3:3], None, None, none.lse) == 0).all()


def test_gradient_where_little_or_nothing_is_left():
    """Rows that are out: also those that stand for NaN; a query whose probability sits on one row, which is the given one."""
    rng = np.random.default_rng(10)
    (q, qv), (r, rv) = make(rng, 35, 36), make(rng, 500, 36)
    bias = np.full(500, -np.inf, dtype=np.float32)
    given = np.tile(np.array([3, 77], dtype=np.int32), (35, 1))
    u = rng.normal(size=(35, 2)).astype(np.float32)
    h = rng.normal(size=35).astype(np.float32)
    assert (check_gradient(q, qv, r, rv, 1.0, bias, given, u, h) == 0).all()
    bias[77] = -3.0
    check_gradient(q, qv, r, rv, 1.0, bias, given, u, h)
    bias[100:300] = 0.0
    bias[150] = np.nan
    r.scales[150, 1] = 255
    got = check_gradient(q, qv, r, np.where(np.arange(500)[:, None] == 150, 0.0, rv), 1.0, bias, given, u, h)
    assert np.isfinite(got).all()
    bias[77] = 60.0
    check_gradient(q, qv, r, np.where(np.arange(500)[:, None] == 150, 0.0, rv), 1.0, bias, given, u, h)


# ---- how they are called -------------------------------------------------------------------------
def everything(q, r, given, u, h, bias):
    out = hps.mx4_logprobs(q, r, given, 9, 3.0, bias)
    d = hps.mx4_logprobs_backward(q, r, given, u, out.lse, out.entropy, h, 3.0, bias)
    return tuple(out) + (d, hps.mx4_scores(q, r, 3.0, bias))


def inputs(seed, m=70, n=5000, dim=64):
    rng = np.random.default_rng(seed)
    (q, _), (r, _) = make(rng, m, dim), make(rng, n, dim, 0.1)
    bias = rng.normal(size=n).astype(np.float32)
    bias[::50] = -np.inf
    return q, r, dev(rng.integers(0, n, size=(m, 2)).astype(np.int32)), dev(rng.normal(size=(m, 2)).astype(np.float32)), \
        dev(rng.normal(size=m).astype(np.float32)), dev(bias)


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_two_calls_give_the_same_bits():
    a = inputs(1)
    assert same(everything(*a), everything(*a))


def test_on_two_streams_at_once():
    a, b = inputs(1), inputs(2)
    want = everything(*a), everything(*b)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for _ in range(3):
        for i, x in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i] = everything(*x)
        torch.cuda.synchronize()
        assert same(got[0], want[0]) and same(got[1], want[1])


def test_captured_and_replayed():
    """Two graphs, each with workspaces of its own, replayed with new inputs and other work between the replays."""
    first, second = inputs(1), inputs(3, m=33, n=3001)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        everything(*first), everything(*second)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x in (first, second):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(everything(*x))
        graphs.append(g)
    for turn in range(4):
        for k, x in enumerate((first, second)):
            new = inputs(10 + turn + 7 * k, *(() if k == 0 else (33, 3001)))
            for to, of in zip(x, new):
                if isinstance(to, hps.Mx4Rows):
                    to.codes.copy_(of.codes)
                    to.scales.copy_(of.scales)
                else:
                    to.copy_(of)
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for k, x in enumerate((first, second)):
            assert same(everything(*x), outs[k])
        torch.cuda.synchronize()


def test_binding_refuses_what_does_not_fit():
    rng = np.random.default_rng(0)
    (q, _), (r, _), (other, _) = make(rng, 4, 64), make(rng, 50, 64), make(rng, 4, 32)
    given, u = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    lse = torch.zeros(4, device="cuda")
    calls = [lambda: hps.mx4_scores(other, r), lambda: hps.mx4_scores(q, r, bias=torch.zeros(49, device="cuda")),
             lambda: hps.mx4_scores(q, r, bias=torch.zeros(50, device="cuda").double()), lambda: hps.mx4_scores(q, r, bias=torch.zeros(50)),
             lambda: hps.mx4_scores(q, r, dtype=torch.float16), lambda: hps.mx4_scores(q, r, out=torch.zeros((4, 49), device="cuda")),
             lambda: hps.mx4_scores(q, r, out=torch.zeros((50, 4), device="cuda").t()),
             lambda: hps.mx4_quantize(torch.zeros((4, 64), device="cuda").half()), lambda: hps.mx4_quantize(torch.zeros((64, 4), device="cuda").t()),
             lambda: hps.mx4_quantize(torch.zeros(64, device="cuda")), lambda: hps.Mx4Rows(q.codes[:, :16], q.scales, 64),
             lambda: hps.Mx4Rows(q.codes[::2], q.scales[::2], 64), lambda: hps.Mx4Rows(q.codes, q.scales[:3], 64), lambda: hps.Mx4Rows(q.codes, q.scales, 32),
             lambda: hps.mx4_logprobs(q, r, given.long()), lambda: hps.mx4_logprobs(q, r, given[:3]), lambda: hps.mx4_logprobs(q, r, given[:, 0]),
             lambda: hps.mx4_logprobs_backward(q, r, given, None, lse), lambda: hps.mx4_logprobs_backward(q, r, given, u[:, :1], lse),
             lambda: hps.mx4_logprobs_backward(q, r, given, u, lse[:3]), lambda: hps.mx4_logprobs_backward(q, r, given, u, lse, d_entropy=lse)]
    for call in calls:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: hps.mx4_logprobs(q, r, top=65), lambda: hps.mx4_logprobs(q, r, top=-1), lambda: hps.mx4_scores(q, r, float("inf")),
                 lambda: hps.mx4_quantize(torch.zeros((4, 6), device="cuda")),
                 lambda: hps.mx4_quantize(torch.zeros((4, 66), device="cuda")[:, :64]),
                 lambda: hps.mx4_quantize(torch.zeros((4, 68), device="cuda")[:, 1:65])):
        with pytest.raises(hps.HpsError) as e:
            call()
        assert e.value.status == hps.EINVAL
    with pytest.raises(TypeError):
        r[3]


@pytest.mark.parametrize("dim", [16, 64])
def test_a_run_of_them_together(dim):
    """Rows of the table are frozen, pooled rows become queries, a loss over chosen rows and the entropy is formed, and its
    gradient goes back into the table: one Adagrad step, as if the gradient had come from the definition in 64 bits."""
    rng = np.random.default_rng(dim)
    n_items, n_users, m = 1500, 400, 48
    kw = dict(lr=0.05, eps=1e-8, init_acc=0.1, init_seed=1)
    items, users = hps.HpsTable(4000, dim, 4096, 64, **kw), hps.HpsTable(1000, dim, 1000, m, **kw)
    item_keys = dev(rng.permutation(10 ** 6)[:n_items].astype(np.int64) + 1)
    user_keys = dev(rng.permutation(10 ** 6)[:n_users].astype(np.int64) + 1)
    items.insert(item_keys, dev((0.3 * rng.normal(size=(n_items, dim))).astype(np.float32)))
    users.insert(user_keys, dev((0.3 * rng.normal(size=(n_users, dim))).astype(np.float32)))
    rows, found = items.get_mx4(item_keys)
    assert found.all()
    item_w = ref.quantize(items.get(item_keys)[0].cpu().numpy())[2]
    for step in range(2):
        lengths = rng.integers(0, 6, size=m)
        offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        asked = user_keys[torch.from_numpy(rng.integers(0, n_users, offsets[-1])).cuda()].contiguous()
        pooled = users.pull(asked, dev(offsets), m, 1)
        queries, rounded = hps.mx4_quantize(pooled, values=True)
        qv = ref.quantize(pooled.cpu().numpy())[2]
        assert np.array_equal(rounded.cpu().numpy(), qv.astype(np.float32))
        chosen = dev(rng.integers(0, n_items, size=(m, 3)).astype(np.int32))
        u = dev(np.full((m, 3), -1.0 / (3 * m), dtype=np.float32))
        h = torch.full((m,), -0.01 / m, device="cuda")
        out = hps.mx4_logprobs(queries, rows, chosen, 5, 4.0)
        d = hps.mx4_logprobs_backward(queries, rows, chosen, u, out.lse, out.entropy, h, 4.0)
        want = ref.query_gradient(qv, item_w, 4.0, None, chosen.cpu().numpy(), u.cpu().numpy(), h.cpu().numpy())
        assert np.all(np.abs(d.cpu().numpy() - want) <= 1e-5 * np.abs(want) + 1e-6 * np.abs(want).max())
        check_logprobs(queries, qv, rows, item_w, 4.0, None, chosen.cpu().numpy(), 5)
        # the step of every touched row
        keys = asked.cpu().numpy()
        w0, a0, _ = users.get(asked)
        users.push(d)
        w1 = users.get(asked)[0].cpu().numpy()
        bag = np.repeat(np.arange(m), lengths)
        for key in np.unique(keys):
            at = np.nonzero(keys == key)[0]
            g = want[bag[at]].sum(axis=0)
            acc = float(a0[at[0], 0]) + np.mean(g * g)
            w = w0[at[0]].double().cpu().numpy() - 0.05 * g / (np.sqrt(acc) + 1e-8)
            assert np.all(np.abs(w1[at[0]] - w) <= 1e-6 + 1e-5 * np.abs(w))


# ---- large ones ----------------------------------------------------------------------------------
def test_a_catalogue_beyond_32_bits():
    """Codes of more than 2^32 bytes: the rows on both sides of that offset, and the last ones, count like any others."""
    n, dim, m = (1 << 27) + 5003, 64, 3
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    codes = torch.randint(-2 ** 63, 2 ** 63 - 1, (n, 4), generator=gen, device="cuda").view(torch.uint8)
    r = hps.Mx4Rows(codes, torch.full((n, 2), 120, dtype=torch.uint8, device="cuda"), dim)
    q, _ = make(np.random.default_rng(3), m, dim)
    # copies of the queries, larger than anything else, where offsets pass 2^31 and 2^32 bytes and at the end
    spots = [0, (1 << 26) - 1, 1 << 26, (1 << 27) - 1, 1 << 27, n - 1]
    for k, at in enumerate(spots):
        r.codes[at] = q.codes[k % m]
        r.scales[at] = 135
    out = hps.mx4_scores(q, r, 0.01)
    for first, last in ((0, 300), ((1 << 26) - 200, (1 << 26) + 200), ((1 << 27) - 200, (1 << 27) + 200), (n - 333, n)):
        assert torch.equal(out[:, first:last], hps.mx4_scores(q, r[first:last], 0.01))
    given = dev(np.array([[spots[k], spots[k + 3]] for k in range(m)], dtype=np.int32))
    got = hps.mx4_logprobs(q, r, given, 10, 0.01)
    best = torch.topk(out, 12, dim=1)
    assert torch.equal(got.top_index[:, :2].long().sort().values, best.indices[:, :2].sort().values)
    lse = torch.logsumexp(out.double(), 1)
    assert (got.lse.double() - lse).abs().max() <= 1e-5 * lse.abs().max()
    assert (got.logp.double() - (out.gather(1, given.long()).double() - lse[:, None])).abs().max() <= 1e-4
    u = torch.full((m, 2), -0.5, device="cuda")
    # nearly all of the probability lies on the copies: the gradient is that of a catalogue of these alone, as far as they count
    d = hps.mx4_logprobs_backward(q, r, given, u, got.lse, scale=0.01)
    p = torch.exp(out.double() - lse[:, None])
    assert p[:, spots].sum(1).min() > 0.999
    w = hps.Mx4Rows(r.codes[spots].contiguous(), r.scales[spots].contiguous(), dim).dequantize().double()
    at = {s: i for i, s in enumerate(spots)}
    picked = torch.stack([w[[at[int(g)] for g in row]].sum(0) for row in given.cpu()]) * -0.5
    want = 0.01 * (picked + p[:, spots] @ w)
    size = 0.01 * w.abs().max()
    assert (d.double() - want).abs().max() <= 2e-3 * size       # (1 - 0.999 of a row's largest value, twice)
    del out, codes, r
    torch.cuda.empty_cache()


def test_scores_beyond_32_bits():
    m, n, dim = 70_000, 65_540, 4
    (q, _), (r, _) = make(np.random.default_rng(4), m, dim), make(np.random.default_rng(5), n, dim)
    out = hps.mx4_scores(q, r, dtype=torch.bfloat16)
    for a, b in ((0, 40), (32_760, 32_780), (65_520, 65_560), (m - 33, m)):
        assert torch.equal(out[a:b], hps.mx4_scores(q[a:b], r, dtype=torch.bfloat16))
    del out
    torch.cuda.empty_cache()


def test_rows_of_a_table_beyond_32_bits_of_codes():
    """A strided input whose rows start more than 2^32 bytes in."""
    n, dim, wide = 1 << 21, 32, 1024
    x = torch.empty((n, wide), dtype=torch.bfloat16, device="cuda")
    x[:, :dim] = torch.randn((n, dim), device="cuda")
    rows = hps.mx4_quantize(x[:, :dim])
    for a, b in ((0, 100), ((1 << 21) - 100, 1 << 21), ((1 << 20) - 50, (1 << 20) + 50)):
        want = hps.mx4_quantize(x[a:b, :dim].contiguous())
        assert torch.equal(rows.codes[a:b], want.codes) and torch.equal(rows.scales[a:b], want.scales)


@pytest.mark.parametrize("m,n,dim", [(1, 1, 8), (300, 7, 16), (1500, 1, 64), (2000, 33, 1024), (5, 100_000, 1024), (70, 3000, 1000)])
def test_extreme_shapes(m, n, dim):
    rng = np.random.default_rng(m + n)
    (q, qv), (r, rv) = make(rng, m, dim), make(rng, n, dim, 0.1)
    given = rng.integers(0, n, size=(m, 2)).astype(np.int32)
    check_logprobs(q, qv, r, rv, 10 / np.sqrt(dim), None, given, 5)
    check_gradient(q, qv, r, rv, 10 / np.sqrt(dim), None, given, rng.normal(size=(m, 2)).astype(np.float32), rng.normal(size=m).astype(np.float32))


def test_an_entropy_that_is_all_there_is_to_lose():
    """Few rows, many given ones: terms that cancel almost entirely."""
    rng = np.random.default_rng(11)
    for seed in range(20):
        (q, qv), (r, rv) = make(rng, 2, 64), make(rng, 3, 64, 0.1)
        given = rng.integers(-1, 3, size=(2, 16)).astype(np.int32)
        check_gradient(q, qv, r, rv, 0.6, None, given, (0.1 * rng.normal(size=(2, 16))).astype(np.float32), rng.normal(size=2).astype(np.float32))


@pytest.mark.parametrize("m", [3, 300])
@pytest.mark.parametrize("n", [40, 700, 100_000])
def test_more_equal_scores_than_there_is_room_for(m, n):
    """All rows alike: the best are the first, whichever way they are found."""
    rng = np.random.default_rng(n)
    one = ref.quantize(rng.normal(size=(1, 8)).astype(np.float32))
    r = hps.Mx4Rows(dev(np.repeat(one[0], n, axis=0)), dev(np.repeat(one[1], n, axis=0)), 8)
    (q, _) = make(rng, m, 8)
    for top in (1, 5, 8, 16, 17, 64):
        got = hps.mx4_logprobs(q, r, top=top)
        want = torch.arange(top, device="cuda", dtype=torch.int32)
        want = torch.where(want < n, want, torch.full_like(want, -1))
        assert (got.top_index == want).all()
        assert (got.top_logp[:, :min(top, n)] + np.log(n)).abs().max() <= 1e-5 * np.log(n)


@pytest.mark.parametrize("top", [1, 3, 8, 16, 33, 64])
@pytest.mark.parametrize("n", [50, 3000, 30_000])
def test_best_rows_of_many_queries(n, top):
    rng = np.random.default_rng(n + top)
    (q, qv), (r, rv) = make(rng, 300, 16), make(rng, n, 16, 0.1)
    check_logprobs(q, qv, r, rv, 2.5, None, None, top)


def test_backward_without_rows_reads_nothing():
    """No rows, but a bias and given rows: called as C, since the binding has no address for an empty bias."""
    (q, _) = make(np.random.default_rng(1), 5, 64)
    none = hps.binding.Mx4Operand(None, None, 0)
    bias, lse = torch.zeros(4, device="cuda"), torch.full((5,), float("-inf"), device="cuda")
    given = torch.full((5, 2), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    given[:, 1] = -5
    u, out = torch.ones((5, 2), device="cuda"), torch.full((5, 64), 3.0, device="cuda")
    space = torch.empty(hps.lib().hps_mx4_logprobs_backward_bytes(5, 0, 64), dtype=torch.uint8, device="cuda")
    st = hps.lib().hps_mx4_logprobs_backward(q._operand(), ctypes.byref(none), 64, 1.0, bias.data_ptr(), lse.data_ptr(), None, given.data_ptr(),
                                             u.data_ptr(), 2, None, out.data_ptr(), space.data_ptr(), space.numel(),
                                             torch.cuda.current_stream().cuda_stream)
    assert st == hps.OK and (out == 0).all()


def test_gradient_of_more_values_than_a_launch_has_workgroups():
    m, n, dim = 1 << 17, 3, 1024
    (r, rv) = make(np.random.default_rng(2), n, dim, 0.1)
    codes = torch.randint(0, 256, (m, dim // 2), dtype=torch.uint8, device="cuda")
    q = hps.Mx4Rows(codes, torch.full((m, dim // 32), 125, dtype=torch.uint8, device="cuda"), dim)
    given = torch.randint(0, n, (m, 1), dtype=torch.int32, device="cuda")
    u = torch.ones((m, 1), device="cuda")
    out = hps.mx4_logprobs(q, r, given, scale=0.05)
    d = hps.mx4_logprobs_backward(q, r, given, u, out.lse, out.entropy, scale=0.05)
    for a, b in ((0, 70), (65_500, 65_600), (m - 70, m)):
        part = q[a:b]
        o = hps.mx4_logprobs(part, r, given[a:b], scale=0.05)
        want = hps.mx4_logprobs_backward(part, r, given[a:b], u[a:b], o.lse, o.entropy, scale=0.05)
        assert torch.equal(d[a:b], want)


@pytest.mark.parametrize("scale", [0.0, 1e-45, -1e-38, 1e-20, 1e6])
def test_gradient_with_scales_of_all_sizes(scale):
    rng = np.random.default_rng(12)
    (q, qv), (r, rv) = make(rng, 40, 64), make(rng, 900, 64, 0.1)
    given = rng.integers(-1, 900, size=(40, 2)).astype(np.int32)
    if scale < 1:
        check_gradient(q, qv, r, rv, scale, None, given, rng.normal(size=(40, 2)).astype(np.float32), rng.normal(size=40).astype(np.float32))
    else:
        out = hps.mx4_logprobs(q, r, dev(given), scale=scale)
        assert torch.isfinite(out.lse).all() and (out.entropy >= -1e-6).all()
