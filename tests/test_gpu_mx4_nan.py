"""A query with a block that stands for NaN (a pooled row that held an infinity) against rows of which some, or all, are taken out by
their bias: a row that is out is out whatever the query holds, and the other queries notice nothing.  Compared with the same call where
the query is an ordinary one, bit for bit but for gradients: whether 32 queries' probabilities go through the matrix unit with all their
bits, or are off by up to 2^-16 of themselves, is decided for all of them together."""
import numpy as np
import pytest
import torch

import paper_2003_05622_amd as hps
import mx4_reference as ref
from test_gpu_mx4 import dev, make

pytestmark = pytest.mark.gpu

INF = float("inf")
# a row of one block, of an odd and of an even number of them, of so many that scale bytes are packed; queries for one wave, and so many
# that waves share the rows (70 of rows above 256 values) or hold two tiles (300)
SHAPES = [(5, 300, 8), (40, 700, 16), (33, 200, 64), (300, 260, 64), (9, 500, 100), (3, 130, 260), (70, 400, 300), (70, 300, 512), (70, 200, 1000),
          (2, 90, 1024)]


def case(m, n, dim, all_out):
    """(queries, the same with a NaN in two of them, rows, bias, which rows are out, the two queries)"""
    rng = np.random.default_rng(m + n + dim)
    (clean, _), (rows, _) = make(rng, m, dim), make(rng, n, dim, 0.1)
    queries = hps.Mx4Rows(clean.codes.clone(), clean.scales.clone(), dim)
    broken = [0, m - 1]
    queries.scales[0, 0] = 255                      # the first block of one, the last of another
    queries.scales[m - 1, -1] = 255
    bias = rng.normal(size=n).astype(np.float32)
    out = np.ones(n, dtype=bool) if all_out else rng.random(n) < 0.3
    out[n // 2] = True
    bias[out] = rng.choice([-np.inf, np.inf, np.nan], size=int(out.sum()))
    return clean, queries, rows, dev(bias), dev(out), broken


def same_or_nan(a, b):
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


@pytest.mark.parametrize("m,n,dim", SHAPES)
@pytest.mark.parametrize("all_out", [False, True])
def test_scores_of_a_query_that_stands_for_nan(m, n, dim, all_out):
    clean, queries, rows, bias, out, broken = case(m, n, dim, all_out)
    want = hps.mx4_scores(clean, rows, 0.5, bias)
    want[broken] = float("nan")
    want[:, out] = -INF
    got = hps.mx4_scores(queries, rows, 0.5, bias)
    assert same_or_nan(got, want)
    narrow = hps.mx4_scores(queries, rows, 0.5, bias, dtype=torch.bfloat16)
    assert same_or_nan(narrow, want.bfloat16())


@pytest.mark.parametrize("m,n,dim", SHAPES)
@pytest.mark.parametrize("all_out", [False, True])
def test_log_probabilities_of_a_query_that_stands_for_nan(m, n, dim, all_out):
    clean, queries, rows, bias, out, broken = case(m, n, dim, all_out)
    given = torch.randint(0, n, (m, 3), dtype=torch.int32, device="cuda")
    given[:, 0], given[:, 1] = -1, n // 2           # padding, a row that is out
    want = hps.mx4_logprobs(clean, rows, given, 9, 0.5, bias)
    got = hps.mx4_logprobs(queries, rows, given, 9, 0.5, bias)
    others = torch.ones(m, dtype=torch.bool, device="cuda")
    others[broken] = False
    for a, b in zip(got, want):
        assert torch.equal(a[others], b[others])
    for i in broken:
        assert (got.top_index[i] == -1).all() and (got.top_logp[i] == -INF).all()
        assert got.logp[i, 0] == 0 and got.logp[i, 1] == -INF
        if all_out:
            assert got.lse[i] == -INF and got.entropy[i] == 0 and got.logp[i, 2] == -INF
        else:
            assert torch.isnan(got.lse[i]) and torch.isnan(got.entropy[i])
            assert got.logp[i, 2] == -INF if bool(out[given[i, 2].long()]) else torch.isnan(got.logp[i, 2])


@pytest.mark.parametrize("m,n,dim", SHAPES)
@pytest.mark.parametrize("all_out", [False, True])
@pytest.mark.parametrize("with_entropy", [False, True])
def test_gradient_of_a_query_that_stands_for_nan(m, n, dim, all_out, with_entropy):
    clean, queries, rows, bias, out, broken = case(m, n, dim, all_out)
    given = torch.randint(0, n, (m, 2), dtype=torch.int32, device="cuda")
    u = torch.randn((m, 2), device="cuda")
    h = torch.randn(m, device="cuda") if with_entropy else None
    fine = hps.mx4_logprobs(clean, rows, given, 0, 0.5, bias)
    want = hps.mx4_logprobs_backward(clean, rows, given, u, fine.lse, fine.entropy, h, 0.5, bias)
    # (lse and entropy as documented for such a query, whatever the forward pass gives)
    lse, entropy = fine.lse.clone(), fine.entropy.clone()
    lse[broken], entropy[broken] = (-INF, 0.0) if all_out else (float("nan"), float("nan"))
    got = hps.mx4_logprobs_backward(queries, rows, given, u, lse, entropy, h, 0.5, bias)
    others = torch.ones(m, dtype=torch.bool, device="cuda")
    others[broken] = False
    # |c_r| <= p_r (|U| + |h| (|log p_r| + H)), of which 2^-16 may be missing on either side
    s = hps.mx4_scores(clean, rows, 0.5, bias)
    deep = torch.where(s == -INF, 0.0, (s - fine.lse[:, None]).abs()).nan_to_num(nan=0.0).amax(1) + fine.entropy
    size = u.abs().sum(1) + (h.abs() * deep if with_entropy else 0.0)
    off = 2 * 2.0 ** -16 * 0.5 * size * rows.dequantize().abs().max()
    assert ((got - want).abs() <= off[:, None])[others].all()
    for i in broken:
        assert (got[i] == 0).all() if all_out else torch.isnan(got[i]).all()


def test_a_pooled_row_that_is_not_finite_goes_through():
    """From values: an infinity makes its block NaN, and rows that are out stay out behind it."""
    rng = np.random.default_rng(3)
    x = torch.randn((4, 64), device="cuda")
    x[2, 40] = INF
    rows, _ = make(rng, 50, 64, 0.1)
    bias = torch.full((50,), -INF, device="cuda")
    queries = hps.mx4_quantize(x)
    assert queries.scales.cpu().tolist()[2][1] == 255
    got = hps.mx4_logprobs(queries, rows, None, 3, 1.0, bias)
    assert (got.lse == -INF).all() and (got.entropy == 0).all() and (got.top_index == -1).all()
    d = hps.mx4_logprobs_backward(queries, rows, None, None, got.lse, got.entropy, torch.ones(4, device="cuda"), 1.0, bias)
    assert (d == 0).all() and (hps.mx4_scores(queries, rows, 1.0, bias) == -INF).all()
    assert np.isneginf(ref.scores(np.full((1, 64), np.nan), np.zeros((50, 64)), 1.0, bias.cpu().numpy())).all()


@pytest.mark.parametrize("dim,m", [(8, 3), (64, 40), (300, 70)])
def test_a_scale_of_nothing_and_large_products(dim, m):
    """All scores are 0, however large the products are that are scaled."""
    n = 5000
    rng = np.random.default_rng(dim)
    queries, rows = hps.Mx4Rows.empty(m, dim, "cuda"), hps.Mx4Rows.empty(n, dim, "cuda")
    for held in (queries, rows):
        held.codes.zero_()
        held.codes[:, 0] = dev(rng.integers(0, 256, size=held.n, dtype=np.uint8))
        held.scales.fill_(127)
        held.scales[:, 0] = 127 + 57                # products up to 72 x 2^114
    given = torch.full((m, 1), 4321, dtype=torch.int32, device="cuda")
    got = hps.mx4_logprobs(queries, rows, given, 4, 0.0)
    log_n = float(np.log(n))
    # (as many equal terms: sums of whole numbers, one logarithm)
    assert (got.lse - log_n).abs().max() <= 8 * 2.0 ** -24 * log_n and (got.entropy - log_n).abs().max() <= 8 * 2.0 ** -24 * log_n
    assert (got.logp + log_n).abs().max() <= 8 * 2.0 ** -24 * log_n
    assert (got.top_index == torch.arange(4, dtype=torch.int32, device="cuda")).all()
    assert (hps.mx4_scores(queries, rows, 0.0) == 0).all()
    d = hps.mx4_logprobs_backward(queries, rows, given, torch.ones((m, 1), device="cuda"), got.lse, got.entropy, torch.ones(m, device="cuda"), 0.0)
    assert (d == 0).all()
