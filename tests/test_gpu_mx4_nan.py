"""A query with a block that stands for NaN (a pooled row that held an infinity) against rows of which some, or all, are taken out by
their bias: a row that is out is out whatever the query holds, and the other queries notice nothing.  Compared bit for bit
with the same call where the query is an ordinary one."""
import numpy as np
import pytest
import torch

import paper_2003_05622_amd as hps
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
