"""The operators on frozen rows (include/hps_mx4.h) without a GPU: exported symbols, sizes, and every refusal, which
comes before anything touches the device; and the gradient's formula, which the GPU tests take as their reference, against differences."""
import ctypes
import os
import re

import numpy as np
import pytest

import paper_2003_05622_amd as hps
from mx4_reference import log_probs, query_gradient

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20         # an aligned address that is never read on these paths
BIG = 1 << 40


def rows(n=10, codes=P, scales=P):
    return ctypes.byref(hps.binding.Mx4Operand(codes, scales, n))


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "hps_mx4.h")).read()
    names = set(re.findall(r"\b(hps_mx4_[a-z_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert names == set(hps.EXPORTS_MX4)
    for n in names:
        assert getattr(hps.lib(), n) is not None


def test_row_sizes():
    L = hps.lib()
    want = {4: (4, 1), 8: (4, 1), 12: (8, 1), 16: (8, 1), 20: (16, 1), 32: (16, 1), 36: (32, 2), 64: (32, 2), 100: (64, 4), 1024: (512, 32)}
    for dim, shape in want.items():
        assert (L.hps_mx4_row_bytes(dim), L.hps_mx4_row_scales(dim)) == shape
    for dim in (0, 2, 6, 1028, 1 << 31):
        assert L.hps_mx4_row_bytes(dim) == 0 and L.hps_mx4_row_scales(dim) == 0


def test_quantize_refuses():
    f = hps.lib().hps_mx4_quantize
    assert f(P, 0, 0, 64, 64, P, P, None, None) == hps.OK
    for bad in (dict(dim=6), dict(dim=0), dict(dim=1028), dict(type=2), dict(type=-1), dict(stride=60), dict(stride=66), dict(values=None),
                dict(codes=None), dict(scales=None), dict(values=P + 4), dict(codes=P + 8), dict(rounded=P + 4),
                dict(type=1, values=P + 4), dict(n=BIG), dict(stride=BIG), dict(n=1 << 39, stride=1 << 39)):
        a = dict(values=P, type=0, n=10, dim=64, stride=64, codes=P, scales=P, rounded=None)
        a.update(bad)
        assert f(a["values"], a["type"], a["n"], a["dim"], a["stride"], a["codes"], a["scales"], a["rounded"], None) == hps.EINVAL, bad


def test_dequantize_and_get_refuse():
    L = hps.lib()
    assert L.hps_mx4_dequantize(rows(0, None, None), 64, None, None) == hps.OK
    for r, dim, out in ((None, 64, P), (rows(), 6, P), (rows(), 64, None), (rows(), 64, P + 4), (rows(codes=P + 8), 64, P),
                        (rows(codes=None), 64, P), (rows(scales=None), 64, P), (rows(BIG), 64, P)):
        assert L.hps_mx4_dequantize(r, dim, out, None) == hps.EINVAL
    assert L.hps_mx4_get(None, P, 1, P, P, P, None) == hps.EINVAL


def test_scores_refuse():
    f = hps.lib().hps_mx4_scores
    assert f(rows(0), rows(), 64, 1.0, None, None, 0, 10, None) == hps.OK
    assert f(rows(), rows(0), 64, 1.0, None, None, 0, 0, None) == hps.OK
    for bad in (dict(q=None), dict(r=None), dict(dim=2), dict(scale=float("inf")), dict(scale=float("nan")), dict(type=2), dict(stride=9),
                dict(stride=1 << 41), dict(out=None), dict(out=P + 2), dict(type=1, out=P + 1), dict(bias=P + 2), dict(q=rows((1 << 20) + 1)),
                dict(r=rows(1 << 31), stride=1 << 31), dict(q=rows(codes=P + 4)), dict(r=rows(scales=None)),
                dict(q=rows(1 << 20), r=rows((1 << 31) - 1), stride=1 << 31)):
        a = dict(q=rows(), r=rows(), dim=64, scale=1.0, bias=None, out=P, type=0, stride=10)
        a.update(bad)
        assert f(a["q"], a["r"], a["dim"], a["scale"], a["bias"], a["out"], a["type"], a["stride"], None) == hps.EINVAL, bad


def test_logprobs_refuse():
    L = hps.lib()
    assert L.hps_mx4_logprobs_bytes(1, 1, 6, 0) == 0 and L.hps_mx4_logprobs_bytes(1, 1, 64, 65) == 0
    assert L.hps_mx4_logprobs_bytes((1 << 20) + 1, 1, 64, 0) == 0 and L.hps_mx4_logprobs_bytes(1, 1 << 31, 64, 0) == 0
    assert 0 < L.hps_mx4_logprobs_bytes(0, 0, 64, 0) <= L.hps_mx4_logprobs_bytes(10, 10, 64, 3)
    need = L.hps_mx4_logprobs_bytes(10, 1000, 64, 3)
    base = dict(q=rows(), r=rows(1000), dim=64, scale=1.0, bias=None, given=P, n_given=2, top=3, lse=P, entropy=P, logp=P, index=P, best=P,
                space=P, size=need)

    def call(**more):
        a = dict(base, **more)
        return L.hps_mx4_logprobs(a["q"], a["r"], a["dim"], a["scale"], a["bias"], a["given"], a["n_given"], a["top"], a["lse"], a["entropy"],
                                  a["logp"], a["index"], a["best"], a["space"], a["size"], None)
    assert call(q=rows(0), lse=None, space=None, size=0) == hps.OK
    for bad in (dict(q=None), dict(r=None), dict(dim=66), dict(scale=float("nan")), dict(scale=float("-inf")), dict(given=None), dict(logp=None),
                dict(n_given=(1 << 20) + 1), dict(top=65), dict(index=None), dict(best=None), dict(lse=None), dict(entropy=None), dict(space=None),
                dict(space=P + 16), dict(bias=P + 1), dict(given=P + 2), dict(lse=P + 2), dict(q=rows((1 << 20) + 1)), dict(r=rows(1 << 31)),
                dict(r=rows(1000, codes=P + 8))):
        assert call(**bad) == hps.EINVAL, bad
    assert call(size=need - 1) == hps.ENOMEM


def test_backward_refuses():
    L = hps.lib()
    assert L.hps_mx4_logprobs_backward_bytes(1, 1, 6) == 0 and L.hps_mx4_logprobs_backward_bytes(1, 1 << 31, 64) == 0
    need = L.hps_mx4_logprobs_backward_bytes(10, 1000, 64)
    base = dict(q=rows(), r=rows(1000), dim=64, scale=1.0, bias=None, lse=P, entropy=P, given=P, dlogp=P, n_given=2, dentropy=P, out=P, space=P,
                size=need)

    def call(**more):
        a = dict(base, **more)
        return L.hps_mx4_logprobs_backward(a["q"], a["r"], a["dim"], a["scale"], a["bias"], a["lse"], a["entropy"], a["given"], a["dlogp"],
                                           a["n_given"], a["dentropy"], a["out"], a["space"], a["size"], None)
    assert call(q=rows(0), lse=None, space=None, size=0) == hps.OK
    for bad in (dict(q=None), dict(r=None), dict(dim=1), dict(scale=float("inf")), dict(lse=None), dict(out=None), dict(out=P + 4), dict(given=None),
                dict(dlogp=None), dict(entropy=None), dict(space=None), dict(space=P + 8), dict(n_given=(1 << 20) + 1), dict(dentropy=P + 2),
                dict(r=rows(1 << 31)), dict(bias=P + 3)):
        assert call(**bad) == hps.EINVAL, bad
    assert call(size=need - 1) == hps.ENOMEM


def test_binding_refuses_tensors_that_are_not_on_a_gpu():
    import torch
    with pytest.raises(ValueError):
        hps.mx4_quantize(torch.zeros(3, 8))
    with pytest.raises(ValueError):
        hps.Mx4Rows(torch.zeros(3, 4, dtype=torch.uint8), torch.zeros(3, 1, dtype=torch.uint8), 8)
    with pytest.raises(hps.HpsError):
        hps.Mx4Rows.empty(3, 7, "cpu")


@pytest.mark.parametrize("seed", range(4))
def test_the_formula_of_the_gradient_against_differences(seed):
    rng = np.random.default_rng(seed)
    m, n, dim, g, scale = 3, 11, 8, 4, 0.7
    q, r = rng.normal(size=(m, dim)), rng.normal(size=(n, dim))
    bias = rng.normal(size=n)
    bias[4] = -np.inf
    given = rng.integers(0, n, size=(m, g)).astype(np.int32)
    given[0, 1], given[1, 0], given[2, 2], given[2, 3] = -1, 4, given[2, 1], n + 3      # padding, a row that is out, twice the same, no row
    u, h = rng.normal(size=(m, g)), rng.normal(size=m)
    used = (given >= 0) & (given < n) & np.isfinite(bias)[np.clip(given, 0, n - 1)]

    def loss(q):
        out = log_probs(q, r, scale, bias, given=given)
        return float(np.sum(np.where(used, u * np.where(used, out["logp"], 0.0), 0.0)) + np.sum(h * out["entropy"]))
    want = query_gradient(q, r, scale, bias, given, u, h)
    step = 1e-5
    for i in range(m):
        for j in range(dim):
            d = np.zeros_like(q)
            d[i, j] = step
            # (central differences: error of order step^2 and of rounding / step, each below 1e-9 here)
            assert abs((loss(q + d) - loss(q - d)) / (2 * step) - want[i, j]) < 1e-7
