"""The operators on frozen rows, as a user of the parameter server calls them.

A catalogue (items, ads) is frozen: its trained rows are held in microscaled 4-bit floating point, E2M1 codes with
one power-of-two scale per 32 values.  Queries (pooled rows) are brought into the same form and meet the catalogue.
The kinds of cases:

  quantize  rows of float32 or bfloat16 into 4 bits, with the values that the codes stand for (a trainer goes on
            with these);
  scores    every query against every row, with a temperature and a bias per row;
  logprobs  over the scores of a query, which are not kept: log-sum-exp, entropy, log probabilities of given rows
            and the best rows;
  backward  the gradient of given rows' log probabilities and of the entropy with respect to the queries.

`own` false: elementary torch operations; true: the framework's calls.
"""
import math

import torch

own = False

# Fields every case has.  m: queries; n: rows of the catalogue (of the input, for quantize); dim: values per row;
# bias: a bias per row, of which some are -inf (rows taken out); given / top: rows asked for by number, and best rows;
# sharp: the standard deviation of a query's scores; dtype: of the rows to quantize, or of the scores;
# wide: values between the starts of two rows to quantize; entropy: whether the entropy has a gradient too.
BASE = dict(kind="logprobs", m=1, n=1, dim=64, bias=False, given=1, top=0, sharp=2.0, dtype="float32", wide=0, entropy=False)


def _case(name, **more):
    case = dict(BASE, **more)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # the pooled rows of one scoring request become queries: latency alone
        _case("quantize_queries", kind="quantize", n=64),
        # a slice of the columns of bfloat16 rows, odd width and number
        _case("quantize_ragged", kind="quantize", n=300_001, dim=100, dtype="bfloat16", wide=112),
        # a catalogue is frozen
        _case("quantize_catalogue", kind="quantize", n=1 << 22),
        # one query against a catalogue
        _case("scores_one", kind="scores", m=1, n=1 << 20),
        # a batch against a shortlist, odd sizes, biased, kept in bfloat16
        _case("scores_ragged", kind="scores", m=333, n=100_003, dim=100, bias=True, dtype="bfloat16"),
        # wide rows, the whole matrix of scores
        _case("scores_wide", kind="scores", m=1024, n=1 << 18, dim=512),
        # one query against a large catalogue: what a retrieval request does
        _case("logprobs_one", m=1, n=1 << 22, top=16),
        # odd sizes, rows taken out, a few given rows, some of them padding
        _case("logprobs_ragged", m=77, n=300_001, dim=100, bias=True, given=3, top=10),
        # a mini-batch's log probabilities over the catalogue
        _case("logprobs_batch", m=1024, n=1 << 20, top=8),
        # narrow rows, few queries
        _case("backward_narrow", kind="backward", m=64, n=65_536, dim=16),
        # distillation: a teacher's best rows are the given ones; entropy regularised, biased, odd sizes
        _case("backward_ragged", kind="backward", m=333, n=100_003, dim=100, bias=True, given=16, entropy=True, sharp=4.0),
        # a mini-batch trained against the catalogue
        _case("backward_batch", kind="backward", m=1024, n=1 << 19),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["quantize", "scores", "logprobs", "logprobs", "backward"])
    dim = rng.choice([4, 8, 16, 16, 20, 32, 36, 64, 64, 64, 96, 100, 128, 128, 192, 256, 260, 512, 1000, 1024])
    if kind == "quantize":
        wide = rng.choice([0, 0, dim + 4 * rng.randint(1, 9)])
        return _case(None, kind=kind, n=_spread(rng, 1, (1 << 28) // max(dim, wide)), dim=dim,
                     dtype=rng.choice(["float32", "float32", "bfloat16"]), wide=wide)
    m = 1 if rng.random() < 0.2 else _spread(rng, 1, 2048)
    # at most the listed ones' products: 2^30 scores, 2^28 of them kept, 1.4 x 10^11 multiplications
    most = min((1 << 28) // m, 137_000_000_000 // (m * dim), 1 << 22)
    if kind == "logprobs":
        most = min((1 << 30) // m, 68_000_000_000 // (m * dim), 1 << 22)
    if kind == "backward":
        most = min((1 << 29) // m, 34_000_000_000 // (m * dim), 1 << 22)
    bias = rng.random() < 0.4
    if bias:
        most = min(most, (1 << 27) // m)
    n = _spread(rng, 1, most)
    return _case(None, kind=kind, m=m, n=n, dim=dim, bias=bias, sharp=rng.choice([0.5, 2.0, 2.0, 6.0]),
                 given=rng.choice([1, 1, 3, 16]) if kind == "backward" else rng.choice([0, 1, 1, 3]),
                 top=rng.choice([0, 1, 8, 16, 50, 64]) if kind == "logprobs" else 0,
                 dtype=rng.choice(["float32", "bfloat16"]) if kind == "scores" else "float32",
                 entropy=kind == "backward" and rng.random() < 0.3)


# ---- the 4-bit form in elementary operations ---------------------------------------------------

def _row_bytes(dim):
    """Bytes of a row's codes: whole blocks of 32 values, or 8 or 16 values for the narrowest rows."""
    return 4 if dim <= 8 else 8 if dim <= 16 else (dim + 31) // 32 * 16


def _to_blocks(x):
    """(x in blocks of 32, zeros behind a row's last value; the blocks' exponents)."""
    blocks = -(-x.shape[1] // 32)
    x = torch.nn.functional.pad(x.float(), (0, 32 * blocks - x.shape[1])).view(x.shape[0], blocks, 32)
    most = x.abs().amax(2)
    exponent = (torch.frexp(most)[1] - 3).clamp(-127, 127)
    return x, torch.where(most > 0, exponent, torch.full_like(exponent, -127))


def _nearest(x, exponent):
    """Numbers (0 .. 7) of the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 nearest to |x| / 2^exponent, ties to even."""
    y = (x * torch.exp2(-exponent.float())[:, :, None]).abs()
    above = (y > 0.25).int() + (y >= 0.75).int() + (y > 1.25).int() + (y >= 1.75).int()
    return above + (y > 2.5).int() + (y >= 3.5).int() + (y > 5.0).int()


def _magnitudes(device):
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=device)


def _values(x):
    blocks, exponent = _to_blocks(x)
    near = _magnitudes(x.device)[_nearest(blocks, exponent).long()] * torch.exp2(exponent.float())[:, :, None]
    return torch.where(blocks < 0, -near, near).reshape(x.shape[0], -1)[:, :x.shape[1]].contiguous()


def _codes(x):
    """(codes, two a byte, the earlier value in the lower half; scales as exponent + 127)."""
    blocks, exponent = _to_blocks(x)
    code = _nearest(blocks, exponent) + 8 * (blocks < 0).int()
    code = code.reshape(x.shape[0], -1)[:, :2 * _row_bytes(x.shape[1])].to(torch.uint8)
    return code[:, 0::2] | code[:, 1::2] << 4, (exponent + 127).to(torch.uint8)


def _decode(codes, scales, dim):
    """The float32 values of rows held as codes and scales."""
    both = torch.stack((codes & 15, codes >> 4), 2).reshape(codes.shape[0], -1).long()
    value = _magnitudes(codes.device)[both & 7]
    value = torch.where(both >= 8, -value, value)[:, :dim]
    return value * torch.exp2(scales.float() - 127.0).repeat_interleave(32, 1)[:, :dim]


# ---- inputs ------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*size):
        return torch.randn(*size, generator=gen, device="cuda")

    m, n, dim = case["m"], case["n"], case["dim"]
    if case["kind"] == "quantize":
        # trained rows: a common scale, rows of popular keys longer than others
        x = normal(n, max(dim, case["wide"])) * (0.05 * torch.exp(0.5 * normal(n, 1)))
        return {"case": case, "x": x.to(getattr(torch, case["dtype"]))[:, :dim]}
    rows = _codes(normal(n, dim) * (0.1 * torch.exp(0.25 * normal(n, 1))))
    queries = _codes(normal(m, dim))
    state = {"case": case, "queries": queries, "rows": rows, "scale": case["sharp"] * 10.0 / math.sqrt(dim), "bias": None}
    if case["bias"]:
        # the logarithm of the rows' popularity; one row in fifty is out of stock
        bias = 0.7 * normal(n)
        state["bias"] = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.02, torch.full_like(bias, -math.inf), bias)
    if case["kind"] == "scores":
        return state
    given = torch.randint(0, n, (m, case["given"]), generator=gen, device="cuda", dtype=torch.int32)
    if case["given"] > 1:
        given = torch.where(torch.rand(given.shape, generator=gen, device="cuda") < 0.05, torch.full_like(given, -1), given)
    state["given"] = given
    if case["kind"] == "backward":
        # the forward's results, which a trainer has kept, and the gradients that come from its loss
        out = _logprobs(dict(state, case=dict(case, given=0, top=0)))
        state["lse"], state["entropy"] = out["lse"], out["entropy"]
        state["d_logp"] = -torch.softmax(normal(m, case["given"]), 1) / m
        state["d_entropy"] = 0.01 * normal(m) / m if case["entropy"] else None
    return state


# ---- the plain forms ---------------------------------------------------------------------------

def _scores(state):
    """float32 scores of every query and row; -inf for rows taken out."""
    dim = state["case"]["dim"]
    dots = torch.matmul(_decode(*state["queries"], dim), _decode(*state["rows"], dim).t())
    if state["bias"] is None:
        return dots * state["scale"] + 0.0
    # (in 64 bits: the sum is rounded once, so that scores next to each other keep their order)
    scale = torch.tensor(state["scale"], dtype=torch.float32, device=dots.device).double()
    out = ~torch.isfinite(state["bias"])
    s = (dots.double() * scale + state["bias"].double()).float() + 0.0
    return torch.where(out[None, :], torch.full_like(s, -math.inf), s)


def _taken(scores, given):
    """Scores of the given rows, and which of them are rows at all (a negative number is padding)."""
    real = given >= 0
    return torch.gather(scores, 1, given.clamp(min=0).long()), real


def _best(scores, top):
    """Numbers of the best rows, best first, the lower number first among equals; -1 where no row is left."""
    m, n = scores.shape
    bits = scores.view(torch.int32).long()
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)          # ascending as the scores are
    key = order * (1 << 32) + torch.arange(n - 1, -1, -1, device=scores.device)
    best = torch.topk(key, min(top, n), 1).values
    best = (n - 1) - (best & 0xFFFFFFFF)
    s = torch.gather(scores, 1, best)
    best = torch.where(s == -math.inf, torch.full_like(best, -1), best)
    pad = (0, top - best.shape[1])
    return torch.nn.functional.pad(best, pad, value=-1).int(), torch.nn.functional.pad(s, pad, value=-math.inf)


def _logprobs(state):
    case, s = state["case"], _scores(state)
    most = s.amax(1, keepdim=True)
    most = torch.where(most == -math.inf, torch.zeros_like(most), most)
    e = torch.exp(s - most)
    total = e.sum(1, keepdim=True)
    lse = most + torch.log(total)
    weighted = torch.where(e > 0, e * (s - most), torch.zeros_like(e)).sum(1, keepdim=True)
    entropy = torch.where(total > 0, torch.log(total) - weighted / total, torch.zeros_like(total))
    out = {"lse": lse[:, 0], "entropy": entropy[:, 0]}
    if case["given"]:
        v, real = _taken(s, state["given"])
        out["logp"] = torch.where(real, torch.where(v == -math.inf, v, v - lse), torch.zeros_like(v))
    if case["top"]:
        out["top_index"], v = _best(s, case["top"])
        out["top_logp"] = torch.where(v == -math.inf, v, v - lse)
    return out


def _backward(state):
    dim, s = state["case"]["dim"], _scores(state)
    rows = _decode(*state["rows"], dim)
    v, real = _taken(s, state["given"])
    u = torch.where(real & (v > -math.inf), state["d_logp"], torch.zeros_like(v))
    held = s > -math.inf
    logp = torch.where(held, s - state["lse"][:, None], torch.zeros_like(s))
    p = torch.where(held, torch.exp(logp), torch.zeros_like(s))
    c = -u.sum(1, keepdim=True) * p
    if state["d_entropy"] is not None:
        c = c - state["d_entropy"][:, None] * p * (logp + state["entropy"][:, None])
    # (sums over all rows of the catalogue, of which little is left: 4096 at a time in 32 bits, these added in 64)
    m, n = s.shape
    pad = -n % 4096
    c = torch.nn.functional.pad(c, (0, pad)).view(m, -1, 4096).transpose(0, 1)
    part = torch.nn.functional.pad(rows, (0, 0, 0, pad)).view(-1, 4096, dim)
    d = torch.bmm(c, part).sum(0, dtype=torch.float64) + (u[:, :, None] * rows[state["given"].clamp(min=0).long()]).sum(1)
    return (d * state["scale"]).float()


# ---- one pass ----------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if not own:
        if case["kind"] == "quantize":
            return _values(state["x"])
        if case["kind"] == "scores":
            return _scores(state).to(getattr(torch, case["dtype"]))
        return _logprobs(state) if case["kind"] == "logprobs" else _backward(state)
    import paper_2003_05622_amd as hps
    if case["kind"] == "quantize":
        return hps.mx4_quantize(state["x"], values=True)[1]
    queries, rows = hps.Mx4Rows(*state["queries"], case["dim"]), hps.Mx4Rows(*state["rows"], case["dim"])
    if case["kind"] == "scores":
        return hps.mx4_scores(queries, rows, scale=state["scale"], bias=state["bias"], dtype=getattr(torch, case["dtype"]))
    if case["kind"] == "backward":
        return hps.mx4_logprobs_backward(queries, rows, state["given"], state["d_logp"], state["lse"], entropy=state["entropy"],
                                         d_entropy=state["d_entropy"], scale=state["scale"], bias=state["bias"])
    got = hps.mx4_logprobs(queries, rows, given=state["given"] if case["given"] else None, top=case["top"],
                           scale=state["scale"], bias=state["bias"])
    out = {"lse": got.lse, "entropy": got.entropy}
    if case["given"]:
        out["logp"] = got.logp
    if case["top"]:
        out["top_index"], out["top_logp"] = got.top_index, got.top_logp
    return out


def work(case):
    m, n, dim = case["m"], case["n"], case["dim"]
    row = _row_bytes(dim) + (dim + 31) // 32
    size = 2 if case["dtype"] == "bfloat16" else 4
    if case["kind"] == "quantize":
        return {"bytes": n * (dim * (size + 4) + row), "flops": 2 * n * dim}
    read = (m + n) * row + (4 * n if case["bias"] else 0)
    if case["kind"] == "scores":
        return {"bytes": read + m * n * size, "flops": 2 * m * n * dim}
    if case["kind"] == "logprobs":
        return {"bytes": read + 4 * m * (2 + 2 * case["given"] + 2 * case["top"]), "flops": 2 * m * n * dim}
    return {"bytes": read + 4 * m * (2 + 2 * case["given"] + dim), "flops": 4 * m * n * dim}


# ---- the definition in 64 bits -----------------------------------------------------------------

def _power(e):
    """2^e in 64 bits, by its bits (a power function may be a last place off)."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _meaning(held, dim):
    """The numbers that held rows stand for, sign, exponent and fraction bits read one by one."""
    codes, scales = held
    one_by_one = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        c = codes.int() >> 4 * half
        e, f = c >> 1 & 3, (c & 1).double()
        magnitude = torch.where(e == 0, 0.5 * f, (1 + 0.5 * f) * _power(e - 1))
        one_by_one[:, half::2] = torch.where((c & 8) != 0, -magnitude, magnitude)
    block = torch.arange(dim, device=codes.device) // 32
    return one_by_one[:, :dim] * _power(scales.long() - 127)[:, block]


def exact(case, seed):
    state = prepare(case, seed)
    dim = case["dim"]
    if case["kind"] == "quantize":
        x = state["x"].double()
        grid = torch.tensor([0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0], dtype=torch.float64, device="cuda")   # even ones first
        for first in range(0, dim, 32):
            part = x[:, first:first + 32]
            exponent = (part.abs().amax(1, keepdim=True).view(torch.int64) >> 52) - 1023
            unit = _power(exponent - 2)
            best, off = torch.zeros_like(part), torch.full_like(part, math.inf)
            for g in grid.tolist():
                d = ((part / unit).abs() - g).abs()
                best, off = torch.where(d < off, torch.full_like(part, g), best), torch.minimum(d, off)
            x[:, first:first + 32] = torch.sign(part) * best * unit
        return x
    rows = _meaning(state["rows"], dim)
    scale = float(torch.tensor(state["scale"], dtype=torch.float32))
    s = torch.mm(_meaning(state["queries"], dim), rows.t()).mul_(scale)
    if case["bias"]:
        s += torch.where(torch.isfinite(state["bias"]), state["bias"].double(), -math.inf)
    if case["kind"] == "scores":
        return s
    lse = torch.logsumexp(s, 1)
    if case["kind"] == "logprobs":
        out = {"lse": lse}
        best = torch.topk(s, min(case["top"], case["n"]), 1).values if case["top"] else None
        if case["given"]:
            where = state["given"].long()
            picked = s.gather(1, where.clamp(min=0))
            picked = torch.where(picked == -math.inf, picked, picked - lse[:, None])
            out["logp"] = torch.where(where < 0, 0.0, picked)
        s = torch.where(s == -math.inf, s, s - lse[:, None])
        out["entropy"] = -torch.special.xlogy(s.exp(), s.exp()).sum(1)
        if case["top"]:
            out["top_index"] = None
            fill = torch.full((case["m"], case["top"] - best.shape[1]), -math.inf, dtype=torch.float64, device="cuda")
            best = torch.where(best == -math.inf, best, best - lse[:, None])
            out["top_logp"] = torch.cat((best, fill), 1)
        return {k: out[k] for k in ("lse", "entropy", "logp", "top_index", "top_logp") if k in out}
    # the gradient, by the chain rule over log p
    p = torch.where(s == -math.inf, 0.0, (s - lse[:, None]).exp())
    where = state["given"].long()
    u = torch.where((where >= 0) & (s.gather(1, where.clamp(min=0)) > -math.inf), state["d_logp"].double(), 0.0)
    d_s = torch.zeros_like(s).scatter_add_(1, where.clamp(min=0), u) - p * u.sum(1, keepdim=True)
    if state["d_entropy"] is not None:
        h = -torch.special.xlogy(p, p).sum(1, keepdim=True)
        d_s -= state["d_entropy"].double()[:, None] * (torch.special.xlogy(p, p) + p * h)
    return torch.mm(d_s, rows) * scale
