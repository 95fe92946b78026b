"""The operators between a drafter's last hidden state and its next input, as timed cases.

  quantize   a matrix in 4 bits (e2m1) with a power-of-two scale for each 32 values of a row, and read back as the values it stands for
  rows       rows of such a matrix by token, the inputs of a drafter whose embedding is its head's matrix
  logits     hidden states, in 4 bits as above or in 8 bits (e4m3) with a scale for each 128 values, times the head's weight in 4 bits
  sample     one token for each row of logits, every row with its own temperature, top-k, top-p and min-p, from given uniforms

Sizes: the vocabularies of this repository's workloads (32000, 128256, 151936) and odd ones between them, batches of one sequence up to a
verified round of 64 sequences with 17 positions, hidden sizes from 128 to 5120.  Hidden states are normalised rows with a spread of scales
over the channels, as behind a norm with a learned gain; weights are N(0, 0.02^2) with a spread over the rows.  Rows of logits are N(0, s^2) with s
between 1/2 and 4, half of them with one token far above the others, as a model's rows are where it is sure of the next token; masked ones
have 30 % of their tokens at -inf, as constrained decoding leaves them.

With `own` false the operators are computed in elementary torch operations, in 32 bits (sampling, whose decisions have borders: in 64) and
rounded once; with it true by the library.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK, BLOCK8, WIDTH = 32, 128, 128             # values to a scale in 4 and in 8 bits; rows are filled up to whole WIDTHs
MOST_ELEMENTS = 128256 * 4096                   # of a quantized matrix
MOST_LOOKUP = 8192 * 4096                       # values of a lookup
MOST_LOGITS = 1088 * 128256 * 4096              # products of a head's call
MOST_ROWS = 1088                                # rows to sample from
# (temperature, top_k, top_p, min_p) of rows of one batch whose users ask for different things; zeros and ones switch a filter off
MIXED = ((1.0, 50, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 0, 0.95, 0.0), (0.7, 0, 0.9, 0.0), (0.8, 40, 1.0, 0.0), (1.0, 0, 1.0, 0.05), (1.0, 0, 1.0, 0.0),
         (0.6, 20, 0.95, 0.02), (1.3, 0, 0.5, 0.0), (1.5, 200, 1.0, 0.1), (0.9, 1000, 0.99, 0.0))
UNIFORM = {"topk_topp": (1.0, 50, 0.9, 0.0), "topp": (0.8, 0, 0.9, 0.0), "minp": (1.2, 0, 1.0, 0.05), "plain": (1.0, 0, 1.0, 0.0)}


def listed():
    return [
        # the hidden states of one draft step, on their way into a 4-bit head: latency alone
        dict(name="quantize_draft_rows", kind="quantize", rows=64, cols=4096, dtype="bf16"),
        # a checkpoint's head, once per load
        dict(name="quantize_head", kind="quantize", rows=128256, cols=4096, dtype="bf16"),
        # the inputs of a batch's next draft position
        dict(name="rows_draft_64", kind="rows", n=64, V=128256, cols=2048, dtype="bf16"),
        # the inputs of a long prompt
        dict(name="rows_prompt", kind="rows", n=8192, V=151936, cols=4096, dtype="bf16"),
        # one user's draft step over a small vocabulary: the weight once through the memory
        dict(name="logits_one_user", kind="logits", N=1, V=32000, K=1024, hidden=4, out="f32"),
        # a draft step of the benchmark's batch
        dict(name="logits_draft_64", kind="logits", N=64, V=128256, K=2048, hidden=8, out="bf16"),
        # the target's rows of a whole round, 64 sequences of 17 positions: matrix-bound
        dict(name="logits_verify_round", kind="logits", N=1088, V=128256, K=4096, hidden=4, out="bf16"),
        # few sequences with long drafts, a vocabulary that fills no tile, fp16 rows
        dict(name="logits_long_drafts", kind="logits", N=325, V=50257, K=5120, hidden=8, out="f16"),
        # one user's token, small vocabulary: launches and latency
        dict(name="sample_one_user", kind="sample", N=1, V=32000, dtype="f32", mode="topk_topp", masked=False),
        # the benchmark's batch, each user with settings of their own
        dict(name="sample_batch_mixed", kind="sample", N=64, V=128256, dtype="bf16", mode="mixed", masked=False),
        # every position of a whole round, mixed settings, the largest vocabulary
        dict(name="sample_round_mixed", kind="sample", N=1088, V=151936, dtype="bf16", mode="mixed", masked=False),
        # constrained decoding by nucleus over an odd vocabulary
        dict(name="sample_masked_nucleus", kind="sample", N=325, V=50257, dtype="f16", mode="topp", masked=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _vocabulary(rng):
    return rng.choice([32000, 128256, 151936, _log_uniform(rng, 1000, 151936), _log_uniform(rng, 1000, 151936)])


def draw(rng):
    kind = rng.choice(["quantize", "rows", "logits", "logits", "sample", "sample"])
    if kind == "quantize":
        cols = _log_uniform(rng, 64, 8192)
        return dict(kind=kind, rows=_log_uniform(rng, 1, min(151936, MOST_ELEMENTS // cols)), cols=cols, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
    V = _vocabulary(rng)
    if kind == "rows":
        cols = _log_uniform(rng, 64, 4096)
        return dict(kind=kind, n=_log_uniform(rng, 1, min(8192, MOST_LOOKUP // cols)), V=V, cols=cols, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
    if kind == "logits":
        K, hidden = WIDTH * _log_uniform(rng, 1, 40), rng.choice([4, 8])
        return dict(kind=kind, N=_log_uniform(rng, 1, min(1088, MOST_LOGITS // (V * K))), V=V, K=K, hidden=hidden,
                    out=rng.choice(["bf16", "bf16", "f16", "f32"] if hidden == 4 else ["bf16", "f16"]))
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    return dict(kind=kind, N=_log_uniform(rng, 1, MOST_ROWS // (2 if dtype == "f32" else 1)), V=V, dtype=dtype,
                mode=rng.choice(["mixed", "mixed", "topk_topp", "topp", "minp", "plain"]), masked=rng.random() < 0.25)


# ---- inputs ------------------------------------------------------------------------------------------------------------------------

def _matrix(rows, cols, dtype, g, scale, spread_rows):
    """N(0, scale^2) times a log-normal spread (factor 1.35 for one standard deviation) over the rows or over the columns."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    s = torch.randn(rows if spread_rows else cols, device="cuda", generator=g).mul_(0.3).exp_()
    x *= (s[:, None] if spread_rows else s[None, :]) * scale
    return x.to(dtype)


def _power_below(amax, most_mantissa, most_exponent):
    """The least e >= -127 with amax <= most_mantissa * 2^(e + most_exponent), most_mantissa in [0.5, 1); 0 for an amax of 0."""
    mantissa, exponent = torch.frexp(amax)                       # amax = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = (exponent - most_exponent + (mantissa > most_mantissa).int()).clamp_(-127, 127)
    return torch.where(amax > 0, e, 0)


def _rounded4(x):
    """x in blocks of 32 of a row (filled up with zeros to whole WIDTHs): multiples of the block's power of two on e2m1's grid, and the powers."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -cols % WIDTH)).view(rows, -1, BLOCK)
    e = _power_below(x.abs().amax(2), 0.75, 3)                   # 6 = 0.75 * 2^3
    y = x * ((127 - e) << 23).view(torch.float32)[:, :, None]    # times 2^-e, exactly
    size = y.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    return torch.round(y / step) * step, e


def _quantized4(x):
    """Codes, two to a byte, the even column's in the low half, and scales (e8m0) of x."""
    y, e = _rounded4(x)
    size = y.abs()
    code = torch.where(size < 2, size * 2, torch.where(size < 4, size + 2, size / 2 + 4)).to(torch.uint8) | (y < 0).to(torch.uint8) << 3
    code = code.view(x.shape[0], -1, 2)
    return (code[:, :, 0] | code[:, :, 1] << 4).view(torch.float4_e2m1fn_x2), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _values4(codes, scale, dtype):
    """The numbers that a 4-bit matrix stands for."""
    b = codes.view(torch.uint8)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=b.device, dtype=dtype)
    code = torch.stack([b & 15, b >> 4], 2).view(b.shape[0], -1)
    v = grid[(code & 7).int()]
    v = torch.where(code > 7, -v, v).view(b.shape[0], -1, BLOCK)
    return (v * scale.to(dtype)[:, :, None]).view(b.shape[0], -1)


def _quantized8(x):
    """Codes (e4m3) and scales (e8m0) of x, whose columns are whole blocks of 128."""
    x = x.float().view(x.shape[0], -1, BLOCK8)
    e = _power_below(x.abs().amax(2), 0.875, 9)                  # 448 = 0.875 * 2^9
    codes = (x * ((127 - e) << 23).view(torch.float32)[:, :, None]).view(x.shape[0], -1).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _values8(codes, scale, dtype):
    return codes.to(dtype).mul_(scale.to(dtype).repeat_interleave(BLOCK8, 1))


def _pieces(rows, cols, most=1 << 27):
    step = max(1, most // cols)
    return [(i, min(rows, i + step)) for i in range(0, rows, step)]


def _by_pieces(x, f):
    """f's pair of bytewise matrices of x, made piece by piece of its rows."""
    parts = [f(x[i:j]) for i, j in _pieces(*x.shape)]
    return tuple(torch.cat([p[k].view(torch.uint8) for p in parts]).view(parts[0][k].dtype) for k in (0, 1))


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    if kind == "quantize":                                       # a handful of rows are hidden states, many a weight
        few = case["rows"] <= MOST_ROWS
        return dict(x=_matrix(case["rows"], case["cols"], DTYPES[case["dtype"]], g, 1.0 if few else 0.02, not few))
    if kind == "rows":
        q, scale = _by_pieces(_matrix(case["V"], case["cols"], torch.bfloat16, g, 0.02, True), _quantized4)
        ids = torch.randint(0, case["V"], (case["n"],), device="cuda", generator=g, dtype=torch.int32)
        ids[torch.rand(case["n"], device="cuda", generator=g) < 0.125] = -1              # sequences that have ended
        return dict(q=q, scale=scale, ids=ids)
    if kind == "logits":
        N, V, K = case["N"], case["V"], case["K"]
        hidden, weight = _matrix(N, K, torch.bfloat16, g, 1.0, False), _matrix(V, K, torch.bfloat16, g, 0.02 * max(1.0, math.sqrt(2048 / K)), True)
        hq, hs = (_quantized4 if case["hidden"] == 4 else _quantized8)(hidden)
        wq, ws = _by_pieces(weight, _quantized4)
        return dict(hq=hq, hs=hs, wq=wq, ws=ws)
    N, V = case["N"], case["V"]
    z = torch.randn(N, V, device="cuda", generator=g)
    r = torch.rand(5, N, device="cuda", generator=g)
    z *= (0.5 * torch.pow(8.0, r[0]))[:, None]
    sure = torch.where(r[1] < 0.5, 8.0 + 6.0 * r[2], 0.0)
    at = (r[3] * V).long().clamp_(max=V - 1)
    z.scatter_add_(1, at[:, None], sure[:, None])
    if case["masked"]:
        z.masked_fill_(torch.rand(N, V, device="cuda", generator=g) < 0.3, -math.inf)
    row = -(-V // 8) * 8                                         # rows begin on 16 bytes
    logits = torch.empty(N, row, dtype=DTYPES[case["dtype"]], device="cuda")[:, :V]
    logits.copy_(z)
    if case["mode"] == "mixed":
        which = (r[4] * len(MIXED)).long().clamp_(max=len(MIXED) - 1)
        settings = torch.tensor(MIXED, device="cuda")[which]
    else:
        settings = torch.tensor(UNIFORM[case["mode"]], device="cuda").repeat(N, 1)
    T, k, p, m = settings.T
    return dict(logits=logits, temperature=T.contiguous(), top_k=k.int().contiguous(), top_p=p.contiguous(), min_p=m.contiguous(),
                u=torch.rand(N, device="cuda", generator=g))


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind = case["kind"]
    empty = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if kind == "quantize":
        K = -(-case["cols"] // WIDTH) * WIDTH
        s["q"] = empty(case["rows"], K // 2, dtype=torch.uint8).view(torch.float4_e2m1fn_x2)
        s["scale"] = empty(case["rows"], K // BLOCK, dtype=torch.uint8).view(torch.float8_e8m0fnu)
        s["values"] = empty(case["rows"], case["cols"], dtype=DTYPES[case["dtype"]])
    elif kind == "rows":
        s["values"] = empty(case["n"], case["cols"], dtype=DTYPES[case["dtype"]])
    elif kind == "logits":
        s["logits"] = empty(case["N"], -(-case["V"] // 8) * 8, dtype=DTYPES[case["out"]])[:, :case["V"]]
    else:
        s["token"], s["kept"] = empty(case["N"], dtype=torch.int32), empty(case["N"], dtype=torch.int32)
        s["prob"] = empty(case["N"])
    if own:                                                      # the scratch memory that a user of the library keeps beside these buffers
        import paper_2411_18462_amd as svip

        if kind == "logits":
            s["workspace"] = svip.new_head_workspace(svip.HEAD_LOGITS_MX, DTYPES[case["out"]], case["N"], case["V"], case["K"])
        elif kind == "sample":
            s["workspace"] = svip.new_sample_workspace(DTYPES[case["dtype"]], case["N"], case["V"])
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------------------

def _own(s):
    import paper_2411_18462_amd as svip

    kind = s["case"]["kind"]
    if kind == "quantize":
        svip.quantize_mx(s["x"], q_out=s["q"], scale_out=s["scale"])
        svip.mx_rows(s["q"], s["scale"], out=s["values"])
        return {"values": s["values"]}
    if kind == "rows":
        svip.mx_rows(s["q"], s["scale"], ids=s["ids"], out=s["values"])
        return {"values": s["values"]}
    if kind == "logits":
        svip.head_logits_mx(s["hq"], s["hs"], s["wq"], s["ws"], logits_out=s["logits"], workspace=s["workspace"])
        return {"logits": s["logits"]}
    svip.sample(s["logits"], u=s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], token_out=s["token"],
                prob_out=s["prob"], kept_out=s["kept"], workspace=s["workspace"])
    return {"token": s["token"], "prob": s["prob"], "kept": s["kept"]}


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "quantize":
        y, e = _rounded4(s["x"])
        return {"values": torch.ldexp(y, e[:, :, None]).view(case["rows"], -1)[:, :case["cols"]].to(s["x"].dtype)}
    if kind == "rows":
        at = s["ids"].clamp(min=0).long()
        v = _values4(s["q"].view(torch.uint8)[at], s["scale"].view(torch.uint8)[at].view(torch.float8_e8m0fnu), torch.float32)[:, :case["cols"]]
        return {"values": torch.where(s["ids"][:, None] < 0, 0.0, v).to(DTYPES[case["dtype"]])}
    if kind == "logits":
        hidden = (_values4 if case["hidden"] == 4 else _values8)(s["hq"], s["hs"], torch.float32)
        return {"logits": (hidden @ _values4(s["wq"], s["ws"], torch.float32).T).to(DTYPES[case["out"]])}
    # sampling: every filter is a threshold on the value, so that equal logits stay or go together
    z = s["logits"].float()
    N, V = z.shape
    greedy = s["temperature"] == 0
    T = torch.where(greedy, 1.0, s["temperature"]).double()[:, None]
    down = z.sort(1, descending=True).values
    top = down[:, :1]
    k = torch.where(s["top_k"] > 0, s["top_k"], V).clamp(max=V).long()[:, None]
    threshold = down.gather(1, k - 1)
    run = torch.where(down >= threshold, ((down - top.double()) / T).exp_(), 0.0).cumsum_(1)
    p = s["top_p"].double()[:, None]
    reached = (run < p * run[:, -1:]).sum(1, keepdim=True).clamp_(max=V - 1)             # the first rank whose cumulative mass is p of all
    threshold = torch.where(p < 1, torch.maximum(threshold, down.gather(1, reached)), threshold)
    del run, down
    x = (z - top.double()) / T
    keep = (z >= threshold) & (x >= s["min_p"].double().log()[:, None]) & (z > -math.inf)
    w = torch.where(keep, x.exp_(), 0.0)
    run = w.cumsum(1)
    total = run[:, -1:]
    token = (run <= s["u"].double()[:, None] * total).sum(1, keepdim=True)
    first = torch.where(z == top, torch.arange(V, device=z.device), V).amin(1, keepdim=True)
    token = torch.where(greedy[:, None], first, token)
    return {"token": token[:, 0].int(), "prob": torch.where(greedy, 1.0, (w.gather(1, token) / total)[:, 0]).float(),
            "kept": torch.where(greedy, 1, keep.sum(1)).int()}


def run(s):
    return _own(s) if own else _plain(s)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "quantize":                                       # the values in, the codes and their scales, the values back
        rows, cols = case["rows"], case["cols"]
        K = -(-cols // WIDTH) * WIDTH
        return {"bytes": 2 * rows * cols * SIZE[case["dtype"]] + rows * (K // 2 + K // BLOCK), "flops": 3 * rows * cols}
    if kind == "rows":                                           # (a row in eight is zeros: no code is read for it)
        n, cols = case["n"], case["cols"]
        K = -(-cols // WIDTH) * WIDTH
        return {"bytes": n * 7 // 8 * (K // 2 + K // BLOCK) + 4 * n + n * cols * SIZE[case["dtype"]], "flops": n * cols}
    if kind == "logits":
        N, V, K = case["N"], case["V"], case["K"]
        hidden = N * K // 2 + N * K // BLOCK if case["hidden"] == 4 else N * K + N * K // BLOCK8
        return {"bytes": hidden + V * K // 2 + V * K // BLOCK + N * V * SIZE[case["out"]], "flops": 2 * N * V * K}
    N, V = case["N"], case["V"]
    return {"bytes": N * V * SIZE[case["dtype"]] + 32 * N, "flops": 4 * N * V}


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------------------------

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_rounded(x):
    """Block by block: the scale is the least power of two (2^-127 or more) that brings the block's largest magnitude to 6 or less; a value
    becomes the nearest of e2m1's, of two as near the one with an even code."""
    rows, cols = x.shape
    K = -(-cols // WIDTH) * WIDTH
    v = torch.zeros(rows, K, dtype=torch.float64, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, K // BLOCK, BLOCK)
    most = v.abs().amax(2, keepdim=True) / 6.0
    e = torch.where(most > 0, most.log2().ceil(), 0.0)
    e = torch.where(most > torch.exp2(e), e + 1, torch.where((most > 0) & (most <= torch.exp2(e - 1)), e - 1, e)).clamp_(min=-127)
    scale = torch.exp2(e)
    size = v.abs() / scale
    near = torch.zeros_like(size)
    for code in range(1, 8):                                     # past the middle between two neighbours, or on it towards an even code
        middle = (GRID[code - 1] + GRID[code]) / 2
        near = torch.where((size >= middle) if code % 2 == 0 else (size > middle), GRID[code], near)
    return (near * scale * v.sign()).view(rows, K)[:, :cols]


def _exact_values(codes, scale, block):
    """A matrix from its codes: 4 bits (two to a byte) or e4m3, sign, exponent and mantissa taken apart."""
    b = codes.view(torch.uint8).long()
    if block == BLOCK:
        b = torch.stack([b % 16, b // 16], 2).flatten(1)
        exponent, mantissa, sign, bias, bits = b // 2 % 4, b % 2, b // 8, 1, 1
    else:
        exponent, mantissa, sign, bias, bits = b // 8 % 16, b % 8, b // 128, 7, 3
    fraction = mantissa.double() / 2 ** bits + (exponent > 0)
    size = torch.ldexp(fraction, exponent.clamp(min=1) - bias)
    power = torch.exp2(scale.view(torch.uint8).double() - 127)
    return torch.where(sign > 0, -size, size).mul_(power.repeat_interleave(block, 1))


def _exact_sample(z, T, k, p, m, u):
    """One row from its sorted values: thresholds by walking down the distinct values."""
    value, at, count = torch.unique(z[z > -math.inf], return_inverse=True, return_counts=True)[0:3]
    value, count = value.flip(0), count.flip(0)                  # downwards
    if T == 0:
        return 1.0
    w = torch.exp((value - value[0]) / T)
    have = count.cumsum(0)
    end = len(value) if k == 0 or k >= z.numel() else int((have < k).sum()) + 1
    mass = (w * count)[:end].cumsum(0)
    if p < 1:
        end = min(end, int((mass < p * mass[-1]).sum()) + 1)
    if m > 0:
        end = min(end, int((value - value[0] >= T * math.log(m)).sum()))
    kept = torch.where(z >= value[end - 1], torch.exp((z - value[0]) / T), 0.0)
    prefix = kept.cumsum(0)
    token = int(torch.searchsorted(prefix, u * float(prefix[-1]), right=True))
    return float(kept[token] / prefix[-1])


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        return {"values": torch.cat([_exact_rounded(s["x"][i:j]) for i, j in _pieces(case["rows"], case["cols"])])}
    if kind == "rows":
        out = torch.zeros(case["n"], case["cols"], dtype=torch.float64, device="cuda")
        use = s["ids"] >= 0
        at = s["ids"][use].long()
        out[use] = _exact_values(s["q"].view(torch.uint8)[at], s["scale"].view(torch.uint8)[at], BLOCK)[:, :case["cols"]]
        return {"values": out}
    if kind == "logits":
        hidden = _exact_values(s["hq"], s["hs"], BLOCK if case["hidden"] == 4 else BLOCK8)
        parts = [hidden @ _exact_values(s["wq"].view(torch.uint8)[i:j], s["ws"].view(torch.uint8)[i:j], BLOCK).T for i, j in _pieces(case["V"], case["K"])]
        return {"logits": torch.cat(parts, 1)}
    settings = zip(s["temperature"].tolist(), s["top_k"].tolist(), s["top_p"].tolist(), s["min_p"].tolist(), s["u"].tolist())
    prob = [_exact_sample(z.double(), *how) for z, how in zip(s["logits"], settings)]
    return {"token": None, "prob": torch.tensor(prob, dtype=torch.float64, device="cuda"), "kept": None}
