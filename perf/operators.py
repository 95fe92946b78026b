"""The operators of a model's head, the layer whose logits every other call of this library reads or judges, as timed cases.

  quantize   a matrix in 8 bits (e4m3) with a power-of-two scale for each block of 128: rows of hidden states in blocks of 1 x 128,
             weights in blocks of 128 x 128
  logits     the product of two such matrices: hidden states times the head's weight, the rows that draft_step and verify read
  loss       cross entropy of hidden states against target tokens over the whole vocabulary, logits never stored
  step       the same with its gradient: loss, then the gradients of the hidden states and of the weight (a drafter's training step;
             with the head frozen, of the hidden states alone)

Sizes: the vocabularies of this repository's workloads (32000, 128256, 151936) and odd ones between them, batches of one sequence up to
a verified round of 64 sequences with 17 positions, hidden sizes from 128 to 5120.  Hidden states are normalised rows with a spread of
scales over the channels, as behind a norm with a learned gain; weights are N(0, 0.02^2) with a spread over the rows, which gives logits
of standard deviation 1 to 3.  Targets follow the logits' size only by chance; one row in eight carries no target (padding, prompts).

With `own` false the operators are computed in elementary torch operations in 32 bits and rounded once; with it true by the library.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 128
E4M3_MAX = 448.0
MOST_ELEMENTS = 128256 * 4096                   # of a quantized matrix
MOST_LOGITS = 1088 * 128256 * 4096              # products of a head_logits call
MOST_LOSS = 8192 * 151936 * 2048                # products of a loss
MOST_STEP = 4096 * 128256 * 4096                # products of each of a step's matrix products


def listed():
    return [
        # the hidden states of one draft step, on their way into an 8-bit head: latency alone
        dict(name="quantize_draft_rows", kind="quantize", rows=64, cols=4096, block_rows=1, dtype="bf16"),
        # a checkpoint's head, once per load (or per training step): a copy that narrows
        dict(name="quantize_head", kind="quantize", rows=128256, cols=4096, block_rows=128, dtype="bf16"),
        # an odd number of rows and columns, whole blocks nowhere at the edges
        dict(name="quantize_ragged_f32", kind="quantize", rows=5001, cols=1000, block_rows=128, dtype="f32"),
        # one user's draft step over a small vocabulary: the weight once through the memory
        dict(name="logits_one_user", kind="logits", N=1, V=32000, K=1024, out="f32"),
        # a draft step of the benchmark's batch
        dict(name="logits_draft_64", kind="logits", N=64, V=128256, K=2048, out="bf16"),
        # the target's rows of a whole round, 64 sequences of 17 positions: matrix-bound
        dict(name="logits_verify_round", kind="logits", N=1088, V=128256, K=4096, out="bf16"),
        # few sequences with long drafts, a vocabulary that fills no tile, fp16 rows
        dict(name="logits_long_drafts", kind="logits", N=325, V=50257, K=5120, out="f16"),
        # scoring one sequence's tokens with a small model
        dict(name="loss_short_f16", kind="loss", N=129, V=32000, D=1024, dtype="f16", T=1.0),
        # evaluation of a long batch over the largest vocabulary
        dict(name="loss_long", kind="loss", N=8192, V=151936, D=2048, dtype="bf16", T=1.0),
        # the smallest training step: a handful of rows, fp32
        dict(name="step_few_rows_f32", kind="step", N=17, V=32000, D=512, dtype="f32", T=1.0, frozen=False),
        # a drafter of hidden size 4096 on one batch of 4096 tokens
        dict(name="step_batch", kind="step", N=4096, V=128256, D=4096, dtype="bf16", T=1.0, frozen=False),
        # the head shared with the target and frozen, a tempered distillation set, odd sizes
        dict(name="step_frozen_odd", kind="step", N=1501, V=50257, D=1032, dtype="bf16", T=2.0, frozen=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _vocabulary(rng):
    return rng.choice([32000, 128256, 151936, _log_uniform(rng, 1000, 151936), _log_uniform(rng, 1000, 151936)])


def draw(rng):
    kind = rng.choice(["quantize", "logits", "logits", "loss", "step", "step"])
    if kind == "quantize":
        cols = _log_uniform(rng, 64, 8192)
        return dict(kind=kind, rows=_log_uniform(rng, 1, min(151936, MOST_ELEMENTS // cols)), cols=cols, block_rows=rng.choice([1, 128]),
                    dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
    V = _vocabulary(rng)
    if kind == "logits":
        K = BLOCK * _log_uniform(rng, 1, 40)
        return dict(kind=kind, N=_log_uniform(rng, 1, min(1088, MOST_LOGITS // (V * K))), V=V, K=K, out=rng.choice(["bf16", "bf16", "f16", "f32"]))
    D, dtype = 8 * _log_uniform(rng, 16, 512), rng.choice(["bf16", "bf16", "f16", "f32"])
    most = (MOST_LOSS if kind == "loss" else MOST_STEP) // (4 if dtype == "f32" else 1)
    c = dict(kind=kind, N=_log_uniform(rng, 1, min(8192 if kind == "loss" else 4096, most // (V * D))), V=V, D=D, dtype=dtype,
             T=rng.choice([1.0, 1.0, 0.7, 2.0]))
    if kind == "step":
        c["frozen"] = rng.random() < 0.25
    return c


# ---- inputs ------------------------------------------------------------------------------------------------------------------------

def _matrix(rows, cols, dtype, g, scale, spread_rows):
    """N(0, scale^2) times a log-normal spread (factor 1.35 for one standard deviation) over the rows or over the columns."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    s = torch.randn(rows if spread_rows else cols, device="cuda", generator=g).mul_(0.3).exp_()
    x *= (s[:, None] if spread_rows else s[None, :]) * scale
    return x.to(dtype)


def _quantized(x, block_rows):
    """Codes (e4m3) and scales (e8m0) of x in blocks of block_rows x 128, columns filled up with zeros to whole blocks."""
    rows, cols = x.shape
    K, R = -(-cols // BLOCK) * BLOCK, -(-rows // block_rows) * block_rows
    x = torch.nn.functional.pad(x.float(), (0, K - cols, 0, R - rows)).view(R // block_rows, block_rows, K // BLOCK, BLOCK)
    amax = x.abs().amax((1, 3))
    mantissa, exponent = torch.frexp(amax)                       # amax = mantissa * 2^exponent, mantissa in [0.5, 1); 448 = 0.875 * 2^9
    e = (exponent - 9 + (mantissa > 0.875).int()).clamp_(-127, 127)
    e = torch.where(amax > 0, e, 0)
    inverse = ((127 - e) << 23).view(torch.float32)              # 2^-e, exactly
    codes = (x * inverse[:, None, :, None]).view(R, K)[:rows].to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _values(codes, scale, block_rows, dtype):
    """The numbers that an 8-bit matrix stands for."""
    s = scale.to(dtype).repeat_interleave(BLOCK, 1)
    if block_rows > 1:
        s = s.repeat_interleave(block_rows, 0)[:codes.shape[0]]
    return codes.to(dtype).mul_(s)


def _pieces(rows, cols, most=1 << 28):
    step = max(1, most // cols) // BLOCK * BLOCK or BLOCK
    return [(i, min(rows, i + step)) for i in range(0, rows, step)]


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["kind"] == "quantize":
        return dict(x=_matrix(case["rows"], case["cols"], DTYPES[case["dtype"]], g, 1.0 if case["block_rows"] == 1 else 0.02, case["block_rows"] > 1))
    N, V, D = case["N"], case["V"], case.get("D") or case["K"]
    dtype = DTYPES[case.get("dtype", "bf16")]
    hidden, weight = _matrix(N, D, dtype, g, 1.0, False), _matrix(V, D, dtype, g, 0.02 * max(1.0, math.sqrt(2048 / D)), True)
    if case["kind"] == "logits":
        hq, hs = _quantized(hidden, 1)
        parts = [_quantized(weight[i:j], BLOCK) for i, j in _pieces(V, D)]
        return dict(hq=hq, hs=hs, wq=torch.cat([p[0] for p in parts]), ws=torch.cat([p[1].view(torch.uint8) for p in parts]).view(torch.float8_e8m0fnu))
    targets = torch.randint(0, V, (N,), device="cuda", generator=g, dtype=torch.int32)
    targets[torch.rand(N, device="cuda", generator=g) < 0.125] = -100
    counted = (targets >= 0).sum().clamp_(min=1)
    return dict(hidden=hidden, weight=weight, targets=targets, grad_loss=torch.full((N,), 1.0, device="cuda") / counted)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind = case["kind"]
    empty = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if kind == "quantize":
        K = -(-case["cols"] // BLOCK) * BLOCK
        s["codes"] = empty(case["rows"], K, dtype=torch.float8_e4m3fn)
        s["scale"] = empty(-(-case["rows"] // case["block_rows"]), K // BLOCK, dtype=torch.float8_e8m0fnu)
        return s
    N, V = case["N"], case["V"]
    if kind == "logits":
        row = -(-V // 8) * 8                                     # rows begin on 16 bytes
        s["logits"] = empty(N, row, dtype=DTYPES[case["out"]])[:, :V]
    else:
        s["loss"], s["lse"] = empty(N), empty(N)
        if kind == "step":
            s["grad_hidden"] = torch.empty_like(s["hidden"])
            s["grad_weight"] = None if case["frozen"] else torch.empty_like(s["weight"])
    if own:                                                      # the scratch memory that a user of the library keeps beside these buffers
        import paper_2411_18462_amd as svip

        call = {"logits": svip.HEAD_LOGITS, "loss": svip.HEAD_LOSS, "step": svip.HEAD_LOSS_GRAD}[kind]
        s["workspace"] = svip.new_head_workspace(call, DTYPES[case.get("dtype") or case["out"]], N, V, case.get("D") or case["K"])
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------------------

def _own(s):
    import paper_2411_18462_amd as svip

    kind = s["case"]["kind"]
    if kind == "quantize":
        svip.quantize_blocks(s["x"], block_rows=s["case"]["block_rows"], q_out=s["codes"], scale_out=s["scale"])
        return {"codes": s["codes"], "scale": s["scale"]}
    if kind == "logits":
        svip.head_logits(s["hq"], s["hs"], s["wq"], s["ws"], logits_out=s["logits"], workspace=s["workspace"])
        return {"logits": s["logits"]}
    T = s["case"]["T"]
    svip.head_loss(s["hidden"], s["weight"], s["targets"], temperature=T, loss_out=s["loss"], lse_out=s["lse"], workspace=s["workspace"])
    out = {"loss": s["loss"], "lse": s["lse"]}
    if kind == "step":
        svip.head_loss_grad(s["hidden"], s["weight"], s["targets"], temperature=T, lse=s["lse"], grad_loss=s["grad_loss"],
                            grad_hidden_out=s["grad_hidden"], grad_weight_out=s["grad_weight"], workspace=s["workspace"])
        out |= {"grad_hidden": s["grad_hidden"], "grad_weight": s["grad_weight"]}
    return out


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "quantize":
        codes, scale = _quantized(s["x"], case["block_rows"])
        return {"codes": codes, "scale": scale}
    if kind == "logits":
        hidden, weight = _values(s["hq"], s["hs"], 1, torch.float32), _values(s["wq"], s["ws"], BLOCK, torch.float32)
        return {"logits": (hidden @ weight.T).to(DTYPES[case["out"]])}
    hidden, weight = s["hidden"].float(), s["weight"].float()
    valid = s["targets"] >= 0
    target = s["targets"].clamp(min=0).long()[:, None]
    z = hidden @ weight.T
    if case["T"] != 1.0:
        z /= case["T"]
    top = z.amax(1, keepdim=True)
    lse = top + (z - top).exp_().sum(1, keepdim=True).log_()
    out = {"loss": torch.where(valid, (lse - z.gather(1, target))[:, 0], 0.0), "lse": lse[:, 0]}
    if kind == "step":
        z.sub_(lse).exp_()
        z.scatter_add_(1, target, torch.full_like(lse, -1.0))
        z *= torch.where(valid, s["grad_loss"] / case["T"], 0.0)[:, None]
        out["grad_hidden"] = (z @ weight).to(s["hidden"].dtype)
        out["grad_weight"] = None if case["frozen"] else (z.T @ hidden).to(s["weight"].dtype)
    return out


def run(s):
    return _own(s) if own else _plain(s)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------------

def work(case):
    if case["kind"] == "quantize":
        rows, K = case["rows"], -(-case["cols"] // BLOCK) * BLOCK
        return {"bytes": rows * case["cols"] * SIZE[case["dtype"]] + rows * K + -(-rows // case["block_rows"]) * (K // BLOCK), "flops": 2 * rows * case["cols"]}
    N, V = case["N"], case["V"]
    if case["kind"] == "logits":
        K = case["K"]
        return {"bytes": N * K + V * K + N * K // BLOCK + -(-V // BLOCK) * K // BLOCK + N * V * SIZE[case["out"]], "flops": 2 * N * V * K}
    D, size = case["D"], SIZE[case["dtype"]]
    w = {"bytes": (N + V) * D * size + 3 * N * 4, "flops": 2 * N * V * D}
    if case["kind"] == "step":                                   # the products of the logits and of either gradient, once each
        w["bytes"] += N * D * size + N * 4 + (0 if case["frozen"] else V * D * size)
        w["flops"] *= 2 if case["frozen"] else 3
    return w


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------------------------

def _exact_quantize(x, block_rows):
    """Codes and scales block by block: the scale is the least power of two (2^-127 or more) that brings the block's largest magnitude to
    448 or less; a code is the nearest multiple of the spacing of 3-bit mantissas at its magnitude, ties to even."""
    rows, cols = x.shape
    K = -(-cols // BLOCK) * BLOCK
    v = torch.zeros(rows, K, dtype=torch.float64, device=x.device)
    v[:, :cols] = x
    per_row = v.abs().view(rows, K // BLOCK, BLOCK).amax(2)
    if block_rows > 1:
        per_row = torch.stack([per_row[i:i + block_rows].amax(0) for i in range(0, rows, block_rows)])
    mantissa, e = torch.frexp(per_row / E4M3_MAX)                # in [0.5, 1) * 2^e: 0.5 is a power of two itself
    e = (e.long() - (mantissa == 0.5).long()).clamp(min=-127)
    scale = torch.where(per_row > 0, _power(e), 1.0)
    each = scale.repeat_interleave(BLOCK, 1)
    if block_rows > 1:
        each = each.repeat_interleave(block_rows, 0)[:rows]
    v /= each
    spacing = _power((torch.frexp(v.abs())[1].long() - 1).clamp(min=-6) - 3)
    return torch.round(v / spacing) * spacing, scale


def _power(e):
    """2^e in 64 bits, exactly."""
    return ((e + 1023) << 52).view(torch.float64)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "quantize":
        parts = [_exact_quantize(s["x"][i:j], case["block_rows"]) for i, j in _pieces(case["rows"], case["cols"], 1 << 27)]
        return {"codes": torch.cat([p[0] for p in parts]), "scale": torch.cat([p[1] for p in parts])}
    if case["kind"] == "logits":
        a, b = _values(s["hq"], s["hs"], 1, torch.float64), _values(s["wq"], s["ws"], BLOCK, torch.float64)
        return {"logits": a @ b.T}
    N, T = case["N"], case["T"]
    W, H, t = s["weight"].double(), s["hidden"].double(), s["targets"].long()
    loss, lse, dH, dW = [], [], [], torch.zeros_like(W) if case["kind"] == "step" and not case["frozen"] else None
    for i, j in _pieces(N, case["V"]):
        z = torch.mm(H[i:j], W.T) / T
        n = torch.logsumexp(z, 1)
        lse.append(n)
        use = t[i:j] >= 0
        at = (torch.arange(j - i, device=z.device)[use], t[i:j][use])
        part = torch.zeros_like(n)
        part[use] = n[use] - z[at]
        loss.append(part)
        if case["kind"] == "step":
            p = torch.softmax(z, 1)
            p[at] -= 1.0
            p *= (use * s["grad_loss"][i:j].double() / T)[:, None]
            dH.append(p @ W)
            if dW is not None:
                dW += p.T @ H[i:j]
    out = {"loss": torch.cat(loss), "lse": torch.cat(lse)}
    if case["kind"] == "step":
        out |= {"grad_hidden": torch.cat(dH), "grad_weight": dW}
    return out
