"""The head's operators against their definitions in 64 bits: 8-bit blocks, logits from them, cross entropy over the vocabulary and its
gradients, and all of them in one drafter's step and round.

Tolerances.  u = finfo.eps / 2 of a type is the most that one rounding is off, relative to the value.
  quantize   exact: the scale is a power of two, the quotient is exact and rounded once.
  logits     products of e4m3 values are exact in fp32 and a row's K of them are summed in fp32: any order is within K u32 of the sum of
             magnitudes; then one rounding to the output type.  16-bit outputs: the 8-bit matrix instructions drop, of 8 products next to one
             another, what lies below 2^-13 of the largest (a product of 2^16 and one of 2^2 next to it sum to 2^16): at most 7 of them,
             each less than 2^-13 of a magnitude in the sum, so 7 x 2^-13 of the sum of magnitudes in all.
  loss, lse  a logit is a sum of D products in fp32 (error at most (D + 2) u32 sum |h w|, fp32 inputs besides: 3 x 2^-22 for the parts); a
             logsumexp is off by no more than its logits are, plus a few u32 of the exponentials and of the result; the loss by twice that.
  gradients  an entry of softmax - one-hot is off by the logits' error d (relative to p: exp(2 d)) and by one rounding to the type that holds it
             (fp32: two parts, 2^-21); the weighted hidden states by one more; the sums by (terms) u32 of the magnitudes; then one rounding
             to the output type, with its smallest number as a floor.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HELD = {"f32": 2.0 ** -21, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}       # rounding of what the products of a gradient are made of


def u(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps      # the spacing below the smallest normal number


def strided(rows, cols, dtype, pad, gen, scale=1.0):
    """A matrix whose rows are `pad` elements further apart than they are long, NaN between them."""
    x = torch.full((rows, cols + pad), float("nan"), dtype=torch.float32, device="cuda")
    x[:, :cols] = torch.randn(rows, cols, device="cuda", generator=gen) * scale
    return x.to(dtype)[:, :cols]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# ---- quantize ------------------------------------------------------------------------------------------------------------------------

def quantize(svip, x, block_rows, pad_q=0, pad_s=0):
    rows, cols = x.shape
    K, R = -(-cols // 128) * 128, -(-rows // block_rows)
    q = torch.full((rows, K + pad_q), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((R, K // 128 + pad_s), 0x55, dtype=torch.uint8, device="cuda")
    svip.quantize_blocks(x, block_rows=block_rows, q_out=q.view(torch.float8_e4m3fn)[:, :K], scale_out=s.view(torch.float8_e8m0fnu)[:, :K // 128])
    assert (q[:, K:] == 0x55).all() and (s[:, K // 128:] == 0x55).all()
    return q[:, :K].contiguous(), s[:, :K // 128].contiguous()


def quantized_by_definition(x, block_rows):
    rows, cols = x.shape
    K, R = -(-cols // 128) * 128, -(-rows // block_rows)
    full = torch.zeros(R * block_rows, K, dtype=torch.float64)
    full[:rows, :cols] = x.double().cpu()
    fin = torch.where(full.isfinite(), full.abs(), 0.0).view(R, block_rows, K // 128, 128).amax((1, 3))
    e = torch.zeros(R, K // 128, dtype=torch.int64)
    for i in range(R):
        for j in range(K // 128):
            a = float(fin[i, j])
            if a:
                n = -127
                while a > 448 * 2.0 ** n:
                    n += 1
                e[i, j] = n
    v = full / (2.0 ** e.double()).repeat_interleave(128, 1).repeat_interleave(block_rows, 0)
    step = 2.0 ** (torch.frexp(v.abs())[1].double() - 1).clamp(min=-6) / 8
    r = (torch.round(v / step) * step)[:rows]
    codes = r.float().to(torch.float8_e4m3fn).view(torch.uint8)           # exact: r is one of its numbers
    return torch.where(r.isfinite(), codes, torch.tensor(0x7f, dtype=torch.uint8)), (e + 127).to(torch.uint8)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 7), (3, 128, 8), (129, 200, 56), (128, 136, 0), (300, 1000, 24)])
def test_quantize(svip, dtype, block_rows, rows, cols, pad):
    t = TYPES[dtype]
    x = strided(rows, cols, t, pad + (-(cols + pad)) % 8, gen(rows + cols))
    x *= torch.exp(2.0 * torch.randn(rows, 1, device="cuda", generator=gen(5))).to(t)
    got, want = quantize(svip, x, block_rows, 16, 3), quantized_by_definition(x, block_rows)
    assert torch.equal(got[1].cpu(), want[1]) and torch.equal(got[0].cpu() & 0x7f, want[0] & 0x7f)
    neg = (want[0] & 0x7f) != 0
    assert torch.equal(got[0].cpu()[neg], want[0][neg])


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_ends_of_the_range(svip, block_rows):
    """Zeros, the largest and smallest numbers, powers of two and 448 times them, ties, infinities and NaN, each in a block of its own."""
    f = torch.finfo(torch.float32)
    heads = [0.0, -0.0, f.max, -f.max, f.smallest_normal, 2.0 ** -149, 448.0, 448.00003, 1.75 * 2.0 ** -120, 1.7500001 * 2.0 ** -120, 2.0 ** 100, 464.0,
             float("inf"), float("-inf"), float("nan"), 1e-30]
    x = torch.zeros(128 if block_rows == 128 else 1, 128 * len(heads))
    for i, h in enumerate(heads):
        block = torch.linspace(-1, 1, 127) * (abs(h) if math.isfinite(h) else 3.0)
        x[-1, 128 * i] = h
        x[-1, 128 * i + 1:128 * (i + 1)] = block
    got, want = quantize(svip, x.cuda(), block_rows), quantized_by_definition(x, block_rows)
    assert torch.equal(got[1].cpu(), want[1])
    same = (got[0].cpu() == want[0]) | ((got[0].cpu() & 0x7f) == 0) & ((want[0] & 0x7f) == 0)
    assert same.all(), torch.nonzero(~same)[:8]


# ---- logits --------------------------------------------------------------------------------------------------------------------------

def eight_bits(rows, K, block_rows, g, pad):
    q = (torch.randn(rows, K + pad, device="cuda", generator=g) * 40).clamp_(-448, 448).to(torch.float8_e4m3fn)
    e = torch.randint(113, 127, (-(-rows // block_rows), K // 128 + 5), device="cuda", generator=g).to(torch.uint8)
    return q[:, :K], e.view(torch.float8_e8m0fnu)[:, :K // 128]


def values(q, s, block_rows):
    return q.double() * s.double().repeat_interleave(128, 1).repeat_interleave(block_rows, 0)[:q.shape[0]]


@pytest.mark.parametrize("N,V,K,out", [(1, 1, 128, "f32"), (1, 1000, 5120, "bf16"), (7, 129, 256, "f16"), (16, 32000, 384, "f32"), (33, 515, 8320, "f32"),
                                       (64, 1283, 1024, "bf16"), (65, 257, 640, "f16"), (130, 2051, 128, "f32"), (257, 1000, 16640, "bf16"),
                                       (300, 4099, 896, "f16"), (1088, 1500, 512, "bf16")])
def test_logits(svip, N, V, K, out):
    g, t = gen(N + V + K), TYPES[out]
    hq, hs = eight_bits(N, K, 1, g, 16)
    wq, ws = eight_bits(V, K, 128, g, 48)
    row = -(-V // 8) * 8 + 8
    z = torch.full((N + 1, row), 7.0, dtype=t, device="cuda")
    workspace = svip.new_head_workspace(svip.HEAD_LOGITS, t, N, V, K)
    svip.head_logits(hq, hs, wq, ws, logits_out=z[:N, :V], workspace=workspace)
    h, w = values(hq, hs, 1), values(wq, ws, 128)
    want, most = h @ w.T, h.abs() @ w.abs().T
    off = (z[:N, :V].double() - want).abs()
    allowed = (K * U32 + (0.0 if out == "f32" else 7 * 2.0 ** -13)) * most + u(t) * want.abs() + tiny(t)
    assert (off <= allowed).all(), float((off / allowed).max())
    assert (z[N] == 7).all() and (z[:, V:] == 7).all()                  # nothing behind the last row or between the rows


def test_logits_nan_code_reaches_its_row_alone(svip):
    g = gen(3)
    hq, hs = eight_bits(5, 256, 1, g, 0)
    wq, ws = eight_bits(300, 256, 128, g, 0)
    hq = hq.clone()
    hq.view(torch.uint8)[2, 200] = 0x7f
    z = torch.zeros(5, 304, device="cuda")
    svip.head_logits(hq, hs, wq, ws, logits_out=z[:, :300], workspace=svip.new_head_workspace(svip.HEAD_LOGITS, torch.float32, 5, 300, 256))
    assert z[2, :300].isnan().all() and z[[0, 1, 3, 4]].isfinite().all()


# ---- loss and gradients --------------------------------------------------------------------------------------------------------------

def inputs(N, V, D, dtype, seed, pad=8):
    g, t = gen(seed), TYPES[dtype]
    h = strided(N, D, t, pad, g)
    w = strided(V, D, t, pad + 16, g, 1.5 / math.sqrt(D))
    y = torch.randint(0, V, (N,), device="cuda", generator=g, dtype=torch.int32)
    y[torch.rand(N, device="cuda", generator=g) < 0.2] = -100
    r = torch.rand(N, device="cuda", generator=g) - 0.3
    return h, w, y, r


class ByDefinition:
    """Loss and gradients in 64 bits, and how far each may be off."""

    def __init__(self, h, w, y, T, dtype, r=None):
        t = TYPES[dtype]
        N, D = h.shape
        V = w.shape[0]
        valid = (y >= 0) & (y < V)
        H, W = torch.where(valid[:, None], h.double(), 0.0), w.double()
        z = H @ W.T / T
        self.valid = valid
        self.lse = torch.logsumexp(z, 1)
        at = y.clamp(0, V - 1).long()[:, None]
        self.loss = torch.where(valid, self.lse - z.gather(1, at)[:, 0], 0.0)
        relative = (D + 4) * U32 + (3 * 2.0 ** -22 if dtype == "f32" else 0.0)
        d = (H.abs() @ W.abs().T).amax(1) / T * relative                 # of a row's logits
        self.lse_off = d + 8 * U32 * (1 + self.lse.abs())
        self.loss_off = torch.where(valid, 2 * d + 8 * U32 * (1 + self.lse.abs() + z.gather(1, at)[:, 0].abs()), 0.0)
        if r is None:
            return
        p = torch.softmax(z, 1)
        one = torch.zeros_like(p).scatter_(1, at, 1.0)
        f = torch.where(valid, r.double() / T, 0.0)[:, None]
        G = (p - one) * f
        drift = (torch.expm1(2 * (d + self.lse_off))[:, None] + 4 * U32) * p      # of p by its logit, its logsumexp and the exponential
        off = (drift + HELD[dtype] * (p - one).abs() + 2.0 ** -40) * f.abs()
        self.dH, self.dW = G @ W, G.T @ H
        self.dH_off = off @ W.abs() + V * U32 * (G.abs() @ W.abs()) + u(t) * self.dH.abs() + tiny(t)
        self.dW_off = off.T @ H.abs() + (N * U32 + HELD[dtype]) * (G.abs().T @ H.abs()) + u(t) * self.dW.abs() + tiny(t)


def within(got, want, most, name):
    off = (got.double() - want).abs()
    assert got.isfinite().all(), name
    assert (off <= most).all(), (name, float((off / most.clamp(min=1e-300)).max()))


SIZES = [(1, 1, 8), (1, 1000, 64), (5, 300, 200), (17, 4099, 136), (64, 2051, 512), (65, 777, 72), (130, 257, 1032), (300, 5001, 256), (513, 1000, 64),
         (1030, 3001, 328)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,D", SIZES)
def test_loss_and_gradients(svip, N, V, D, dtype):
    h, w, y, r = inputs(N, V, D, dtype, N + V + D)
    T = 0.7 if N % 2 else 1.0
    ws = svip.new_head_workspace(svip.HEAD_LOSS_GRAD, h.dtype, N, V, D)
    loss, lse = torch.full((N,), 9.0, device="cuda"), torch.full((N,), 9.0, device="cuda")
    svip.head_loss(h, w, y, temperature=T, loss_out=loss, lse_out=lse, workspace=ws)
    want = ByDefinition(h, w, y, T, dtype, r)
    within(lse[want.valid], want.lse[want.valid], want.lse_off[want.valid], "lse")
    within(loss, want.loss, want.loss_off, "loss")
    dh = torch.full((N + 1, D + 8), 7.0, dtype=h.dtype, device="cuda")
    dw = torch.full((V + 1, D + 24), 7.0, dtype=h.dtype, device="cuda")
    svip.head_loss_grad(h, w, y, temperature=T, lse=lse, grad_loss=r, grad_hidden_out=dh[:N, :D], grad_weight_out=dw[:V, :D], workspace=ws)
    within(dh[:N, :D], want.dH, want.dH_off, "gradient of hidden")
    within(dw[:V, :D], want.dW, want.dW_off, "gradient of weight")
    assert (dh[N] == 7).all() and (dh[:, D:] == 7).all() and (dw[V] == 7).all() and (dw[:, D:] == 7).all()
    assert (dh[:N, :D][~want.valid] == 0).all()
    # either gradient alone, and both again: the same bits
    dh2, dw2 = torch.zeros_like(dh), torch.zeros_like(dw)
    svip.head_loss_grad(h, w, y, temperature=T, lse=lse, grad_loss=r, grad_hidden_out=dh2[:N, :D], workspace=ws)
    svip.head_loss_grad(h, w, y, temperature=T, lse=lse, grad_loss=r, grad_weight_out=dw2[:V, :D], workspace=ws)
    assert torch.equal(dh2[:N, :D], dh[:N, :D]) and torch.equal(dw2[:V, :D], dw[:V, :D])
    assert svip.workspace_flags(ws) == 0
