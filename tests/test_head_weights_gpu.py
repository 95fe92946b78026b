"""Gradients of the head's loss where the rows carry different weights (grad_loss): against the definition in 64 bits, each rounding counted once.

Tolerance of the weight's gradient.  What the products read of G = softmax - one-hot is rounded once, by u of itself.  Up to 64 rows it is m G, m 2^e the rows'
weights with 1/2 < |m| <= 1, in two parts: u^2 in bf16, 2^-22 of two fp16 parts.  fp16 holds it times 2^15, so half a step of its subnormal numbers, 2^-25,
is 2^-40 before the scale and at most 2^-39 of the weight behind 1 / |m| < 2.  The hidden states are multiplied by 2^e up to 64 rows, which rounds nothing, and by
the weight relative to the largest above, which rounds by u unless all weights are equal (a quotient of 1).  fp16 and the parts of fp32 put the
largest |grad_loss x hidden| at 2^13 or above, so that half a step below the normal numbers, 2^-25, is at most 2^-38 of it.  fp32: parts keep 2^-22
of either operand, and the product of the two low parts, 2^-22, is left out; the weighting's quotient and product 2^-23.  Sums: (rows + 2) u32 of the
magnitudes, then the result's own rounding.
"""
import math

import pytest
import torch

from test_head_gpu import ByDefinition, TYPES, U32, gen, inputs, run_loss, tiny, u, within

pytestmark = pytest.mark.gpu

TWO_PARTS = {"bf16": 2.0 ** -16, "f16": 2.0 ** -22, "f32": 2.0 ** -21}


def weight_gradient_off(h, w, y, r, T, dtype, want):
    t, (N, D) = TYPES[dtype], h.shape
    V = w.shape[0]
    H, W = torch.where(want.valid[:, None], h.double(), 0.0), w.double()
    z, f = H @ W.T / T, torch.where(want.valid, r.double().abs() / T, 0.0)[:, None]
    p = torch.softmax(z, 1)
    G = p - torch.zeros_like(p).scatter_(1, y.clamp(0, V - 1).long()[:, None], 1.0)
    d = (H.abs() @ W.abs().T).amax(1) / T * ((D + 4) * U32 + (3 * 2.0 ** -22 if dtype == "f32" else 0.0))
    held = u(t) if N > 64 and dtype != "f32" else TWO_PARTS[dtype]
    hidden = 2.0 ** -21 if dtype == "f32" else u(t) if N > 64 and len(r.unique()) > 1 else 0.0
    off = (torch.expm1(2 * (d + want.lse_off))[:, None] + 6 * U32) * p + (held + hidden) * G.abs() + 2.0 ** -39
    floor = 0.0 if dtype == "bf16" else 2.0 ** -38 * float((f * H.abs()).max()) * (G.abs() * (f > 0)).sum(0)[:, None]
    return (off * f).T @ H.abs() + floor + (N + 2) * U32 * ((G.abs() * f).T @ H.abs()) + u(t) * want.dW.abs() + tiny(t)


def check(svip, h, w, y, r, T, dtype):
    want, got = ByDefinition(h, w, y, T, dtype, r), run_loss(svip, h, w, y, T, r)
    within(got["dw"], want.dW, weight_gradient_off(h, w, y, r, T, dtype, want), "gradient of weight")
    within(got["dh"], want.dH, want.dH_off + 2.0 ** -39 * (torch.where(want.valid, r.abs(), 0.0).double() / T)[:, None] * w.double().abs().sum(0), "gradient of hidden")
    assert (got["dh"][~want.valid] == 0).all()
    return want, got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,D", [(1, 1000, 64), (2, 4099, 136), (8, 515, 1032), (33, 2051, 72), (64, 300, 520), (65, 777, 72), (300, 2000, 256), (513, 1000, 64)])
def test_weights_with_full_mantissas(svip, N, V, D, dtype):
    """Weights with full mantissas, of either sign: up to 64 rows the result's is the only rounding in 16 bits."""
    h, w, y, r = (t.contiguous() for t in inputs(N, V, D, dtype, N + V))
    y[0] = V - 1
    check(svip, h, w, y, r, 0.7 if N % 2 else 1.0, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,D", [(3, 1000, 64), (65, 777, 72), (300, 2000, 256), (513, 1000, 64)])
def test_one_weight_of_all_rows_rounds_nothing(svip, N, V, D, dtype):
    """A mean over the rows: a weight that is no power of two."""
    h, w, y, r = (t.contiguous() for t in inputs(N, V, D, dtype, N + V))
    y[0] = V - 1
    check(svip, h, w, y, torch.full_like(r, 0.37), 1.0, dtype)


@pytest.mark.parametrize("dtype,top", [("f16", 8192.0), ("bf16", 1.0), ("bf16", 1e30), ("f32", 1.0), ("f32", 1e-20)])
@pytest.mark.parametrize("N,V,D", [(7, 900, 64), (64, 2051, 136), (200, 3000, 72), (640, 20000, 520)])
def test_weights_of_very_different_size(svip, N, V, D, dtype, top):
    """From 1e-6 of the largest on: the token of a row of small weight has its -1 from that row alone, an ordinary number of the type."""
    h, w, y, r = (t.contiguous() for t in inputs(N, V, D, dtype, N + D))
    y[:4] = torch.tensor([0, 1, V - 2, V - 1], device="cuda", dtype=torch.int32)
    r = top * 10.0 ** (-6.0 * torch.rand(N, device="cuda", generator=gen(3))) * torch.sign(r)
    r[0], r[1], r[3] = top, top * 1e-6, -top * 2.0 ** -20
    check(svip, h, w, y, r, 1.0, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [20, 200])
def test_rows_of_weight_zero_add_nothing(svip, dtype, N):
    V, D = 700, 64
    h, w, y, r = (t.contiguous() for t in inputs(N, V, D, dtype, 21))
    off = torch.arange(N, device="cuda") % 3 == 1
    r[off] = 0.0
    got, none = run_loss(svip, h, w, y, 1.0, r), run_loss(svip, h, w, torch.where(off, -1, y), 1.0, r)
    assert (got["dh"][off] == 0).all() and torch.equal(got["dh"], none["dh"]) and torch.equal(got["dw"], none["dw"])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [20, 200])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_weight_that_is_no_number_reaches_its_row_and_the_weight(svip, dtype, N, bad):
    V, D = 700, 64
    h, w, y, r = (t.contiguous() for t in inputs(N, V, D, dtype, 22))
    y[2] = 5
    want = run_loss(svip, h, w, y, 1.0, r)
    r[2] = bad
    got = run_loss(svip, h, w, y, 1.0, r)
    others = torch.arange(N, device="cuda") != 2
    assert not got["dh"][2].isfinite().any() and torch.equal(got["dh"][others], want["dh"][others])
    assert not got["dw"].isfinite().any()
