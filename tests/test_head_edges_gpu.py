"""The head's loss at the ends of what its inputs may be: fp32 rows of very different size (as values and in two fp16 parts), targets at the ends of int32,
one workspace for calls of several sizes."""
import pytest
import torch

from test_head_gpu import TYPES, U32, gen, inputs, run_loss, tiny, u, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,V,D", [(40, 3000, 136), (200, 2000, 64), (1024, 20000, 520)])
def test_fp32_rows_of_very_different_size(svip, N, V, D):
    """Rows of the weight and of the hidden states from 2^-20 of the largest on; the largest sizes go in parts.

    A part keeps 2^-22 of a value, or half a step, 2^-25, below fp16's normal numbers, with the largest of a row of hidden states and of the whole weight at
    2^14 or above: 2^-39 of that largest; the product of two low parts, 2^-22, is left out.  G and the weighted hidden states (largest at
    2^13 or above: 2^-38) likewise.  As values nothing but the sums' (D + 4) u32 is lost, which is less.
    """
    g = gen(N + V)
    size = lambda n: 2.0 ** (-20.0 * torch.rand(n, 1, device="cuda", generator=g))  # noqa: E731
    h = torch.randn(N, D, device="cuda", generator=g) * size(N)
    w = torch.randn(V, D, device="cuda", generator=g) * size(V) * 4.0 / D ** 0.5
    y = torch.randint(0, V, (N,), device="cuda", generator=g, dtype=torch.int32)
    y[::5] = -1
    r = torch.rand(N, device="cuda", generator=g) - 0.3
    got = run_loss(svip, h, w, y, 1.0, r)
    H, W, use = h.double(), w.double(), y >= 0
    at, f = y.clamp(min=0).long()[:, None], torch.where(use, r.double(), 0.0)[:, None]
    z = H @ W.T
    lse = torch.logsumexp(z, 1)
    top = W.abs().max()
    d = (((D + 4) * U32 + 3 * 2.0 ** -22) * (H.abs() @ W.abs().T) + 2.0 ** -39 * (top * H.abs().sum(1)[:, None] + H.abs().amax(1)[:, None] * W.abs().sum(1)[None, :])).amax(1)
    off_lse = d + 8 * U32 * (1 + lse.abs())
    zt = z.gather(1, at)[:, 0]
    within(got["lse"], lse, off_lse, "lse")
    within(got["loss"], torch.where(use, lse - zt, 0.0), torch.where(use, 2 * d + 8 * U32 * (1 + lse.abs() + zt.abs()), 0.0), "loss")
    p = torch.softmax(z, 1)
    G = p - torch.zeros_like(p).scatter_(1, at, 1.0)
    off = ((torch.expm1(2 * (d + off_lse))[:, None] + 6 * U32) * p + 2.0 ** -22 * G.abs() + 2.0 ** -39) * f.abs()
    G = G.abs() * f.abs()
    dH, dW = (p * f) @ W - f * W[at[:, 0]], (p * f).T @ H
    dW.index_add_(0, at[:, 0], -f * H)
    within(got["dh"], dH, off @ W.abs() + (V * U32 + 2.0 ** -21) * (G @ W.abs()) + 2.0 ** -39 * top * G.sum(1)[:, None] + u(h.dtype) * dH.abs() + tiny(h.dtype), "hidden")
    floor = 2.0 ** -38 * float((f.abs() * H.abs()).max()) * (G > 0).double().sum(0)[:, None]        # (|softmax - one-hot| is at most 1)
    within(got["dw"], dW, off.T @ H.abs() + ((N + 2) * U32 + 2.0 ** -21) * (G.T @ H.abs()) + floor + u(h.dtype) * dW.abs() + tiny(h.dtype), "weight")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [9, 90])
def test_targets_at_the_ends_of_int32(svip, dtype, N):
    h, w, y, r = (t.contiguous() for t in inputs(N, 300, 64, dtype, 41))
    ends, none = y.clone(), y.clone()
    for i, v in enumerate((-2 ** 31, -2 ** 31 + 1, 2 ** 31 - 1, 300, -1)):
        ends[i], none[i] = v, -100
    ws = svip.new_head_workspace(svip.HEAD_LOSS_GRAD, h.dtype, N, 300, 64)
    want, got = run_loss(svip, h, w, none, 1.0, r), run_loss(svip, h, w, ends, 1.0, r, ws)
    assert all(torch.equal(want[k], got[k]) for k in want)
    assert svip.workspace_flags(ws) == svip.FLAG_BAD_TOKEN


@pytest.mark.parametrize("dtype", TYPES)
def test_one_workspace_for_calls_of_several_sizes(svip, dtype):
    """As many bytes as the call that needs most, which is not always the one of the most rows; and the calls do not disturb one another."""
    sizes = [(n, 3000, 256) for n in (300, 64, 20, 1, 200, 33)]
    need = [svip.head_workspace_bytes(call, TYPES[dtype], *s) for s in sizes for call in (svip.HEAD_LOGITS, svip.HEAD_LOSS, svip.HEAD_LOSS_GRAD)]
    ws = torch.full((max(need),), 0xff, dtype=torch.uint8, device="cuda")
    ws[:256] = 0
    for N, V, D in sizes:
        h, w, y, r = (t.contiguous() for t in inputs(N, V, D, dtype, N))
        want, got = run_loss(svip, h, w, y, 1.0, r), run_loss(svip, h, w, y, 1.0, r, ws)
        assert all(torch.equal(want[k], got[k]) for k in want)


@pytest.mark.parametrize("dtype,N,V,D", [("f16", 33, 3000, 256), ("f16", 300, 3000, 256), ("bf16", 33, 3000, 256), ("f32", 1024, 20000, 520)])
def test_replayed_graph_of_rows_of_different_weights(svip, dtype, N, V, D):
    """Loss and gradients captured once and replayed over new inputs between eager work, rows of other weights and other rows without a target each
    time; fp32 in parts, whose maxima the workspace holds.  One workspace for the eager calls and the graph, one after the other."""
    h, w, y, r = (t.contiguous() for t in inputs(N, V, D, dtype, 43))
    ws = svip.new_head_workspace(svip.HEAD_LOSS_GRAD, h.dtype, N, V, D)
    out = run_loss(svip, h, w, y, 1.0, r, ws)

    def step():
        svip.head_loss(h, w, y, loss_out=out["loss"], lse_out=out["lse"], workspace=ws)
        svip.head_loss_grad(h, w, y, lse=out["lse"], grad_loss=r, grad_hidden_out=out["dh"], grad_weight_out=out["dw"], workspace=ws)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        g = gen(200 + i)
        h.copy_(torch.randn(N, D, device="cuda", generator=g) * 4.0 ** i)
        w.copy_(torch.randn(V, D, device="cuda", generator=g) * 0.05)
        y.copy_(torch.randint(-V // 4, V, (N,), device="cuda", generator=g))
        r.copy_(10.0 ** (i - 4.0 * torch.rand(N, device="cuda", generator=g)))
        step()
        torch.cuda.synchronize()
        want = {k: v.clone() for k, v in out.items()}
        for v in out.values():
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k in out:
            assert torch.equal(out[k].view(torch.uint8), want[k].view(torch.uint8)), (i, k)


def test_two_calls_at_once_on_streams_of_their_own(svip):
    """fp16 and fp32 in parts, each in its own workspace full of what another call left."""
    cases = [tuple(t.contiguous() for t in inputs(N, V, D, dtype, N)) for N, V, D, dtype in
             ((300, 5000, 256, "f16"), (40, 9000, 136, "f16"), (1024, 20000, 520, "f32"))]
    spaces = [svip.new_head_workspace(svip.HEAD_LOSS_GRAD, h.dtype, h.shape[0], w.shape[0], h.shape[1]) for h, w, _, _ in cases]
    want = [run_loss(svip, h, w, y, 1.0, r) for h, w, y, r in cases]
    for ws in spaces:
        ws[256:] = 0x7f
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], []
    for (h, w, y, r), ws, s in zip(cases, spaces, streams):
        with torch.cuda.stream(s):
            got.append(run_loss(svip, h, w, y, 1.0, r, ws))
    torch.cuda.synchronize()
    assert all(torch.equal(a[k], b[k]) for a, b in zip(want, got) for k in a)
