"""The largest sizes that the head's calls take: those whose launches would need more threads than a launch can have (2^32 - 1) are gone through in
pieces, or refused before anything is enqueued."""
import ctypes

import pytest
import torch

import paper_2411_18462_amd as svip

BF = torch.bfloat16


def _pointer():
    buf = ctypes.create_string_buffer(1 << 12)
    return buf, (ctypes.addressof(buf) + 255) & ~255          # a fake, aligned "device" pointer, never dereferenced


@pytest.mark.parametrize("rows,cols", [(262657, 65408), (1 << 22, 4000)])
def test_fp32_blocks_of_one_row_past_a_launch_are_refused(rows, cols):
    """2^27 - 1 blocks of 1 x 128 (7 x 73 x 262657), eight a workgroup of 256, would be 2^32 threads; and more than 2^27 in any type."""
    keep, p = _pointer()
    K = -(-cols // 128) * 128
    assert svip.load().svip_quantize_blocks(p, 0, rows, cols, cols, 1, p, K, p, K // 128, None) == 2
    del keep


@pytest.mark.parametrize("N,D", [(1 << 20, 1 << 14), ((1 << 20) - 3, (1 << 14) - 8), (1 << 17, 1 << 17)])
@pytest.mark.parametrize("dtype", [torch.float32, BF, torch.float16])
def test_gradients_of_too_many_hidden_values_are_refused(N, D, dtype):
    """A thread of the last kernel makes four values of one row; 2^34 of them, rows filled up to fours and channels to 256, are 2^32 threads."""
    keep, p = _pointer()
    V = 1000
    assert svip.head_workspace_bytes(svip.HEAD_LOSS_GRAD, dtype, N, V, D) == 0
    assert svip.head_workspace_bytes(svip.HEAD_LOSS_GRAD, dtype, N // 2, V, D) > 0
    assert svip.head_workspace_bytes(svip.HEAD_LOSS, dtype, N, V, D) > 0
    code = {torch.float32: 0, BF: 1, torch.float16: 2}[dtype]
    assert svip.load().svip_head_loss_grad(p, p, code, N, V, D, D, D, 1.0, p, p, p, p, D, p, D, p, 1 << 60, None) == 2
    del keep


@pytest.mark.gpu
@pytest.mark.parametrize("N,V,D,dtype", [(1 << 20, 1 << 19, 64, BF), (1 << 20, (1 << 19) + 1000, 16, torch.float32)])
def test_loss_of_more_tiles_than_a_launch_takes(N, V, D, dtype):
    """2^23 tiles of 512 threads; and as many rows of fp32 in parts, whose vocabulary goes in pieces.  Checked at rows from everywhere."""
    from test_head_gpu import U32, ByDefinition, gen, within

    g = gen(31)
    h = torch.randn(N, D, device="cuda", generator=g).to(dtype)
    w = torch.randn(V, D, device="cuda", generator=g).mul_(1.5 / D ** 0.5).to(dtype)
    y = torch.randint(0, V, (N,), device="cuda", generator=g, dtype=torch.int32)
    y[::97] = V - 1 - torch.arange(len(y[::97]), device="cuda", dtype=torch.int32) % 300         # (of the last piece, too)
    loss, lse = torch.full((N,), 9.0, device="cuda"), torch.full((N,), 9.0, device="cuda")
    svip.head_loss(h, w, y, loss_out=loss, lse_out=lse, workspace=svip.new_head_workspace(svip.HEAD_LOSS, dtype, N, V, D))
    at = torch.cat([torch.tensor([0, 1, 255, 256, N - 257, N - 1], device="cuda"), torch.randint(0, N, (60,), device="cuda", generator=g)])
    at = torch.cat([at, at // 97 * 97])
    want = ByDefinition(h[at], w, y[at], 1.0, {BF: "bf16", torch.float32: "f32"}[dtype])
    joined = (V // 128 + 1) * U32 * U32                              # (records are joined in 64 bits)
    within(lse[at], want.lse, want.lse_off + joined, "lse")
    within(loss[at], want.loss, want.loss_off + joined, "loss")
    assert ((lse > 0) & (lse < 40) & (loss > -1e-3)).all()
