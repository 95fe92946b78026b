"""The head's calls without a GPU: what they refuse on the host, before anything is enqueued, and their workspace sizes."""
import ctypes

import pytest
import torch

import paper_2411_18462_amd as svip

F32, BF, F16 = torch.float32, torch.bfloat16, torch.float16


def _pointer():
    buf = ctypes.create_string_buffer(1 << 12)
    return buf, (ctypes.addressof(buf) + 255) & ~255          # a fake, aligned "device" pointer, never dereferenced


def test_workspace_bytes_of_the_head():
    f = svip.head_workspace_bytes
    for bad in ((3, BF, 8, 100, 64), (-1, BF, 8, 100, 64), (0, torch.float64, 8, 100, 64), (0, BF, 0, 100, 64), (0, BF, 8, 0, 64), (0, BF, 8, 100, 0),
                (1, BF, (1 << 20) + 1, 100, 64), (1, BF, 8, (1 << 22) + 1, 64), (1, BF, 8, 100, (1 << 17) + 1)):
        assert f(*bad) == 0, bad
        with pytest.raises(svip.SvipError):
            svip.new_head_workspace(*bad)
    for dtype in (F32, BF, F16):
        for N, V, D in ((1, 1, 8), (64, 32000, 512), (65, 32000, 1024), (161, 50257, 4096), (4096, 128256, 4096), (1 << 20, 1 << 22, 64), (300, 151936, 5120)):
            sizes = [f(c, dtype, N, V, D) for c in (svip.HEAD_LOGITS, svip.HEAD_LOSS, svip.HEAD_LOSS_GRAD)]
            assert all(s > 0 and s % 256 == 0 for s in sizes)
            assert sizes[2] >= sizes[1], (dtype, N, V, D)         # one workspace serves a loss and its gradient
    # a batch's logits are not held: 4096 x 128256 of them would be a GiB in 16 bits
    assert f(svip.HEAD_LOSS_GRAD, BF, 4096, 128256, 4096) < 480 << 20


def test_host_checks_of_the_head():
    lib = svip.load()
    keep, p = _pointer()
    N, V, D = 4, 100, 64

    def quantize(**kw):
        a = dict(x=p, dtype=1, rows=5, cols=200, stride=208, block=1, q=p, qs=256, s=p, ss=2)
        a.update(kw)
        return lib.svip_quantize_blocks(a["x"], a["dtype"], a["rows"], a["cols"], a["stride"], a["block"], a["q"], a["qs"], a["s"], a["ss"], None)

    assert quantize(x=None) == 1 and quantize(q=None) == 1 and quantize(s=None) == 1
    assert quantize(dtype=3) == 3 and quantize(dtype=-1) == 3
    assert quantize(rows=0) == 2 and quantize(cols=0) == 2 and quantize(stride=192) == 2 and quantize(qs=240) == 2 and quantize(ss=1) == 2
    assert quantize(rows=(1 << 22) + 1) == 2 and quantize(cols=(1 << 17) + 1, stride=1 << 18, qs=1 << 18, ss=1 << 12) == 2
    assert quantize(rows=1 << 22, cols=4096, stride=4096, qs=4096, ss=32) == 2
    assert quantize(x=p + 1) == 4 and quantize(x=p + 2, dtype=0) == 4 and quantize(q=p + 8) == 4 and quantize(qs=264) == 4
    assert quantize(block=0) == 6 and quantize(block=64) == 6

    def logits(**kw):
        a = dict(h=p, hs=p, w=p, ws=p, N=N, V=V, K=256, sh=256, shs=2, sw=256, sws=2, z=p, dtype=1, row=104, space=p, bytes=1 << 12)
        a.update(kw)
        return lib.svip_head_logits(a["h"], a["hs"], a["w"], a["ws"], a["N"], a["V"], a["K"], a["sh"], a["shs"], a["sw"], a["sws"], a["z"],
                                    a["dtype"], a["row"], a["space"], a["bytes"], None)

    for name in ("h", "hs", "w", "ws", "z"):
        assert logits(**{name: None}) == 1
    assert logits(dtype=5) == 3
    assert logits(N=0) == 2 and logits(V=0) == 2 and logits(K=0) == 2 and logits(K=200) == 2 and logits(sh=128) == 2 and logits(sw=240) == 2
    assert logits(shs=1) == 2 and logits(sws=1) == 2 and logits(row=96) == 2 and logits(sh=(1 << 24) + 16) == 2 and logits(sw=(1 << 24) + 16) == 2
    assert logits(h=p + 8) == 4 and logits(w=p + 4) == 4 and logits(z=p + 2) == 4 and logits(row=102) == 4 and logits(sh=264) == 4
    assert logits(dtype=0, row=102) == 4
    assert logits(space=None) == 5 and logits(space=p + 16) == 5 and logits(bytes=256) == 5

    def loss(**kw):
        a = dict(h=p, w=p, dtype=1, N=N, V=V, D=D, sh=D, sw=D, T=1.0, y=p, loss=p, lse=p, space=p, bytes=1 << 20)
        a.update(kw)
        return lib.svip_head_loss(a["h"], a["w"], a["dtype"], a["N"], a["V"], a["D"], a["sh"], a["sw"], a["T"], a["y"], a["loss"], a["lse"],
                                  a["space"], a["bytes"], None)

    for name in ("h", "w", "y", "loss", "lse"):
        assert loss(**{name: None}) == 1
    assert loss(dtype=9) == 3
    assert loss(N=0) == 2 and loss(N=-1) == 2 and loss(V=0) == 2 and loss(D=0) == 2 and loss(sh=D - 8) == 2 and loss(sw=(1 << 23) + 8) == 2
    assert loss(h=p + 2) == 4 and loss(sw=D + 4) == 4 and loss(D=D - 4) == 4 and loss(dtype=0, D=62) == 4
    assert loss(T=0.0) == 6 and loss(T=float("inf")) == 6 and loss(T=float("nan")) == 6 and loss(T=-1.0) == 6
    need = svip.head_workspace_bytes(svip.HEAD_LOSS, BF, N, V, D)
    assert loss(space=None) == 5 and loss(bytes=need - 1) == 5 and loss(space=p + 128) == 5

    def grad(**kw):
        a = dict(h=p, w=p, dtype=1, N=N, V=V, D=D, sh=D, sw=D, T=1.0, y=p, lse=p, g=p, dh=p, sdh=D, dw=p, sdw=D, space=p, bytes=1 << 20)
        a.update(kw)
        return lib.svip_head_loss_grad(a["h"], a["w"], a["dtype"], a["N"], a["V"], a["D"], a["sh"], a["sw"], a["T"], a["y"], a["lse"], a["g"],
                                       a["dh"], a["sdh"], a["dw"], a["sdw"], a["space"], a["bytes"], None)

    for name in ("h", "w", "y", "lse", "g"):
        assert grad(**{name: None}) == 1
    assert grad(dh=None, dw=None) == 1
    assert grad(dtype=4) == 3 and grad(V=0) == 2 and grad(sdh=D - 8) == 2 and grad(sdw=D - 8) == 2 and grad(dh=None, sdw=1 << 24) == 2
    assert grad(dh=p + 8) == 4 and grad(dw=p + 8) == 4 and grad(sdw=D + 4) == 4
    assert grad(T=0.0) == 6
    need = svip.head_workspace_bytes(svip.HEAD_LOSS_GRAD, BF, N, V, D)
    assert grad(space=None) == 5 and grad(bytes=need - 1) == 5
    del keep


def test_the_binding_refuses_before_it_calls():
    x = torch.zeros(4, 256, dtype=BF)
    q, s = torch.zeros(4, 256, dtype=torch.float8_e4m3fn), torch.zeros(4, 2, dtype=torch.float8_e8m0fnu)
    y, v = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    ws = torch.zeros(1 << 12, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device tensor"):
        svip.quantize_blocks(x, q_out=q, scale_out=s)
    with pytest.raises(svip.SvipError, match="block_rows"):
        svip.quantize_blocks(x, block_rows=32, q_out=q, scale_out=s)
    with pytest.raises(svip.SvipError, match="float32, bfloat16 or float16"):
        svip.quantize_blocks(x.double(), q_out=q, scale_out=s)
    with pytest.raises(ValueError, match="device tensor"):
        svip.head_logits(q, s, q, s, logits_out=torch.zeros(4, 4), workspace=ws)
    with pytest.raises(svip.SvipError, match="logits_out"):
        svip.head_logits(q, s, q, s, logits_out=torch.zeros(4, 4, dtype=torch.float64), workspace=ws)
    with pytest.raises(ValueError, match="device tensor"):
        svip.head_loss(x, x, y, loss_out=v, lse_out=v, workspace=ws)
    with pytest.raises(ValueError, match="device tensor"):
        svip.head_loss_grad(x, x, y, lse=v, grad_loss=v, grad_hidden_out=x, workspace=ws)
    with pytest.raises(ValueError, match="several devices"):
        svip.head_loss(x, x.to("meta"), y, loss_out=v, lse_out=v, workspace=ws)
