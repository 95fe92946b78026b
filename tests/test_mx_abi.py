"""The 4-bit head's calls and the sampler without a GPU: what they refuse on the host, before anything is enqueued, and their workspace sizes."""
import ctypes

import pytest
import torch

import paper_2411_18462_amd as svip

F32, BF, F16 = torch.float32, torch.bfloat16, torch.float16
E4, E8, S8 = torch.float4_e2m1fn_x2, torch.float8_e4m3fn, torch.float8_e8m0fnu


def _pointer():
    buf = ctypes.create_string_buffer(1 << 12)
    return buf, (ctypes.addressof(buf) + 255) & ~255          # a fake, aligned "device" pointer, never dereferenced


def test_workspace_bytes():
    f = svip.head_workspace_bytes
    for N, V, K in ((1, 1, 128), (1, 32000, 1024), (64, 128256, 2048), (65, 32000, 4096), (1088, 151936, 5120), (1 << 20, 1 << 22, 128)):
        assert f(svip.HEAD_LOGITS_MX, BF, N, V, K) > 0 and f(svip.HEAD_LOGITS_MX, BF, N, V, K) % 256 == 0
    for bad in ((4, BF, 8, 100, 128), (3, torch.int8, 8, 100, 128), (3, BF, 0, 100, 128), (3, BF, 8, 0, 128), (3, BF, 8, 100, 0), (3, BF, 8, (1 << 22) + 1, 128)):
        assert f(*bad) == 0
    g = svip.sample_workspace_bytes
    for dtype in (F32, BF, F16):
        for N, V in ((1, 1), (64, 128256), (1088, 151936), (1 << 20, 7), (1, 1 << 22)):
            assert g(dtype, N, V) > 0 and g(dtype, N, V) % 256 == 0
    for bad in ((torch.float64, 8, 100), (BF, 0, 100), (BF, 8, 0), (BF, (1 << 20) + 1, 100), (BF, 8, (1 << 22) + 1)):
        assert g(*bad) == 0
        with pytest.raises(svip.SvipError):
            svip.new_sample_workspace(*bad)


def test_host_checks_of_quantize_and_rows():
    lib = svip.load()
    keep, p = _pointer()

    def quantize(**kw):
        a = dict(x=p, dtype=1, rows=5, cols=200, stride=208, q=p, qs=128, s=p, ss=8)
        a.update(kw)
        return lib.svip_quantize_mx(a["x"], a["dtype"], a["rows"], a["cols"], a["stride"], a["q"], a["qs"], a["s"], a["ss"], None)

    assert quantize(x=None) == 1 and quantize(q=None) == 1 and quantize(s=None) == 1
    assert quantize(dtype=3) == 3 and quantize(dtype=-1) == 3
    assert quantize(rows=0) == 2 and quantize(cols=0) == 2 and quantize(stride=199) == 2 and quantize(qs=112) == 2 and quantize(ss=4) == 2
    assert quantize(rows=(1 << 22) + 1) == 2 and quantize(cols=(1 << 17) + 1, stride=1 << 18, qs=1 << 18, ss=1 << 13) == 2
    assert quantize(rows=1 << 22, cols=4096, stride=4096, qs=2048, ss=128) == 2 and quantize(qs=(1 << 24) + 16) == 2
    assert quantize(x=p + 1) == 4 and quantize(x=p + 2, dtype=0) == 4 and quantize(q=p + 8) == 4 and quantize(qs=136) == 4
    assert quantize(s=p + 2) == 4 and quantize(ss=10) == 4

    def rows(**kw):
        a = dict(q=p, s=p, rows=50, cols=200, qs=128, ss=8, ids=p, n=5, out=p, dtype=1, so=200)
        a.update(kw)
        return lib.svip_mx_rows(a["q"], a["s"], a["rows"], a["cols"], a["qs"], a["ss"], a["ids"], a["n"], a["out"], a["dtype"], a["so"], None)

    assert rows(q=None) == 1 and rows(s=None) == 1 and rows(out=None) == 1
    assert rows(dtype=7) == 3
    assert rows(rows=0) == 2 and rows(cols=0) == 2 and rows(n=0) == 2 and rows(so=199) == 2 and rows(qs=112) == 2 and rows(ss=4) == 2
    assert rows(ids=None, n=51) == 2 and rows(n=(1 << 22) + 1) == 2 and rows(n=1 << 22, cols=8192, so=8192, qs=4096, ss=256) == 2
    assert rows(out=p + 1) == 4 and rows(out=p + 2, dtype=0) == 4 and rows(q=p + 4) == 4 and rows(s=p + 1) == 4


def test_host_checks_of_logits():
    lib = svip.load()
    keep, p = _pointer()

    def logits(**kw):
        a = dict(h=p, hs=p, bits=4, w=p, ws=p, N=4, V=100, K=256, sh=128, shs=8, sw=128, sws=8, z=p, dtype=1, row=104, space=p, bytes=1 << 12)
        a.update(kw)
        return lib.svip_head_logits_mx(a["h"], a["hs"], a["bits"], a["w"], a["ws"], a["N"], a["V"], a["K"], a["sh"], a["shs"], a["sw"], a["sws"],
                                        a["z"], a["dtype"], a["row"], a["space"], a["bytes"], None)

    for name in ("h", "hs", "w", "ws", "z"):
        assert logits(**{name: None}) == 1
    assert logits(dtype=5) == 3 and logits(bits=8, dtype=0, sh=256, row=104) == 3
    assert logits(bits=6) == 6 and logits(bits=0) == 6
    assert logits(N=0) == 2 and logits(V=0) == 2 and logits(K=0) == 2 and logits(K=192) == 2 and logits(row=96) == 2
    assert logits(sh=112) == 2 and logits(sw=112) == 2 and logits(shs=4) == 2 and logits(sws=4) == 2 and logits(sw=(1 << 24) + 16) == 2
    assert logits(bits=8, sh=240, shs=2) == 2 and logits(bits=8, sh=256, shs=1) == 2
    assert logits(h=p + 8) == 4 and logits(w=p + 4) == 4 and logits(z=p + 2) == 4 and logits(row=102) == 4 and logits(sh=136) == 4
    assert logits(hs=p + 2) == 4 and logits(ws=p + 1) == 4 and logits(shs=10) == 4 and logits(sws=9) == 4 and logits(bits=8, sh=264, shs=2) == 4
    assert logits(space=None) == 5 and logits(space=p + 16) == 5 and logits(bytes=256) == 5


def test_host_checks_of_sample():
    lib = svip.load()
    keep, p = _pointer()

    def sample(**kw):
        a = dict(z=p, dtype=1, N=4, V=100, row=104, T=p, k=p, p=p, m=p, u=p, token=p, prob=p, kept=p, space=p, bytes=1 << 12)
        a.update(kw)
        return lib.svip_sample(a["z"], a["dtype"], a["N"], a["V"], a["row"], a["T"], a["k"], a["p"], a["m"], a["u"], a["token"], a["prob"], a["kept"],
                               a["space"], a["bytes"], None)

    assert sample(z=None) == 1 and sample(u=None) == 1 and sample(token=None) == 1
    assert sample(dtype=4) == 3
    assert sample(N=0) == 2 and sample(V=0) == 2 and sample(row=96) == 2 and sample(N=(1 << 20) + 1) == 2 and sample(V=(1 << 22) + 1, row=1 << 23) == 2
    assert sample(z=p + 8) == 4 and sample(row=102) == 4 and sample(dtype=0, row=102) == 4
    need = svip.sample_workspace_bytes(BF, 4, 100)
    assert sample(space=None) == 5 and sample(space=p + 128) == 5 and sample(bytes=need - 1) == 5


def test_python_refuses_host_tensors_and_wrong_types():
    x = torch.zeros(2, 128)
    q, s = torch.zeros(2, 64, dtype=torch.uint8).view(E4), torch.zeros(2, 4, dtype=torch.uint8).view(S8)
    with pytest.raises(ValueError, match="device tensor"):
        svip.quantize_mx(x, q_out=q, scale_out=s)
    with pytest.raises(svip.SvipError):
        svip.quantize_mx(x.double(), q_out=q, scale_out=s)
    with pytest.raises(ValueError, match="device tensor"):
        svip.mx_rows(q, s, out=x)
    with pytest.raises(svip.SvipError):
        svip.mx_rows(q, s, out=x.int())
    space, z = torch.zeros(512, dtype=torch.uint8), torch.zeros(2, 2)
    with pytest.raises(ValueError, match="device tensor"):
        svip.head_logits_mx(q, s, q, s, logits_out=z, workspace=space)
    with pytest.raises(svip.SvipError):
        svip.head_logits_mx(x, s, q, s, logits_out=z, workspace=space)
    with pytest.raises(svip.SvipError):                              # 8-bit hidden states have 16-bit logits
        svip.head_logits_mx(x.to(E8), s, q, s, logits_out=z, workspace=space)
    with pytest.raises(ValueError, match="device tensor"):
        svip.sample(z, u=z[0], token_out=z[0].int(), workspace=space)
    with pytest.raises(svip.SvipError):
        svip.sample(z.double(), u=z[0], token_out=z[0].int(), workspace=space)
