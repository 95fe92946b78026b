"""The 4-bit head on the GPU against plain implementations in 64 bits: quantisation, rows read back, logits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF, F16 = torch.float32, torch.bfloat16, torch.float16
E4, E8, S8 = torch.float4_e2m1fn_x2, torch.float8_e4m3fn, torch.float8_e8m0fnu
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def up(n, to):
    return -(-n // to) * to


def reference(x):
    """Codes [rows, K] (0 .. 15) and scale codes [rows, K / 32] of x, value by value, on the CPU in 64 bits."""
    rows, cols = x.shape
    v = torch.zeros(rows, up(cols, 128), dtype=torch.float64)
    v[:, :cols] = x
    v = v.view(rows, -1, 32)
    finite = v.isfinite().all(2)
    amax = torch.where(finite, v.abs().amax(2), 0.0)
    e = torch.full(amax.shape, -127, dtype=torch.int64)
    for k in range(-127, 128):                                   # the least e with amax <= 6 * 2^e
        e = torch.where(amax > 6.0 * 2.0 ** k, k + 1, e)
    e = torch.where(amax == 0, 0, e)
    y = (v / torch.exp2(e.double())[:, :, None]).abs()
    code = torch.zeros_like(y, dtype=torch.int64)
    for c in range(1, 8):
        middle = (GRID[c - 1] + GRID[c]) / 2
        code = torch.where((y > middle) | ((y == middle) & (c % 2 == 0)), c, code)
    code += 8 * v.signbit()
    code = torch.where(finite[:, :, None], code, 0)
    return code.view(rows, -1), torch.where(finite, e + 127, 255)


def values(code, scale):
    """The numbers, in 64 bits."""
    v = GRID[code & 7] * torch.where(code > 7, -1.0, 1.0)
    s = torch.where(scale == 255, math.nan, torch.exp2(scale.double() - 127))
    return (v.view(code.shape[0], -1, 32) * s[:, :, None]).view(code.shape)


def unpack(q, cols=None):
    b = q.cpu().view(torch.uint8)
    return torch.stack([b & 15, b >> 4], 2).view(b.shape[0], -1).long()


def empty_mx(rows, K, fill=0xA5, extra=0):
    """Buffers of codes and scales (rows `extra` * 16 bytes longer than they need be), filled with a byte that nothing here writes everywhere."""
    q = torch.full((rows, K // 2 + 16 * extra), fill, dtype=torch.uint8, device="cuda")
    s = torch.full((rows, K // 32 + 16 * extra), fill, dtype=torch.uint8, device="cuda")
    return q, s


def quantized(svip, x, extra=0):
    rows, K = x.shape[0], up(x.shape[1], 128)
    q, s = empty_mx(rows, K, extra=extra)
    svip.quantize_mx(x, q_out=q[:, :K // 2].view(E4), scale_out=s[:, :K // 32].view(S8))
    torch.cuda.synchronize()
    assert (q[:, K // 2:] == 0xA5).all() and (s[:, K // 32:] == 0xA5).all()
    return q[:, :K // 2].view(E4), s[:, :K // 32].view(S8)


def check_quantized(x, q, s):
    code, scale = reference(x.cpu())
    assert torch.equal(s.cpu().view(torch.uint8).long(), scale)
    got = unpack(q)
    assert torch.equal(got & 7, code & 7)
    assert torch.equal((got > 7) & (got & 7 != 0), (code > 7) & (code & 7 != 0))      # (the sign of a zero may be either)


@pytest.mark.parametrize("dtype", [F32, BF, F16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (2, 32), (3, 33), (5, 127), (7, 128), (9, 129), (64, 1000), (130, 257), (1, 4096), (300, 2056), (17, 5120)])
def test_quantize(svip, dtype, rows, cols):
    x = (torch.randn(rows, cols, generator=gen(rows * 7 + cols)) * torch.exp(2.0 * torch.randn(rows, 1, generator=gen(3)))).to(dtype).cuda()
    q, s = quantized(svip, x, extra=rows % 3)
    check_quantized(x, q, s)


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_quantize_every_border(svip, dtype):
    """Values on and next to the middles between neighbours, at scales up and down the range."""
    base = torch.cat([GRID, (GRID[1:] + GRID[:-1]) / 2]).float()
    near = torch.cat([base, torch.nextafter(base, torch.tensor(9.0)), torch.nextafter(base, torch.tensor(-9.0))]) if dtype == F32 else base
    blocks = []
    for e in ((-140, -127, -126, -20, 0, 1, 60, 125) if dtype != F16 else (-20, -14, 0, 12)):
        for part in near.split(15):
            for most in (6.0, 3.1, 5.0):
                row = torch.zeros(32)
                row[:len(part)] = part.clamp(max=most)
                row[15:15 + len(part)] = -part.clamp(max=most)
                row[31] = most
                blocks.append(torch.ldexp(row.double(), torch.tensor(e)).to(dtype))
    n = up(len(blocks), 4)
    x = torch.zeros(n, 32, dtype=dtype)
    x[:len(blocks)] = torch.stack(blocks)
    x = x.view(n // 4, 128).cuda()
    q, s = quantized(svip, x)
    check_quantized(x, q, s)


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_quantize_not_finite_and_largest(svip, dtype):
    x = torch.randn(6, 256, generator=gen(5)).to(dtype)
    x[0, 3], x[1, 40], x[2, 255] = math.nan, math.inf, -math.inf
    x[3, :] = 0
    x[4, 64:96] = torch.finfo(dtype).max
    x[5, 0:32] = torch.finfo(dtype).tiny / 4
    x = x.cuda()
    q, s = quantized(svip, x)
    check_quantized(x, q, s)
    assert [int(s.view(torch.uint8)[r, c]) for r, c in ((0, 0), (1, 1), (2, 7))] == [255] * 3
    out = torch.empty(6, 256, dtype=dtype, device="cuda")
    svip.mx_rows(q, s, out=out)
    assert out[0, :32].isnan().all() and out[1, 32:64].isnan().all() and out[2, 224:].isnan().all() and out.isnan().sum() == 96


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_quantize_any_stride_and_alignment(svip, dtype):
    whole = torch.randn(40, 700, generator=gen(11)).to(dtype).cuda()
    for x in (whole[:, 1:334], whole[3::2, 5:5 + 128], whole[:, 699:], whole.as_strided((9, 256), (259, 1), 7)):
        q, s = quantized(svip, x, extra=1)
        check_quantized(x, q, s)
    with pytest.raises(svip.SvipError):                          # rows that overlap
        quantized(svip, whole.as_strided((9, 256), (3, 1), 7))


@pytest.mark.parametrize("dtype", [F32, BF, F16])
@pytest.mark.parametrize("rows,cols,n", [(1, 1, 1), (3, 33, 5), (50, 128, 64), (1000, 1000, 333), (500, 4096, 17), (64, 4097, 64)])
def test_rows(svip, dtype, rows, cols, n):
    x = (torch.randn(rows, cols, generator=gen(cols)) * torch.exp(1.5 * torch.randn(rows, 1, generator=gen(8)))).bfloat16().cuda()
    q, s = quantized(svip, x, extra=1)
    want = values(unpack(q), s.cpu().view(torch.uint8).long())[:, :cols]
    ids = torch.randint(0, rows, (n,), generator=gen(n), dtype=torch.int32)
    ids[::5] = -1
    ids[min(n - 1, 3)] = rows - 1
    ids[n // 2] = rows if n > 4 else ids[n // 2]
    whole = torch.full((n + 2, cols + 3), 77.0, dtype=dtype, device="cuda")
    out = whole[1:n + 1, 1:cols + 1]                              # rows at any alignment, and nothing around them written
    svip.mx_rows(q, s, ids=ids.cuda(), out=out)
    ref = want[ids.clamp(0, rows - 1).long()].to(dtype)           # (a value has two significant bits: the cast rounds once)
    ref[ids < 0] = 0
    ref[ids >= rows] = math.nan
    assert torch.equal(out.cpu().nan_to_num(nan=123.0), ref.nan_to_num(nan=123.0))
    whole[1:n + 1, 1:cols + 1] = 77.0
    assert (whole == 77.0).all()
    m = min(n, rows)
    first = torch.empty(m, cols, dtype=dtype, device="cuda")
    svip.mx_rows(q, s, out=first)
    assert torch.equal(first.cpu(), want[:m].to(dtype))


def test_rows_scales_at_the_ends(svip):
    """Every scale, with every code, in every type."""
    code = torch.arange(16).repeat(8).view(1, 128).repeat(256, 1)
    q = (code[:, ::2] | code[:, 1::2] << 4).to(torch.uint8).cuda().view(E4)
    s = torch.arange(256)[:, None].repeat(1, 4)
    for dtype in (F32, BF, F16):
        out = torch.empty(256, 128, dtype=dtype, device="cuda")
        svip.mx_rows(q, s.to(torch.uint8).cuda().view(S8), out=out)
        want = values(code, s).to(F32).to(dtype)
        assert torch.equal(out.cpu().nan_to_num(nan=0.25, posinf=3e4, neginf=-3e4), want.nan_to_num(nan=0.25, posinf=3e4, neginf=-3e4)), dtype


# ---- logits --------------------------------------------------------------------------------------------------------------------------------

def matrix4(rows, K, seed, spread=2, extra=0):
    """Random codes and scales between 2^-spread and 2^spread, in rows longer than need be, with the values in 64 bits."""
    g = gen(seed)
    code = torch.randint(0, 16, (rows, K), generator=g)
    scale = 127 + torch.randint(-spread, spread + 1, (rows, K // 32), generator=g)
    q, s = empty_mx(rows, K, extra=extra)
    q[:, :K // 2] = (code[:, ::2] | code[:, 1::2] << 4).to(torch.uint8).cuda()
    s[:, :K // 32] = scale.to(torch.uint8).cuda()
    return q[:, :K // 2].view(E4), s[:, :K // 32].view(S8), values(code, scale)


def matrix8(rows, K, seed, spread=2, extra=0):
    g = gen(seed)
    code = torch.randn(rows, K, generator=g).mul_(40).clamp_(-448, 448).to(E8)
    scale = 127 + torch.randint(-spread, spread + 1, (rows, K // 128), generator=g)
    q = torch.full((rows, K + 16 * extra), 0x7F, dtype=torch.uint8, device="cuda")
    s = torch.full((rows, K // 128 + 3 * extra), 255, dtype=torch.uint8, device="cuda")
    q[:, :K] = code.view(torch.uint8).cuda()
    s[:, :K // 128] = scale.to(torch.uint8).cuda()
    v = code.double() * torch.exp2(scale.double() - 127).repeat_interleave(128, 1)
    return q[:, :K].view(E8), s[:, :K // 128].view(S8), v


def logits(svip, h, w, dtype, V, N, stream=None, extra=0):
    out = torch.full((N + 1, up(V, 8) + 8 * extra), 55.0, dtype=dtype, device="cuda")
    K = 2 * w[0].shape[1]
    ws = svip.new_head_workspace(svip.HEAD_LOGITS_MX, dtype, N, V, K)
    svip.head_logits_mx(h[0], h[1], w[0], w[1], logits_out=out[:N, :V], workspace=ws)
    torch.cuda.synchronize()
    assert (out[N] == 55).all() and (out[:N, V:] == 55).all()
    return out[:N, :V].cpu().double()


def check_logits(got, h, w, K, dtype, bits):
    """Sums of K products: in fp32 each of the K / 128 additions of an instruction's sum, and the up to 128 within it, round by half a step of at
    most the sum of magnitudes; hidden states in 8 bits: up to 7 of 8 products lose what lies below 2^-13 of the largest.  Then one rounding."""
    exact, size = h @ w.T, h.abs() @ w.abs().T
    bound = (K / 128 + 128) * 2.0 ** -24 * size
    if bits == 8:
        bound = bound + 7 * 2.0 ** -13 * size
    step = torch.finfo(dtype).eps / 2
    bound = bound + step * (exact.abs() + bound) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    off = (got - exact).abs()
    assert (off <= bound).all(), float((off / bound).max())


SIZES = [(1, 1, 128), (1, 7, 256), (2, 64, 384), (3, 65, 128), (16, 129, 640), (31, 500, 256), (32, 513, 1152), (33, 300, 256), (64, 1000, 512), (65, 1000, 384),
         (127, 260, 256), (129, 257, 896), (300, 777, 256), (1, 3000, 4096), (5, 70, 8192), (64, 129, 4224), (256, 2049, 128), (513, 4100, 256)]


@pytest.mark.parametrize("bits,dtype", [(4, F32), (4, BF), (4, F16), (8, BF), (8, F16)])
@pytest.mark.parametrize("N,V,K", SIZES)
def test_logits(svip, bits, dtype, N, V, K):
    w = matrix4(V, K, seed=V + K, extra=V % 2)
    h = (matrix4 if bits == 4 else matrix8)(N, K, seed=N + K, spread=3, extra=N % 2)
    if dtype == F16:                                             # sums within the type's range
        shift = 8
        h = (h[0], (h[1].view(torch.uint8) - shift).view(S8) if h[1].is_contiguous() else (h[1].contiguous().view(torch.uint8) - shift).view(S8), h[2] * 2.0 ** -shift)
    got = logits(svip, h, w, dtype, V, N, extra=K % 3)
    check_logits(got, h[2], w[2], K, dtype, bits)


@pytest.mark.parametrize("N,V", [(70, 66000), (1, 128256), (300, 33000), (1088, 16500)])
def test_logits_of_many_tiles(svip, N, V):
    """Grids of more tiles than the chip holds, on a small K: every tile in its place."""
    K = 128
    w, h = matrix4(V, K, seed=1), matrix4(N, K, seed=2)
    out = torch.empty(N, up(V, 8), dtype=BF, device="cuda")[:, :V]
    svip.head_logits_mx(h[0], h[1], w[0], w[1], logits_out=out, workspace=svip.new_head_workspace(svip.HEAD_LOGITS_MX, BF, N, V, K))
    exact = h[2].cuda() @ w[2].cuda().T
    size = h[2].abs().cuda() @ w[2].abs().cuda().T
    assert ((out.double() - exact).abs() <= 2.0 ** -8 * exact.abs() + 2.0 ** -16 * size).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("N,V,K", [(200, 33000, 1408), (20, 33000, 4736), (20, 33000, 128), (64, 33000, 640), (300, 33000, 4480), (66, 1003, 5248), (257, 2001, 2176)])
def test_logits_of_a_vocabulary(svip, bits, N, V, K):
    """The tiles of large vocabularies over several groups of scales, and ends inside of a step."""
    w, h = matrix4(V, K, seed=V + K), (matrix4 if bits == 4 else matrix8)(N, K, seed=N + K, spread=3)
    got = logits(svip, h, w, BF, V, N)
    check_logits(got, h[2], w[2], K, BF, bits)


@pytest.mark.parametrize("bits", [4, 8])
def test_logits_scales_at_the_ends(svip, bits):
    """Scales from 2^-127 up to 2^127 whose product is about one, and the NaN of e8m0 on either side."""
    N, V, K = 40, 200, 256
    w, h = matrix4(V, K, seed=3, spread=0), (matrix4 if bits == 4 else matrix8)(N, K, seed=4, spread=0)
    # rows of hidden states by 2^d, tokens by 2^-d in turn
    d = torch.tensor([-127, -100, -20, 0, 20, 100, 127])
    hd, wd = d[torch.arange(N) % 7], -d[torch.arange(V) % 7]
    hs = (127 + hd)[:, None].repeat(1, h[1].shape[1])
    ws = (127 + wd)[:, None].repeat(1, K // 32)
    hs[5, 1], ws[9, 3] = 255, 255
    h8, w8 = hs.to(torch.uint8).cuda().view(S8), ws.to(torch.uint8).cuda().view(S8)
    got = logits(svip, (h[0], h8), (w[0], w8), BF, V, N)
    hv, wv = h[2] * torch.exp2(hd.double())[:, None], w[2] * torch.exp2(wd.double())[:, None]
    nan = torch.zeros(N, V, dtype=torch.bool)
    nan[5], nan[:, 9] = True, True
    assert torch.equal(got.isnan(), nan)
    near = (hd[:, None] + wd[None, :] == 0) & ~nan
    size = hv.abs() @ wv.abs().T
    off = (got - hv @ wv.T).abs()
    bound = 2.0 ** -8 * (hv @ wv.T).abs() + (2.0 ** -16 + (7 * 2.0 ** -13 if bits == 8 else 0)) * size
    assert (off[near] <= bound[near]).all()


def test_logits_refuse_wrong_shapes(svip):
    w, h, h8 = matrix4(20, 256, 1), matrix4(4, 256, 2), matrix8(4, 256, 3)
    out, ws = torch.empty(4, 24, dtype=BF, device="cuda")[:, :20], svip.new_head_workspace(svip.HEAD_LOGITS_MX, BF, 4, 20, 256)
    ok = dict(logits_out=out, workspace=ws)
    svip.head_logits_mx(h[0], h[1], w[0], w[1], **ok)
    for args in ((h[0][:, :64], h[1], w[0], w[1]), (h[0], h[1][:, :4], w[0], w[1]), (h[0], h[1], w[0][:, :64], w[1]), (h[0], h[1], w[0], w[1][:19]),
                 (h8[0], h[1], w[0], w[1]), (h[0], h8[1], w[0], w[1]), (h8[0][:, :128], h8[1], w[0], w[1])):
        with pytest.raises(ValueError):
            svip.head_logits_mx(*args, **ok)
    with pytest.raises(ValueError):
        svip.head_logits_mx(h[0], h[1], w[0], w[1], logits_out=out[:3], workspace=ws)
    with pytest.raises(svip.SvipError):
        svip.head_logits_mx(h8[0], h8[1], w[0], w[1], logits_out=torch.empty(4, 20, device="cuda"), workspace=ws)
    with pytest.raises(svip.SvipError):
        svip.head_logits_mx(h[0], h[1], w[0], w[1], logits_out=out, workspace=ws[:256])
