"""svip_head_logits_mx by its largest tiles (256 x 256 with hidden states in 4 bits, 256 x 128 in 8) in several columns of tiles, every type of result."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF, F16 = torch.float32, torch.bfloat16, torch.float16
E4, E8, S8 = torch.float4_e2m1fn_x2, torch.float8_e4m3fn, torch.float8_e8m0fnu


def matrix(rows, K, bits, seed, shift=0):
    """Random codes and scales between 2^-2 and 2^2 (times 2^shift), and the numbers that they stand for, in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    block = 32 if bits == 4 else 128
    scale = 127 + shift + torch.randint(-2, 3, (rows, K // block), device="cuda", generator=g)
    if bits == 4:
        code = torch.randint(0, 16, (rows, K), device="cuda", generator=g, dtype=torch.uint8)
        q = (code[:, ::2] | code[:, 1::2] << 4).view(E4)
        v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda", dtype=torch.float64)[(code & 7).long()]
        v = torch.where(code > 7, -v, v)
    else:
        q = torch.randn(rows, K, device="cuda", generator=g).mul_(40).clamp_(-448, 448).to(E8)
        v = q.double()
    v = v.view(rows, -1, block) * torch.exp2(scale.double() - 127)[:, :, None]
    return q, scale.to(torch.uint8).view(S8), v.view(rows, K)


# 300 rows: 2 columns of tiles (8 bits: 3), the last not full; 17.5 steps of 256 values, in 4 bits five groups of scales.  1088: 5 columns (9), of
# which four go side by side.  Either V ends inside a tile.
@pytest.mark.parametrize("bits,dtype", [(4, F32), (4, BF), (4, F16), (8, BF), (8, F16)])
@pytest.mark.parametrize("N,V,K", [(300, 32600, 4480), (1088, 50200, 640)])
def test_large_tiles_in_several_columns(svip, N, V, K, bits, dtype):
    hq, hs, hv = matrix(N, K, bits, seed=N, shift=-10 if dtype == F16 else 0)        # (sums within fp16's range)
    wq, ws, wv = matrix(V, K, 4, seed=V)
    row = -(-V // 8) * 8 + 8
    out = torch.full((N + 1, row), 55.0, dtype=dtype, device="cuda")
    space = svip.new_head_workspace(svip.HEAD_LOGITS_MX, dtype, N, V, K)
    for turn in range(2):                                        # and the same bits again
        svip.head_logits_mx(hq, hs, wq, ws, logits_out=out[:N, :V], workspace=space)
        if turn == 0:
            first = out.clone()
    assert torch.equal(out, first) and (out[N] == 55).all() and (out[:, V:] == 55).all()
    got = out[:N, :V].double()
    for a in range(0, V, 8192):
        w = wv[a:a + 8192]
        exact, size = hv @ w.T, hv.abs() @ w.abs().T
        # each of the K / 128 additions to an instruction's sum, and the up to 128 within it, round by half a step of at most the sum of
        # magnitudes; in 8 bits up to 7 of 8 products lose what lies below 2^-13 of the largest; then one rounding
        bound = (K / 128 + 128) * 2.0 ** -24 * size
        if bits == 8:
            bound += 7 * 2.0 ** -13 * size
        bound += torch.finfo(dtype).eps / 2 * (exact.abs() + bound) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
        off = (got[:, a:a + 8192] - exact).abs()
        assert (off <= bound).all(), (a, float((off / bound).max()))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("N,V,K", [(3, 5003, 4096), (20, 40000, 2048), (64, 128256, 2048), (100, 5003, 4096), (100, 60000, 1152), (325, 50257, 1152)])
def test_the_same_bits_again(svip, N, V, K, bits):
    """Each kind of tile, whole and with K in splits, over again with other work between."""
    hq, hs, _ = matrix(N, K, bits, seed=1)
    wq, ws, _ = matrix(V, K, 4, seed=2)
    out = torch.empty(N, -(-V // 8) * 8, dtype=BF, device="cuda")[:, :V]
    space = svip.new_head_workspace(svip.HEAD_LOGITS_MX, BF, N, V, K)
    first = None
    for turn in range(6):
        out.fill_(float(turn))
        space[512:].fill_(0xFF)                                  # (behind the flag word: sums of an earlier call)
        svip.head_logits_mx(hq, hs, wq, ws, logits_out=out, workspace=space)
        first = out.clone() if first is None else first
        assert torch.equal(out.view(torch.int16), first.view(torch.int16))
