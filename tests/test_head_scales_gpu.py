"""The scales of head_logits over their whole range, e8m0 from 2^-127 to 2^127 and NaN: products of powers of two, which have one right result in every type."""
import pytest
import torch

from test_head_gpu import TYPES, eight_bits, gen

pytestmark = pytest.mark.gpu
E8 = torch.float8_e8m0fnu


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("rows", [[0, 1, 100, 127, 200, 254, 255], list(range(40)), list(range(200, 256)), list(range(256))])
def test_every_pair_of_scales(svip, rows, out):
    """Codes of 1, so that a logit is 128 times the two scales: numbers, subnormal numbers, 0, infinity or NaN."""
    K, V, N = 128, 256 * 128, len(rows)
    ones = torch.ones(V, K, device="cuda").to(torch.float8_e4m3fn)
    a, b = torch.tensor(rows, device="cuda"), torch.arange(256, device="cuda")
    z = torch.zeros(N, V, dtype=TYPES[out], device="cuda")
    svip.head_logits(ones[:N], a.to(torch.uint8)[:, None].contiguous().view(E8), ones, b.to(torch.uint8)[:, None].contiguous().view(E8), logits_out=z,
                     workspace=svip.new_head_workspace(svip.HEAD_LOGITS, z.dtype, N, V, K))
    want = 2.0 ** (7 + a[:, None].double() + b[None, :].double() - 254)
    want[(a == 255)[:, None] | (b == 255)[None, :]] = float("nan")
    want = want.to(z.dtype).repeat_interleave(128, 1)
    assert torch.equal(z.isnan(), want.isnan()) and torch.equal(z.nan_to_num(nan=0.0, posinf=9.0), want.nan_to_num(nan=0.0, posinf=9.0))


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("N,V,K", [(3, 301, 4096), (40, 1999, 2304), (65, 515, 640), (300, 4099, 8960)])
def test_a_scale_of_nan_reaches_its_row_or_its_tokens_alone(svip, N, V, K, out):
    """In any block of K: of a row of hidden states, and of 128 tokens of the weight."""
    g, t = gen(N + V), TYPES[out]
    hq, hs = eight_bits(N, K, 1, g, 0)
    wq, ws = eight_bits(V, K, 128, g, 0)
    hs, ws = (s.contiguous().view(torch.uint8) for s in (hs, ws))
    space = svip.new_head_workspace(svip.HEAD_LOGITS, t, N, V, K)
    logits = []
    for bad in (False, True):
        if bad:
            hs[N - 1, K // 128 - 1] = 255
            ws[1, 0] = 255
        z = torch.zeros(N, -(-V // 8) * 8, dtype=t, device="cuda")
        svip.head_logits(hq, hs.view(E8), wq, ws.view(E8), logits_out=z[:, :V], workspace=space)
        logits.append(z[:, :V])
    nan = torch.zeros(N, V, dtype=torch.bool, device="cuda")
    nan[N - 1], nan[:, 128:256] = True, True
    assert logits[1][nan].isnan().all() and torch.equal(logits[1][~nan], logits[0][~nan])
