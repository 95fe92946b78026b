"""svip_sample's draw among tokens that weigh less than half a unit of the row's sums each, and on the borders of equal cells."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF, F16 = torch.float32, torch.bfloat16, torch.float16
TILE = 4096                                                      # logits to a tile


def gen(seed):
    return torch.Generator().manual_seed(seed)


def sample(svip, z, u, T=1.0, k=0, p=1.0):
    N, V = z.shape
    out = dict(token_out=torch.full((N,), -7, dtype=torch.int32, device="cuda"), prob_out=torch.empty(N, device="cuda"),
               kept_out=torch.empty(N, dtype=torch.int32, device="cuda"))
    full = lambda x, t: torch.full((N,), x, dtype=t, device="cuda")  # noqa: E731
    ws = svip.new_sample_workspace(z.dtype, N, V)
    svip.sample(z, u=u.cuda(), temperature=full(T, F32), top_k=full(k, torch.int32), top_p=full(p, F32), workspace=ws, **out)
    torch.cuda.synchronize()
    assert svip.workspace_flags(ws) == 0
    return out["token_out"].cpu().numpy(), out["prob_out"].cpu().double().numpy(), out["kept_out"].cpu().numpy()


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_tokens_of_less_than_a_unit(svip, dtype):
    """A token of weight 1 in front of 2^22 of 2^-41.1 = 0.46 units (a unit is 2^-40 at this size), and at the end of each tile seven that are masked
    with the type's lowest value.  The draw falls among the small ones, never on a mask, and where it should: at and the masses in front of a tile are off by
    up to half a unit for each tile, whose sums are rounded once, and the draw in the tile by another half, one for the rounding of at, one for the token's own
    cell."""
    V, tail, units = 1 << 22, -28.5, 2.0 ** 40
    N = 24
    z = torch.full((1, V), tail, dtype=dtype, device="cuda")
    z.view(-1, TILE)[:, -7:] = torch.finfo(dtype).min
    z[0, 0] = 0.0
    z = z.repeat(N, 1)
    u = 1.0 - torch.arange(1, N + 1) * 2.0 ** -24
    token, prob, kept = sample(svip, z, u)
    row = z[0].double().cpu().numpy()
    w = np.exp(row)
    run = np.cumsum(w)
    total = run[-1]
    assert (kept == V).all()
    assert (row[token] == tail).all(), (token, row[token])
    assert (np.abs(prob - w[token] / total) <= 2.0 ** -23 * w[token] / total).all()
    bound = (V // TILE + 0.5 + 1.0 + 1.0) / units + 1e-12 * total
    assert (np.abs(run[token] - u.double().numpy() * total) <= bound).all()
    assert len(set(token.tolist())) == N                         # 2^-24 apart: some 36 tiles


@pytest.mark.parametrize("dtype", [F32, BF])
def test_uniforms_on_the_cells_borders(svip, dtype):
    """Equal logits beside masks, tiles that hold different numbers of them, uniforms on the borders of cells, u V' = i: token i, or i - 1.  The sums in front of a
    tile and the total are off by up to half a unit for each of five tiles, u times the total by another: less than the 2^47 units of a cell."""
    V = 5 * TILE
    z = torch.zeros(V, dtype=dtype)
    z[torch.randperm(V, generator=gen(1))[:V - (1 << 13)]] = -math.inf
    live = torch.nonzero(z == 0.0)[:, 0].numpy()
    N = 64
    i = torch.randint(0, 1 << 13, (N,), generator=gen(2))
    i[0], i[1] = 0, (1 << 13) - 1
    token, prob, kept = sample(svip, z.repeat(N, 1).cuda(), i * 2.0 ** -13)
    assert ((token == live[i.numpy()]) | (token == live[np.maximum(i.numpy() - 1, 0)])).all() and (kept == 1 << 13).all() and (prob == 2.0 ** -13).all()
