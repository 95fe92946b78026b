"""svip_sample's border of top-p and min-p where it is found by one workgroup to a row and marked by others: more than 1024 workgroups of tiles in a call."""
import math

import pytest
import torch

from test_sample_gpu import SETTINGS, gen, logits, reference, run

pytestmark = pytest.mark.gpu

F32, BF, F16 = torch.float32, torch.bfloat16, torch.float16
# beside the others' settings: top-p with min-p, either of which decides, top-p with a border next to the end of the steps, and rows that go to the sweeps
MORE = [(0.9, 0, 0.9, 0.02), (1.4, 0, 0.99, 1e-3), (0.8, 0, 0.6, 1e-5), (1.0, 0, 1.0 - 2.0 ** -20, 0.0), (1e-7, 0, 0.9, 0.1), (1.0, 0, 1.0, 1.0)]


def special_rows(z):
    """Rows without weight, of NaN, with +inf, flat ones with more tokens in a step than a list has, of few values, masked with the type's lowest value."""
    N, V = z.shape
    inf = math.inf
    z[3] = -inf
    z[4] = math.nan
    z[5, V // 3], z[5, V - 1] = inf, inf
    z[6] = 1.5
    z[7].copy_((z[7].float() * 2).round() / 2)
    z[8] = torch.finfo(z.dtype).min
    z[9, ::3] = math.nan
    z[10, : V // 2] = -inf
    z[11] = torch.finfo(z.dtype).min
    z[11, V // 2:V // 2 + 40] = torch.linspace(-3, 3, 40).to(z)
    z[12].copy_(z[12].float() * 0.01)
    z[13, 1:] = -inf


@pytest.mark.parametrize("dtype", [F32, BF, F16])
@pytest.mark.parametrize("N,V", [(1100, 1000), (600, 20003), (130, 128256)])
def test_border_of_many_rows(svip, dtype, N, V):
    """Against the definition, and against calls of fewer rows, whose tiles look for the border by themselves: the same bits, and so in a workspace that
    another call has left."""
    z = logits(N, V, dtype, seed=N + V, masked=0.0)
    special_rows(z)
    settings = SETTINGS + MORE
    # rows 3 .. 13 meet top-p and min-p alone and together in turn
    which = [settings[n % len(settings)] if not 3 <= n <= 13 else (MORE + [(0.7, 0, 0.9, 0.0), (1.2, 0, 1.0, 0.05)])[(n + V) % 8] for n in range(N)]
    T, k, p, m = zip(*which)
    u = torch.rand(N, generator=gen(V))
    token, prob, kept, flags = run(svip, z, u, T, k, p, m)
    assert flags == 0
    for first in range(0, N, 100):                               # (100 rows of 128256: 800 workgroups)
        a = slice(first, first + 100)
        t, pr, kp, _ = run(svip, z[a], u[a], T[a], k[a], p[a], m[a])
        assert (t == token[a]).all() and (pr == prob[a]).all() and (kp == kept[a]).all()
    near = checked = 0
    for n in list(range(40)) + list(range(40, N, max(1, N // 60))):
        f = lambda x: float(torch.tensor(x, dtype=F32))  # noqa: E731
        want = reference(z[n].double().cpu().numpy(), f(T[n]), k[n], f(p[n]), f(m[n]), float(u[n]))
        checked += 1
        if want[3]:
            near += 1
            continue
        assert token[n] == want[0] and kept[n] == want[2], (n, which[n], token[n], kept[n], want)
        assert abs(prob[n] - want[1]) <= (2.0 ** -23 + 1e-11) * want[1], (n, prob[n], want)
    assert near <= checked // 25


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_border_of_many_rows_in_a_used_workspace(svip, dtype):
    """One workspace for calls of several sizes and settings: what a call finds there of another changes nothing."""
    sizes = [(600, 20003), (1100, 1000), (40, 20003), (600, 20003)]
    need = max(svip.sample_workspace_bytes(dtype, *s) for s in sizes)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)
    ws[:256] = 0                                                 # (the flag word)
    for turn, (N, V) in enumerate(sizes):
        z = logits(N, V, dtype, seed=turn)
        settings = SETTINGS + MORE
        T, k, p, m = zip(*[settings[(n + 3 * turn) % len(settings)] for n in range(N)])
        u = torch.rand(N, generator=gen(turn))
        want = run(svip, z, u, T, k, p, m)
        dev = lambda x, t: torch.as_tensor(x, dtype=t).cuda()  # noqa: E731
        token, kept, prob = torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, device="cuda")
        svip.sample(z, u=dev(u, F32), temperature=dev(T, F32), top_k=dev(k, torch.int32), top_p=dev(p, F32), min_p=dev(m, F32), token_out=token,
                    prob_out=prob, kept_out=kept, workspace=ws)
        assert (token.cpu().numpy() == want[0]).all() and (prob.cpu().numpy() == want[1]).all() and (kept.cpu().numpy() == want[2]).all()
    assert svip.workspace_flags(ws) == 0


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_bad_rows_among_many(svip, dtype):
    N, V = 1100, 500
    z = logits(N, V, dtype, seed=9)
    T, k, p, m = ([x] * N for x in (0.7, 0, 0.9, 0.01))
    p[50], m[700], T[1099] = 0.0, 2.0, math.nan
    token, prob, kept, flags = run(svip, z, torch.rand(N, generator=gen(1)), T, k, p, m)
    bad = [50, 700, 1099]
    assert flags == svip.FLAG_BAD_SETTING
    assert (token[bad] == -1).all() and (kept[bad] == 0).all() and (prob[bad] == 0).all()
    assert (token >= 0).sum() == N - 3 and (kept >= 1).sum() == N - 3
