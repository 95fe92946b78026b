"""svip_sample against the definition in 64 bits, row by row, and the 4-bit head, the sampler and the lookup as a drafting loop uses them."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF, F16 = torch.float32, torch.bfloat16, torch.float16


def gen(seed):
    return torch.Generator().manual_seed(seed)


def reference(z, T, k, p, m, u):
    """(token, prob, kept, near) of one row of 64-bit numbers.  near: a decision lies within rounding of its border.  Masses are sums of up to V weights, each
    off by up to half a unit 2^-S of the largest weight, 1, and by 1e-12 of itself (what the series leaves out, 2.3e-13, and the rounding of
    exponents up to a thousand); exponents, which min_p goes by, by 1e-13 of themselves."""
    V = len(z)
    half_units = V * 2.0 ** -(min(51, 62 - math.ceil(math.log2(V))) + 1)
    z = np.where(np.isnan(z), -np.inf, z)
    top = z.max()
    if top == -np.inf:
        return -1, 0.0, 0, False
    if T == 0:
        return int(z.argmax()), 1.0, 1, False
    with np.errstate(invalid="ignore", over="ignore"):
        x = np.where(z == top, 0.0, (z - top) / T)
    w = np.exp(x)
    keep = z > -np.inf
    near = False
    if 0 < k < V:
        keep &= z >= np.sort(z)[::-1][k - 1]
    if p < 1:
        values, at = np.unique(-z[keep], return_inverse=True)
        mass = np.cumsum(np.bincount(at, weights=w[keep]))
        near |= bool((np.abs(mass - p * mass[-1]) < half_units + 1e-12 * mass[-1]).any())
        keep &= z >= -values[int((mass < p * mass[-1]).sum())]
    if m > 0:
        near |= bool((np.abs(x - math.log(m)) < 1e-13 * (1 - math.log(m)))[x < 0].any())
        keep &= x >= math.log(m)
    kept = np.where(keep, w, 0.0)
    run = np.cumsum(kept)
    near |= bool((np.abs(run - u * run[-1]) < half_units + 1e-12 * run[-1])[:-1][kept[1:] > 0].any())
    token = int((run <= u * run[-1]).sum())
    return token, kept[token] / run[-1], int(keep.sum()), near


def run(svip, z, u, T=None, k=None, p=None, m=None, prob=True, kept=True):
    N, V = z.shape
    dev = lambda x, t: None if x is None else torch.as_tensor(x, dtype=t).cuda()  # noqa: E731
    token = torch.full((N,), -7, dtype=torch.int32, device="cuda")
    pr = torch.full((N,), -7.0, device="cuda") if prob else None
    kp = torch.full((N,), -7, dtype=torch.int32, device="cuda") if kept else None
    ws = svip.new_sample_workspace(z.dtype, N, V)
    svip.sample(z, u=dev(u, F32), temperature=dev(T, F32), top_k=dev(k, torch.int32), top_p=dev(p, F32), min_p=dev(m, F32), token_out=token,
                prob_out=pr, kept_out=kp, workspace=ws)
    torch.cuda.synchronize()
    return token.cpu().numpy(), pr.cpu().numpy() if prob else None, kp.cpu().numpy() if kept else None, svip.workspace_flags(ws)


def rows_of(N, V, dtype, fill=60000.0, pad=8):
    """[N, V] in rows that go on behind V with a number that would win every draw."""
    row = -(-V // 8) * 8 + pad
    return torch.full((N, row), fill, dtype=dtype, device="cuda")[:, :V]


def check(svip, z, u, T=None, k=None, p=None, m=None):
    N, V = z.shape
    token, prob, kept, flags = run(svip, z, u, T, k, p, m)
    assert flags == 0
    f = lambda x, other: np.full(N, other) if x is None else np.asarray(torch.as_tensor(x, dtype=F32 if other != 0 or x is m else torch.int32))  # noqa: E731
    T, k, p, m = f(T, 1.0), (np.zeros(N, int) if k is None else np.asarray(k)), f(p, 1.0), (np.zeros(N) if m is None else np.asarray(torch.as_tensor(m, dtype=F32)))
    zz, uu = z.cpu().double().numpy(), np.asarray(torch.as_tensor(u, dtype=F32)).astype(np.float64)
    near = 0
    for n in range(N):
        want = reference(zz[n], float(T[n]), int(k[n]), float(p[n]), float(m[n]), float(uu[n]))
        if want[3]:
            near += 1
            continue
        assert token[n] == want[0] and kept[n] == want[2], (n, token[n], kept[n], want)
        assert abs(prob[n] - want[1]) <= (2.0 ** -23 + 1e-11) * want[1], (n, prob[n], want)        # one rounding to fp32, taken double
    assert near <= max(1, N // 50)


def logits(N, V, dtype, seed, masked=0.0):
    g = gen(seed)
    x = torch.randn(N, V, generator=g) * (0.5 * 8.0 ** torch.rand(N, 1, generator=g))
    sure = torch.rand(N, generator=g) < 0.5
    at = torch.randint(0, V, (N,), generator=g)
    x[torch.arange(N), at] += torch.where(sure, 8 + 6 * torch.rand(N, generator=g), 0.0)
    if masked:
        x[torch.rand(N, V, generator=g) < masked] = -math.inf
    z = rows_of(N, V, dtype)
    z.copy_(x)
    return z


SIZES = [(1, 1), (2, 2), (3, 7), (2, 8), (4, 9), (5, 63), (5, 64), (5, 65), (7, 255), (9, 1000), (6, 4096), (6, 4097), (6, 8191), (5, 16385), (8, 32000), (3, 50257), (4, 128256),
         (2, 151936), (70, 2000)]
SETTINGS = [(1.0, 0, 1.0, 0.0), (1.0, 50, 0.9, 0.0), (0.7, 0, 0.9, 0.0), (0.8, 40, 1.0, 0.0), (1.2, 0, 1.0, 0.05), (0.6, 20, 0.95, 0.02), (1.3, 0, 0.5, 0.0), (0.0, 5, 0.5, 0.5),
            (1.5, 200, 1.0, 0.1), (0.9, 1000, 0.99, 0.0), (1.0, 1, 1.0, 0.0), (2.0, 0, 0.999, 1e-6), (0.05, 3, 0.3, 0.0), (30.0, 0, 0.8, 0.0), (1.0, 5000, 0.7, 0.001)]


@pytest.mark.parametrize("dtype", [F32, BF, F16])
@pytest.mark.parametrize("N,V", SIZES)
def test_settings_by_row(svip, dtype, N, V):
    for turn in range(3):
        z = logits(N, V, dtype, seed=100 * turn + V, masked=0.3 if turn == 2 and V > 60 else 0.0)
        which = [SETTINGS[(n + 5 * turn) % len(SETTINGS)] for n in range(N)]
        T, k, p, m = zip(*which)
        check(svip, z, torch.rand(N, generator=gen(V + turn)), T, k, p, m)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("setting", SETTINGS)
def test_each_setting(svip, dtype, setting):
    N, V = 12, 32000
    T, k, p, m = ([x] * N for x in setting)
    check(svip, logits(N, V, dtype, seed=7), torch.rand(N, generator=gen(9)), T, k, p, m)


@pytest.mark.parametrize("dtype", [F32, BF, F16])
@pytest.mark.parametrize("V", [1500, 5003, 32000, 70001])
@pytest.mark.parametrize("kind", ["plain", "masked", "ties"])
def test_top_k_that_the_chunks_do_not_decide(svip, dtype, V, kind):
    """More tokens than chunks of 64 logits, up to what the list of candidates holds and beyond, all but so many masked, and on values that repeat."""
    T, k, p, m = zip((1.0, 24, 1.0, 0.0), (1.5, 600, 0.9, 0.0), (0.9, 1000, 0.99, 0.0), (1.0, 1024, 1.0, 0.01), (2.0, 1025, 0.95, 0.0), (1.0, 3000, 1.0, 0.0), (3.0, 4096, 0.8, 0.001),
                     (1.0, 4097, 0.9, 0.0), (1.0, V - 1, 1.0, 0.0))
    z = logits(len(T), V, dtype, seed=V + 1, masked=0.97 if kind == "masked" else 0.0)
    if kind == "ties":
        z.copy_((z.float() * 4).round() / 4)
    check(svip, z, torch.rand(len(T), generator=gen(V)), T, k, p, m)


@pytest.mark.parametrize("V,dtype", [(300001, BF), (1 << 22, F16), ((1 << 22) - 3, F32)])
def test_large_vocabularies(svip, V, dtype):
    """More chunks than a workgroup's threads keep, and as many as there may be."""
    T, k, p, m = zip((1.0, 0, 1.0, 0.0), (1.0, 50, 0.9, 0.0), (0.7, 0, 0.9, 0.0), (1.2, 0, 1.0, 0.05), (0.9, 1024, 0.99, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 1025, 1.0, 0.01))
    check(svip, logits(7, V, dtype, seed=2), torch.rand(7, generator=gen(4)), T, k, p, m)


@pytest.mark.parametrize("scale", [0.0, 1e-3, 0.05, 0.5])
@pytest.mark.parametrize("setting", [(1.0, 0, 0.9, 0.0), (1.0, 60000, 0.5, 0.0), (1.0, 0, 1.0, 1e-4), (1.0, 0, 1.0, 0.0), (0.1, 30000, 1.0, 0.0), (1.0, 9000, 0.97, 0.2)])
def test_flat_rows(svip, scale, setting):
    """Kept sets of most of the vocabulary, and rows of one value."""
    N, V = 4, 100003
    for dtype in (F32, BF):
        z = rows_of(N, V, dtype)
        z.copy_(torch.randn(N, V, generator=gen(3)) * scale)
        T, k, p, m = ([x] * N for x in setting)
        check(svip, z, [0.0, 0.37, 0.5, 1 - 2.0 ** -24], T, k, p, m)


def test_settings_left_out(svip):
    z = logits(6, 5000, BF, seed=1)
    u = torch.rand(6, generator=gen(2))
    check(svip, z, u)
    check(svip, z, u, T=[0.5] * 6)
    check(svip, z, u, k=[10] * 6)
    check(svip, z, u, p=[0.5] * 6)
    check(svip, z, u, m=[0.1] * 6)
    a = run(svip, z, u, k=[10] * 6)
    b = run(svip, z, u, k=[10] * 6, prob=False, kept=False)
    assert (a[0] == b[0]).all() and b[1] is None


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_masks_and_numbers_that_are_none(svip, dtype):
    V = 3001
    inf, nan = math.inf, math.nan
    z = rows_of(12, V, dtype)
    z.copy_(torch.randn(12, V, generator=gen(4)))
    z[0] = -inf                                                  # nothing is left
    z[1] = nan
    z[2] = -inf
    z[2, 1234] = -5.0                                            # one token
    z[3, ::2] = nan
    z[4, 17] = inf                                               # +inf leaves weight to nothing else
    z[4, 2999] = inf
    z[5] = torch.finfo(dtype).min                                # masks of the type's lowest value, all of them
    z[6] = torch.finfo(dtype).min
    z[6, 2000:2003] = 1.0
    z[7, :] = -inf
    z[7, 5], z[7, 6], z[7, 7] = -0.0, 0.0, nan
    z[8, 0], z[8, V - 1] = -inf, 20.0
    z[9] = torch.finfo(dtype).max
    z[10] = nan
    z[10, 3000] = -inf
    u = torch.rand(12, generator=gen(6))
    for T, k, p, m in ((1.0, 0, 1.0, 0.0), (1.0, 2, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.3), (0.0, 0, 1.0, 0.0), (3e38, 3, 0.5, 0.0), (1e-38, 0, 0.9, 0.5)):
        check(svip, z, u, [T] * 12, [k] * 12, [p] * 12, [m] * 12)


def test_ties_stay_together(svip):
    z = rows_of(4, 1000, F32)
    z.copy_(-torch.arange(1000.0))
    z[:, 100:164] = 3.0                                          # 64 equal largest
    token, prob, kept, _ = run(svip, z, [0.0, 0.5, 0.25, 1 - 2.0 ** -24], [1.0, 1.0, 0.0, 1.0], [1, 64, 1, 10], [1.0, 0.01, 1.0, 1.0])
    assert token.tolist() == [100, 132, 100, 163] and kept.tolist() == [64, 64, 1, 64]
    assert prob.tolist() == [1 / 64, 1 / 64, 1.0, 1 / 64]


def test_uniforms_walk_the_vocabulary(svip):
    """A row of equal logits: token floor(u V)."""
    V, N = 4096, 512
    z = rows_of(N, V, BF)
    z.fill_(-3.0)
    u = torch.arange(N) / N + 2.0 ** -13
    token, prob, kept, _ = run(svip, z, u, [0.5] * N)
    assert (token == (u * V).long().numpy()).all() and (kept == V).all() and (prob == 1 / V).all()


def test_bad_settings_are_flagged(svip):
    nan, inf = math.nan, math.inf
    rows = [(1.0, 0, 1.0, 0.0, 0.5, True), (-1.0, 0, 1.0, 0.0, 0.5, False), (nan, 0, 1.0, 0.0, 0.5, False), (inf, 0, 1.0, 0.0, 0.5, False),
            (1.0, -1, 1.0, 0.0, 0.5, False), (1.0, 0, 0.0, 0.0, 0.5, False), (1.0, 0, -0.5, 0.0, 0.5, False), (1.0, 0, nan, 0.0, 0.5, False),
            (1.0, 0, 1.0, -0.1, 0.5, False), (1.0, 0, 1.0, 1.1, 0.5, False), (1.0, 0, 1.0, nan, 0.5, False), (1.0, 0, 1.0, 0.0, 1.0, False),
            (1.0, 0, 1.0, 0.0, -0.1, False), (1.0, 0, 1.0, 0.0, nan, False), (1.0, 2 ** 31 - 1, 7.0, 1.0, 0.0, True)]
    z = logits(len(rows), 2500, BF, seed=12)
    T, k, p, m, u, good = zip(*rows)
    token, prob, kept, flags = run(svip, z, u, T, k, p, m)
    assert flags == svip.FLAG_BAD_SETTING
    good = np.array(good)
    assert (token[~good] == -1).all() and (prob[~good] == 0).all() and (kept[~good] == 0).all()
    assert (token[good] >= 0).all() and (kept[good] >= 1).all()


def test_law(svip):
    """A million draws with a filter on eight tokens: chi-square against the filtered weights (5 degrees of freedom, 99.9 % quantile 20.52)."""
    z = torch.tensor([1.0, 0.5, -1.0, 2.0, 0.0, 1.5, -3.0, 0.25])
    N = 1 << 20
    rows = z.repeat(N, 1).cuda()
    token, prob, kept, _ = run(svip, rows, torch.rand(N, generator=gen(77)), [0.8] * N, [6] * N)
    w = np.exp(z.double().numpy() / 0.8)
    w[[2, 6]] = 0
    want = w / w.sum() * N
    have = np.bincount(token, minlength=8)
    assert (kept == 6).all() and have[2] == 0 and have[6] == 0
    use = want > 0
    assert ((have[use] - want[use]) ** 2 / want[use]).sum() < 20.52


def test_far_rows(svip):
    """Rows further apart than 2^32 bytes."""
    V, stride, N = 1000, 1 << 29, 6
    if torch.cuda.mem_get_info()[0] < 2 * N * stride:
        pytest.skip("not enough memory")
    whole = torch.empty(N * stride, dtype=BF, device="cuda")
    z = whole.as_strided((N, V), (stride, 1))
    z.copy_(logits(N, V, BF, seed=5))
    check(svip, z, torch.rand(N, generator=gen(1)), [0.9] * N, [30] * N, [0.9] * N)


def test_streams_side_by_side_and_the_same_bits(svip):
    """Two calls under way at once in workspaces of their own, and every run the same."""
    N, V = 40, 40000
    z = [logits(N, V, BF, seed=s) for s in (1, 2)]
    u = torch.rand(N, generator=gen(3))
    T, k, p, m = zip(*[SETTINGS[n % len(SETTINGS)] for n in range(N)])
    want = [run(svip, x, u, T, k, p, m) for x in z]
    dev = [torch.as_tensor(x, dtype=t).cuda() for x, t in ((T, F32), (k, torch.int32), (p, F32), (m, F32), (u, F32))]
    streams = [torch.cuda.Stream() for _ in z]
    spaces = [svip.new_sample_workspace(BF, N, V) for _ in z]
    outs = [[(torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, dtype=torch.int32, device="cuda")) for _ in range(5)] for _ in z]
    torch.cuda.synchronize()
    for turn in range(5):
        for i, st in enumerate(streams):
            token, prob, kept = outs[i][turn]
            svip.sample(z[i], u=dev[4], temperature=dev[0], top_k=dev[1], top_p=dev[2], min_p=dev[3], token_out=token, prob_out=prob, kept_out=kept,
                        workspace=spaces[i], stream=st)
    torch.cuda.synchronize()
    for i in range(2):
        for token, prob, kept in outs[i]:
            assert (token.cpu().numpy() == want[i][0]).all() and (prob.cpu().numpy() == want[i][1]).all() and (kept.cpu().numpy() == want[i][2]).all()


def test_refusals(svip):
    z = logits(4, 100, BF, seed=1)
    ws = svip.new_sample_workspace(BF, 4, 100)
    u, token = torch.rand(4, device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda")
    ok = dict(u=u, token_out=token, workspace=ws)
    svip.sample(z, **ok)
    for bad in (dict(u=u[:3]), dict(u=u.double()), dict(token_out=token.long()), dict(token_out=token[:3]), dict(temperature=u[:3]), dict(top_k=u),
                dict(top_p=u.half()), dict(min_p=torch.rand(8, device="cuda")[::2]), dict(prob_out=token), dict(kept_out=u)):
        with pytest.raises(ValueError):
            svip.sample(z, **{**ok, **bad})
    with pytest.raises(ValueError):
        svip.sample(z.t(), **ok)
    with pytest.raises(svip.SvipError):
        svip.sample(z.float()[:, 1:97], **ok)                    # rows not on 16 bytes
    with pytest.raises(svip.SvipError):
        svip.sample(z, u=u, token_out=token, workspace=ws[:256])


# ---- together ------------------------------------------------------------------------------------------------------------------------------

def test_a_drafting_loop_in_a_graph(svip):
    """Hidden state -> 4 bits -> logits -> token -> the token's row, the next hidden state, four positions long: eager, and captured and replayed with new
    inputs between eager runs; every step against the definitions on what the step before it gave."""
    B, V, D, steps = 9, 5003, 384, 4
    E4, S8 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
    weight = (torch.randn(V, D, generator=gen(1)) * 0.3).bfloat16().cuda()
    wq, wsc = torch.empty(V, D // 2, dtype=torch.uint8, device="cuda").view(E4), torch.empty(V, D // 32, dtype=torch.uint8, device="cuda").view(S8)
    svip.quantize_mx(weight, q_out=wq, scale_out=wsc)
    table = torch.empty(V, D, dtype=F32, device="cuda")
    svip.mx_rows(wq, wsc, out=table)
    hidden0 = torch.empty(B, D, dtype=BF, device="cuda")
    u = torch.empty(steps, B, device="cuda")
    T, k, p, m = (torch.as_tensor(x, dtype=t).cuda() for x, t in zip(zip(*[SETTINGS[n] for n in range(B)]), (F32, torch.int32, F32, F32)))

    def buffers():
        return dict(hidden=[torch.empty(B, D, dtype=BF, device="cuda") for _ in range(steps)], hq=torch.empty(B, D // 2, dtype=torch.uint8, device="cuda").view(E4),
                    hs=torch.empty(B, D // 32, dtype=torch.uint8, device="cuda").view(S8), z=[torch.empty(B, 5008, dtype=BF, device="cuda")[:, :V] for _ in range(steps)],
                    token=[torch.empty(B, dtype=torch.int32, device="cuda") for _ in range(steps)], prob=[torch.empty(B, device="cuda") for _ in range(steps)],
                    hw=svip.new_head_workspace(svip.HEAD_LOGITS_MX, BF, B, V, D), sw=svip.new_sample_workspace(BF, B, V))

    def loop(b):
        hidden = hidden0
        for j in range(steps):
            svip.quantize_mx(hidden, q_out=b["hq"], scale_out=b["hs"])
            svip.head_logits_mx(b["hq"], b["hs"], wq, wsc, logits_out=b["z"][j], workspace=b["hw"])
            svip.sample(b["z"][j], u=u[j], temperature=T, top_k=k, top_p=p, min_p=m, token_out=b["token"][j], prob_out=b["prob"][j], workspace=b["sw"])
            svip.mx_rows(wq, wsc, ids=b["token"][j], out=b["hidden"][j])
            hidden = b["hidden"][j]

    def fill(seed):
        hidden0.copy_(torch.randn(B, D, generator=gen(seed)))
        u.copy_(torch.rand(steps, B, generator=gen(seed + 1)))

    eager, captured = buffers(), buffers()
    fill(10)
    loop(eager)
    torch.cuda.synchronize()
    x = hidden0.float()
    for j in range(steps):                                       # hidden states of a table's row are on its grid already: quantised without error
        if j:
            want = x.double() @ table.double().T
            size = x.double().abs() @ table.double().abs().T
            assert ((eager["z"][j].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -16 * size).all()
        ref = [reference(eager["z"][j][n].cpu().double().numpy(), *(float(s[n]) if s is not k else int(s[n]) for s in (T, k, p, m)), float(u[j, n])) for n in range(B)]
        assert eager["token"][j].tolist() == [r[0] for r in ref]
        x = table[eager["token"][j].long()]
        assert torch.equal(eager["hidden"][j].float(), x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        loop(captured)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        loop(captured)
    for seed in (10, 20, 30, 10):
        fill(seed)
        loop(eager)
        torch.cuda.synchronize()
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            for j in range(steps):
                assert torch.equal(captured["token"][j], eager["token"][j]) and torch.equal(captured["prob"][j], eager["prob"][j])
                assert torch.equal(captured["z"][j], eager["z"][j]) and torch.equal(captured["hidden"][j], eager["hidden"][j])


def test_two_graphs_share_workspaces(svip):
    """Calls of two sizes, K in splits, captured into a graph each on the same two workspaces, replayed in turn on one stream with eager calls between."""
    E4, S8 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
    V, K = 3001, 2176
    sizes = (70, 5)
    wq, wsc = torch.empty(V, K // 2, dtype=torch.uint8, device="cuda").view(E4), torch.empty(V, K // 32, dtype=torch.uint8, device="cuda").view(S8)
    svip.quantize_mx((torch.randn(V, K, generator=gen(1)) * 0.2).bfloat16().cuda(), q_out=wq, scale_out=wsc)
    hw = torch.empty(max(svip.head_workspace_bytes(svip.HEAD_LOGITS_MX, BF, n, V, K) for n in sizes), dtype=torch.uint8, device="cuda")
    sw = svip.new_sample_workspace(BF, max(sizes), V)
    state = []
    for N in sizes:
        T, k, p, m = (torch.as_tensor(x, dtype=t).cuda() for x, t in zip(zip(*[SETTINGS[n % len(SETTINGS)] for n in range(N)]), (F32, torch.int32, F32, F32)))
        state.append(dict(x=torch.empty(N, K, dtype=BF, device="cuda"), u=torch.empty(N, device="cuda"), T=T, k=k, p=p, m=m,
                          hq=torch.empty(N, K // 2, dtype=torch.uint8, device="cuda").view(E4), hs=torch.empty(N, K // 32, dtype=torch.uint8, device="cuda").view(S8),
                          z=torch.empty(N, 3008, dtype=BF, device="cuda")[:, :V], token=torch.empty(N, dtype=torch.int32, device="cuda"),
                          kept=torch.empty(N, dtype=torch.int32, device="cuda")))

    def step(s, hw, sw):
        svip.quantize_mx(s["x"], q_out=s["hq"], scale_out=s["hs"])
        svip.head_logits_mx(s["hq"], s["hs"], wq, wsc, logits_out=s["z"], workspace=hw)
        svip.sample(s["z"], u=s["u"], temperature=s["T"], top_k=s["k"], top_p=s["p"], min_p=s["m"], token_out=s["token"], kept_out=s["kept"], workspace=sw)

    graphs = []
    for s in state:
        s["x"].normal_()
        s["u"].uniform_()
        step(s, hw, sw)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(s, hw, sw)
    for turn in range(4):
        want = []
        for N, s in zip(sizes, state):
            s["x"].copy_(torch.randn(N, K, generator=gen(turn)))
            s["u"].copy_(torch.rand(N, generator=gen(50 + turn)))
            step(s, svip.new_head_workspace(svip.HEAD_LOGITS_MX, BF, N, V, K), svip.new_sample_workspace(BF, N, V))
            want.append([s[x].clone() for x in ("z", "token", "kept")])
            for x in ("z", "token", "kept"):
                s[x].zero_()
        for i in (0, 1) if turn % 2 else (1, 0):
            graphs[i].replay()
        torch.cuda.synchronize()
        for s, w in zip(state, want):
            assert all(torch.equal(s[x], y) for x, y in zip(("z", "token", "kept"), w))


def test_sampled_tokens_go_on_to_verification(svip):
    """The sampler's probability is that of svip_warp_logits' row: what svip_draft_step and svip_verify call q(x) of the filtered row."""
    N, V = 16, 9000
    z = logits(N, V, F32, seed=31)
    u = torch.rand(N, generator=gen(32))
    token, prob, kept, _ = run(svip, z, u, [0.8] * N, [40] * N, [0.9] * N)
    rows = torch.empty(N, 1, V, device="cuda")
    rows[:, 0] = z
    count = torch.empty(N, dtype=torch.int32, device="cuda")
    svip.warp_logits(rows, temperature=0.8, top_k=40, top_p=float(torch.tensor(0.9)), kept_out=count)
    assert count.tolist() == kept.tolist()
    q = torch.softmax(rows[:, 0].double() / float(torch.tensor(0.8)), 1)
    assert torch.allclose(q[torch.arange(N), torch.as_tensor(token).long()].cpu(), torch.as_tensor(prob).double(), rtol=1e-6, atol=0)
