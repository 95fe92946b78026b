"""Tokens of svip_sample in a round that svip_verify checks: both sides filtered by one setting."""
import numpy as np
import pytest
import torch

from helpers import Round, check_verify
from test_sample_draw_gpu import gen, sample

pytestmark = pytest.mark.gpu

F32, BF, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype", [F32, BF, F16])
@pytest.mark.parametrize("k,p", [(0, 1.0), (40, 1.0), (0, 0.9), (40, 0.9)])
def test_a_round_of_sampled_tokens_is_verified(svip, dtype, k, p):
    """svip_sample's tokens, drawn from rows as they are, are drafted from what svip_warp_logits leaves of them with the same settings: svip_verify over such
    rows of drafter and target takes or corrects them as the oracle does."""
    B, gamma, V, T = 12, 3, 5003, 0.8
    pad = -(-V // 8) * 8
    z = torch.randn(B, gamma, V, generator=gen(41)) * 2.5
    draft = torch.empty(B, gamma, pad, dtype=dtype, device="cuda")[:, :, :V]
    target = torch.empty(B, gamma + 1, pad, dtype=dtype, device="cuda")[:, :, :V]
    draft.copy_(z)
    target.copy_(torch.cat([z + 0.7 * torch.randn(B, gamma, V, generator=gen(42)), torch.randn(B, 1, V, generator=gen(43)) * 2.5], 1))
    rows = draft.reshape(B * gamma, V)
    if rows.stride(0) != pad:                                    # (reshape may copy: rows begin on 16 bytes)
        rows = torch.empty(B * gamma, pad, dtype=dtype, device="cuda")[:, :V].copy_(rows)
    token, prob, kept = sample(svip, rows, torch.rand(B * gamma, generator=gen(44)), T, k, p)
    g = Round(svip, draft, target, torch.zeros(B, gamma), torch.rand(B, gamma, generator=gen(45)), torch.rand(B, generator=gen(46)), T, 1.0)
    exact_p = float(torch.tensor(p))                             # the fp32 number that the rows' settings hold
    left = torch.empty(B * gamma, dtype=torch.int32, device="cuda")
    svip.warp_logits(g.draft, temperature=T, top_k=k, top_p=exact_p, kept_out=left)
    svip.warp_logits(g.target, temperature=T, top_k=k, top_p=exact_p)
    assert (left.cpu().numpy() == kept).all()
    q = torch.softmax(g.draft.double() / float(torch.tensor(T)), 2).cpu().view(B * gamma, V).numpy()
    assert np.allclose(q[np.arange(B * gamma), token], prob, rtol=1e-6, atol=0)
    g.tokens.copy_(torch.as_tensor(token).view(B, gamma))
    g.draft_len.fill_(gamma)
    g.verify(lse=None)
    st = check_verify(g.draft.cpu(), g.target.cpu(), T, token.reshape(B, gamma), np.full(B, gamma), g.u_accept.cpu(), g.u_resample.cpu(), g)
    assert st["seqs"] == B and len(set(g.n_accepted.tolist())) > 1
