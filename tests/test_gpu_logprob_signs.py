"""Log probabilities are no more than 0 and entropies no less, also of rows whose distribution is one token's."""
import math

import pytest
import torch

from paper_2311_15806_b200 import binding as B
from tests import int8_reference as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("scale", [1.0, 0.7, 3.0])
@pytest.mark.parametrize("T,V", [(1000, 1), (1000, 2), (1000, 900), (400, 9001), (20, 40009), (2, 128000), (300, 90001)])
def test_no_probability_is_above_one(dtype, scale, T, V):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T + V)
    l = torch.randn((T, V), generator=gen, device="cuda") * 2
    sure = torch.randint(0, V, (T,), generator=gen, device="cuda")
    at = torch.arange(T, device="cuda")
    l[at, sure] += 30 + 40 * torch.rand((T,), generator=gen, device="cuda")
    if V > 1:
        l[::3] = -math.inf                              # nothing but that token
        l[at[::3], sure[::3]] = torch.randn((len(at[::3]),), generator=gen, device="cuda") * 20
    l = l.to(R.TYPES[dtype])
    tokens = sure.int()[:, None].contiguous()
    lp, ent = torch.empty((T, 1), device="cuda"), torch.empty(T, device="cuda")
    top, tlp = torch.empty((T, 3), dtype=torch.int32, device="cuda"), torch.empty((T, 3), device="cuda")
    B.pipe_token_logprobs(l, tokens, lp, entropy=ent, top=top, top_logprobs=tlp, scale=scale)
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_OK
    assert torch.equal(top[:, 0], tokens[:, 0]) and torch.equal(tlp[:, :1], lp)
    assert (lp <= 0).all() and (tlp <= 0).all() and (ent >= 0).all()
    w_lp, w_ent, w_ids, w_top, tol, ent_tol = R.logprobs(l.cpu(), tokens.cpu(), 3, scale)
    R.close(lp, w_lp, tol, 1 + w_lp.abs())
    R.close(ent, w_ent, ent_tol, 1 + w_ent.abs())
    assert torch.equal(top.cpu(), w_ids)
