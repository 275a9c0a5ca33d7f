"""The paged decode step at the ends of what it takes: as many requests as a grid has, more heads than CTAs at work."""
import math

import pytest
import torch

from paper_2510_25600_b200 import binding as P
from tests import paged_common as pc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("hint", [0, 1, 70000])
def test_as_many_requests_as_there_can_be(kind, hint):
    # a row each, every 97th request without one: the output is the value, the log-sum-exp the logit
    n, d, dtype = 65535, 64, pc.TYPES[kind]
    g = torch.Generator("cuda").manual_seed(110)
    kp, vp, q = (torch.randn(shape, generator=g, device="cuda").to(dtype) for shape in ((n, 1, 1, d), (n, 1, 1, d), (n, 1, d)))
    table = torch.randperm(n, generator=g, device="cuda").to(torch.int32)[:, None]
    lens = torch.ones(n, dtype=torch.int32, device="cuda")
    lens[::97] = 0
    lse, status = torch.full((n, 1), float("nan"), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = P.purekv_decode_paged(q, kp, vp, table, lens, max_len=hint, lse=lse, status=status)
    assert P.purekv_poll_status(status) == 0
    page, there = table[:, 0].long(), lens > 0
    want = torch.where(there[:, None], vp[page, 0, 0], torch.zeros((), dtype=dtype, device="cuda"))
    assert torch.equal(out[:, 0], want)                                   # one weight of 1: the value as it is
    terms = q[:, 0].double() * kp[page, 0, 0].double() / math.sqrt(d)
    assert torch.isneginf(lse[~there]).all()
    assert ((lse[:, 0].double() - terms.sum(1)).abs() <= pc.lse_tolerance(terms.sum(1), terms.abs().sum(1), d))[there].all()


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("H,hkv", [(400, 400), (1200, 600)])
def test_more_heads_than_ctas_at_work(kind, H, hkv):
    lens, d = [0, 70, 3, 300], 64
    c = pc.Cache(111, lens, hkv, d, kind)
    q = torch.randn((len(lens), H, d), generator=torch.Generator().manual_seed(111)).to(torch.float32 if kind == "fp32" else torch.bfloat16)
    cache, scales = c.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for hint in (0, 1, 300, 100000):
        lse = torch.full((len(lens), H), float("nan"), device="cuda")
        out = P.purekv_decode_paged(q.cuda(), *cache, max_len=hint, out=torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda"), lse=lse, status=status, **scales)
        assert P.purekv_poll_status(status) == 0
        got, got_lse = out.cpu().double(), lse.cpu().double()
        assert (got[0] == 0).all() and torch.isneginf(got_lse[0]).all()
        for r in (1, 2, 3):
            o, z, weight, size = pc.attention(q[r].double(), c.rows(r, "k"), c.rows(r, "v"))
            assert ((got[r] - o).abs() <= pc.attention_tolerance("fp32" if kind == "fp32" else "bf16", kind, o, weight, size, d)).all(), (hint, r)
            assert ((got_lse[r] - z).abs() <= pc.lse_tolerance(z, size, d)).all(), (hint, r)
