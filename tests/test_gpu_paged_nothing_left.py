"""Requests of the paged decode step that have rows, none of which counts: o = 0 and lse = -inf, as for a request without rows."""
import pytest
import torch

from paper_2510_25600_b200 import binding as P
from tests import paged_common as pc

pytestmark = pytest.mark.gpu
HINTS = (0, 1, 64, 129, 257, 600, 9000, (1 << 31) - 1)


def step(cache, scales, q, hint):
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = P.purekv_decode_paged(q, *cache, max_len=hint, out=torch.full_like(q, float("nan")), lse=lse, status=status, **scales)
    return out, lse, status.item()


def is_nothing(out, lse):
    return (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 16), (128, 12)])
def test_every_page_is_missing(kind, d, page):
    c = pc.Cache(60, [40, 700, 9000, 5], 2, d, kind, page)
    cache, scales = c.cuda()
    q = torch.randn((4, 8, d), generator=torch.Generator().manual_seed(60)).to(torch.float32 if kind == "fp32" else torch.bfloat16).cuda()
    for hint in HINTS:
        want, want_lse, st = step(cache, scales, q, hint)
        assert st == 0
        kp, vp, table, lens = cache
        table = table.clone()
        table[:3] = -1
        out, lse, st = step((kp, vp, table, lens), scales, q, hint)
        assert st == P.ERR_BAD_PAGE and is_nothing(out[:3], lse[:3]), hint
        assert torch.equal(out[3], want[3]) and torch.equal(lse[3], want_lse[3])


def test_no_columns_and_no_pages():
    q = torch.ones((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    lens = torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    for n_pages, columns in ((2, 0), (0, 2)):
        pool = torch.zeros((n_pages, 16, 2, 64), dtype=torch.bfloat16, device="cuda")
        for hint in HINTS:
            out, lse, st = step((pool, pool, torch.zeros((2, columns), dtype=torch.int32, device="cuda"), lens), {}, q, hint)
            assert st == P.ERR_BAD_PAGE and is_nothing(out, lse)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_every_logit_is_minus_infinity(kind):
    c = pc.Cache(61, [300, 6000], 1, 128, kind)
    cache, _ = c.cuda()
    cache[0][..., 0] = float("-inf")
    cache[0][..., 1:] = 0
    q = torch.zeros((2, 3, 128), dtype=torch.float32 if kind == "fp32" else torch.bfloat16, device="cuda")
    q[..., 0] = 1
    for hint in HINTS:
        out, lse, st = step(cache, {}, q, hint)
        assert st == 0 and is_nothing(out, lse)
