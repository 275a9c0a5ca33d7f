"""Every way of launching the paged decode step against attention in 64 bits: the hint of the longest request picks the form (clusters of
1 to 16 CTAs, small CTAs, several of them per SM, the balanced form), whatever the lengths are, and the outputs, the log-sum-exps and the
status have to be right for each."""
import pytest
import torch

from paper_2510_25600_b200 import binding as P
from tests import paged_common as pc

pytestmark = pytest.mark.gpu
HINTS = (0, 1, 16, 64, 65, 128, 129, 200, 256, 257, 400, 600, 1200, 2048, 2049, 4000, 9000, 1 << 15, 1 << 17, (1 << 31) - 1)


def batches():
    g = torch.Generator().manual_seed(90)
    yield [1000]
    yield [700, 0, 3, 64]
    yield [129, 255, 256, 257, 1, 0, 511, 512, 513]
    yield torch.randint(0, 300, (24,), generator=g).tolist()
    yield torch.randint(0, 200, (90,), generator=g).tolist()


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("H,hkv,d,page", [(28, 4, 128, 16), (8, 2, 64, 32), (24, 2, 128, 7), (2, 1, 64, 64)])
def test_every_way_against_64_bits(kind, H, hkv, d, page):
    dtype = "fp32" if kind == "fp32" else "bf16"
    for lens in batches():
        c = pc.Cache(90, lens, hkv, d, kind, page)
        q = (1.5 * torch.randn((len(lens), H, d), generator=torch.Generator().manual_seed(91))).to(torch.float32 if kind == "fp32" else torch.bfloat16)
        want = [pc.attention(q[r].double(), c.rows(r, "k"), c.rows(r, "v")) for r in range(len(lens))]
        o, z, weight, size = (torch.stack(x) for x in zip(*want))
        tol = pc.attention_tolerance(dtype, kind, o.flatten(0, 1), weight.flatten(0, 1), size.flatten(), d).view(o.shape)
        z_tol = pc.lse_tolerance(z, size, d)
        empty = torch.tensor(lens) == 0
        cache, scales = c.cuda()
        dq, status = q.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
        for hint in HINTS:
            lse = torch.full((len(lens), H), float("nan"), device="cuda")
            out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
            P.purekv_decode_paged(dq, *cache, max_len=hint, out=out, lse=lse, status=status, **scales)
            assert P.purekv_poll_status(status) == 0, hint
            got, got_lse = out.cpu().double(), lse.cpu().double()
            assert ((got - o).abs() <= tol).all(), (lens, hint)
            assert (got[empty] == 0).all() and torch.isneginf(got_lse[empty]).all(), (lens, hint)
            assert ((got_lse - z).abs() <= z_tol)[~empty].all(), (lens, hint)
