"""The balanced form of purekv_decode_paged where its short runs have work: they do from more than eight tiles per CTA at work on (2368 tiles
with two CTAs per SM, 3552 with three), so that CTAs go from run to run, and requests are cut into parts that several CTAs hold."""
import pytest
import torch

from paper_2510_25600_b200 import binding as P
from tests import paged_common as pc

pytestmark = pytest.mark.gpu


def rows(c, r, which):
    """Request r's rows [n, hkv, d] in the values they stand for, on the GPU in 64 bits."""
    pool, scale = (c.k, c.k_scale) if which == "k" else (c.v, c.v_scale)
    at = torch.arange(max(0, c.lens[r]))
    held = pool.view(torch.uint8) if c.kind == "e4m3" else pool
    x = held[c.table[r, at // c.page].long(), at % c.page].view(pool.dtype).cuda().double()
    return x if scale is None else x * scale.cuda().double()[:, None]


def check(seed, lens, H, hkv, d, kind, page, tile, calls=1):
    c = pc.Cache(seed, lens, hkv, d, kind, page)
    three = kind == "e4m3" and H // hkv <= 8
    assert sum(-(-n // tile) for n in lens) * hkv > 8 * 148 * (3 if three else 2), "every tile would be in a long run"
    q = (1.5 * torch.randn((len(lens), H, d), generator=torch.Generator().manual_seed(seed))).to(torch.float32 if kind == "fp32" else torch.bfloat16).cuda()
    cache, scales = c.cuda()
    status, lse = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty((len(lens), H), device="cuda")
    got = None
    for hint in [0, (1 << 31) - 1] * calls:
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        P.purekv_decode_paged(q, *cache, max_len=hint, out=out, lse=lse.fill_(float("nan")), status=status, **scales)
        assert P.purekv_poll_status(status) == 0
        assert got is None or (torch.equal(got, out) and torch.equal(z, lse)), "which CTA takes a run must not change its result"
        got, z = out, lse.clone()
    dtype = "fp32" if kind == "fp32" else "bf16"
    for r, n in enumerate(lens):
        if n == 0:
            assert (got[r] == 0).all() and torch.isneginf(z[r]).all()
            continue
        o, s, weight, size = pc.attention(q[r].double(), rows(c, r, "k"), rows(c, r, "v"))
        assert ((got[r].double() - o).abs() <= pc.attention_tolerance(dtype, kind, o, weight, size, d)).all(), r
        assert ((z[r].double() - s).abs() <= pc.lse_tolerance(s, size, d)).all(), r


def lengths(seed, n, low, high):
    return torch.randint(low, high + 1, (n,), generator=torch.Generator().manual_seed(seed)).tolist()


@pytest.mark.parametrize("page", [16, 12])
@pytest.mark.parametrize("kind,H,hkv,d,n,high,tile", [
    ("bf16", 8, 4, 128, 14, 5000, 64), ("bf16", 10, 2, 64, 30, 9000, 128), ("fp32", 4, 4, 128, 8, 5000, 32), ("fp32", 6, 2, 64, 20, 6000, 64),
    ("e4m3", 8, 8, 128, 24, 5000, 128), ("e4m3", 24, 2, 64, 60, 12000, 256),
])
def test_long_requests(kind, H, hkv, d, n, high, tile, page):
    check(40, [0, 1] + lengths(41, n - 2, high // 2, high) + [0], H, hkv, d, kind, page, tile)


@pytest.mark.parametrize("page", [16, 7])
@pytest.mark.parametrize("kind,H,hkv,d", [("bf16", 8, 8, 128), ("bf16", 72, 8, 64), ("fp32", 8, 8, 64), ("e4m3", 16, 8, 64), ("e4m3", 80, 8, 128)])
def test_many_short_requests(kind, H, hkv, d, page):
    # more requests than the CTAs' table of sums has groups, some of them empty, ends of requests in every run
    check(42, lengths(43, 500, 1, 90) + [0] * 7, H, hkv, d, kind, page, 256)


@pytest.mark.parametrize("kind,tile", [("bf16", 64), ("e4m3", 128)])
def test_one_long_request_among_short_ones(kind, tile):
    lens = lengths(44, 127, 1, 900)
    lens[5] = 40000 if kind == "bf16" else 16000
    check(45, lens, 8, 4 if kind == "bf16" else 8, 128, kind, 32, tile)


@pytest.mark.parametrize("kind,hkv,tile", [("bf16", 4, 64), ("e4m3", 8, 128)])
def test_again_and_again(kind, hkv, tile):
    check(46, lengths(47, 16, 3000, 4500), 8, hkv, 128, kind, 16, tile, calls=20)
