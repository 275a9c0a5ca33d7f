"""Stores into the paged cache that are larger than one pass of the kernels' blocks over their work: several batches of rows for each of a
compaction's warps, more requests than a block keeps offsets of, offsets past 32 bits, prompts into e4m3 pages."""
import types

import pytest
import torch

from paper_2510_25600_b200 import binding as P
from tests import paged_common as pc
from tests.test_gpu_paged_append import check as check_append

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def starts(counts):
    return [0, *torch.tensor(counts).cumsum(0).tolist()]


def check(seed, lens, kept, layers, hkv, d, kind, page, n_pages=None, prefix=0):
    g = torch.Generator("cuda").manual_seed(seed)
    dtype = torch.float32 if kind == "fp32" else torch.bfloat16
    cu, ck, t = starts(lens), starts(kept), sum(kept)
    k, v = (torch.empty((layers, cu[-1], hkv, d), dtype=dtype, device="cuda").normal_(generator=g) for _ in "kv")
    idx = torch.empty((layers, hkv, t), dtype=torch.int32, device="cuda")
    for r, (n, m) in enumerate(zip(lens, kept)):
        idx[:, :, ck[r]:ck[r + 1]] = torch.rand((layers, hkv, n), generator=g, device="cuda").argsort(dim=2)[:, :, :m].sort(dim=2).values
    counts = [-(-(prefix + m) // page) for m in kept]
    n_pages = n_pages or sum(counts) + 3
    order = n_pages - 1 - torch.randperm(sum(counts), generator=g, device="cuda").to(torch.int32)   # the pool's last pages
    table = torch.full((len(lens), max(counts) + 1), -1, dtype=torch.int32, device="cuda")
    for r, n in enumerate(counts):
        table[r, :n] = order[sum(counts[:r]):sum(counts[:r]) + n]
    pools = [torch.empty((layers, n_pages, page, hkv, d), dtype=pc.TYPES[kind], device="cuda") for _ in "kv"]
    used = order.long().sort().values
    for x in pools:                                     # the pages that are anybody's; no others may change, but those are not all looked at
        x.view(torch.uint8)[:, used] = torch.randint(0, 256, (layers, len(used), page, hkv, d * x.element_size()), generator=g, device="cuda", dtype=torch.uint8)
    before = [x.view(torch.uint8)[:, used].clone() for x in pools]
    scales = {n: 0.005 + 0.02 * torch.rand((layers, hkv), generator=g, device="cuda") for n in ("k_scale", "v_scale")} if kind == "e4m3" else {}
    status = ints([0])
    P.purekv_compact_paged(k, v, idx, types.SimpleNamespace(cu_seqlens=ints(cu)), types.SimpleNamespace(cu_kept=ints(ck)), *pools, table,
                           ints([prefix + m for m in kept]), status=status, **scales)
    assert P.purekv_poll_status(status) == 0
    req = torch.repeat_interleave(torch.arange(len(kept)), torch.tensor(kept)).cuda()
    row = prefix + torch.arange(t, device="cuda") - ints(ck)[req]
    at = torch.searchsorted(used, table[req, row // page].long()), row % page
    src = ints(cu)[req].long() + idx.long()
    for x, was, rows, name in ((pools[0], before[0], k, "k_scale"), (pools[1], before[1], v, "v_scale")):
        have = x.view(torch.uint8)[:, used]
        for layer in range(layers):
            want = torch.stack([rows[layer, src[layer, h], h] for h in range(hkv)], dim=1)
            if kind == "e4m3":
                got = have[layer][at].view(torch.float8_e4m3fn).double()
                value = (want.double() / scales[name][layer].double()[:, None]).clamp(-448, 448)
                assert ((got - value).abs() <= pc.stored_tolerance("e4m3", value, value.abs())).all()
                was[layer][at] = have[layer][at]        # (compared above)
            else:
                was[layer][at] = want.view(torch.uint8)
        assert torch.equal(have, was)


# 444 blocks of 8 warps take 32 rows each of 128 bytes, 16 of 256 or of other sizes, 8 of 512 (as k and v have them): 113 664, 56 832 and 28 416 rows at a time
@pytest.mark.parametrize("kind,d,layers,hkv,kept", [
    ("bf16", 64, 7, 5, [5000, 1, 0, 2777, 4099]), ("bf16", 128, 5, 3, [4001, 333, 5003]), ("fp32", 64, 3, 4, [7001, 5555]), ("fp32", 128, 4, 2, [9001, 0, 300]),
    ("e4m3", 64, 6, 8, [3001, 2999, 17]), ("e4m3", 128, 4, 4, [8191, 1]), ("bf16", 96, 5, 4, [4003, 2222]), ("e4m3", 48, 3, 7, [6007]), ("bf16", 128, 2, 1, [65000]),
])
def test_several_batches_for_every_warp(kind, d, layers, hkv, kept):
    per_pass = 444 * 8 * {128: 32, 512: 8}.get(d * (4 if kind == "fp32" else 2), 16)
    assert layers * hkv * sum(kept) > 2 * per_pass
    check(80, [n + n // 3 + 2 for n in kept], kept, layers, hkv, d, kind, 16, prefix=5)


@pytest.mark.parametrize("kind,n_req", [("bf16", 256), ("bf16", 257), ("e4m3", 900)])
def test_many_requests(kind, n_req):
    kept = [(7 * r) % 40 for r in range(n_req)]
    check(81, [n + 3 for n in kept], kept, 2, 3, 128, kind, 8)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_pools_past_32_bits(kind):
    check(82, [900, 500], [300, 120], 3, 8, 128, kind, 64, n_pages=14000)          # 2.7e9 elements


def test_rows_past_32_bits():
    check(83, [700000, 20000], [3000, 700], 3, 8, 128, "bf16", 64)                 # 2.2e9 elements of k and of v


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("d,rot,interleaved,page,layout", [(128, 128, False, 16, "nhd"), (64, 32, True, 7, "hnd"), (96, 48, False, 64, "nhd")])
def test_prompts_of_several_tokens_a_block(kind, d, rot, interleaved, page, layout):
    # from 593 tokens on a block takes four of them
    check_append(84, [700, 640, 9], [601, 300, 2], 6, 2, d, kind, page, layout, rot=rot, interleaved=interleaved)
    check_append(85, [593], [593], 3, 1, d, kind, page, layout, rot=rot, interleaved=interleaved, with_q=False)


def test_a_token_of_each_of_many_requests():
    check_append(86, [1 + r % 30 for r in range(700)] + [0, 0], [1] * 702, 4, 2, 64, "e4m3", one_each=True)
