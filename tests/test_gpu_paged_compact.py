"""purekv_compact_paged: every kept row in its slot, all layers, and every other slot as it was."""
import types

import pytest
import torch

from paper_2510_25600_b200 import binding as P
from tests import paged_common as pc

pytestmark = pytest.mark.gpu


def check(seed, lens, kept, hkv, d, kind, page=16, layout="nhd", n_layers=2, prefix=0, padding=(), layer_gap=0):
    """`prefix` rows of every request are in the cache before; the requests in `padding` store nothing."""
    g = torch.Generator().manual_seed(seed)
    dtype = "fp32" if kind == "fp32" else "bf16"
    c = pc.Cache(seed, [prefix] * len(lens), hkv, d, kind, page, layout, n_layers, room=max(kept + [1]))
    c.seq_lens = torch.tensor([0 if r in padding else prefix + m for r, m in enumerate(kept)], dtype=torch.int32)
    t, cu, ck = sum(lens), [0], [0]
    for n, m in zip(lens, kept):
        cu.append(cu[-1] + n)
        ck.append(ck[-1] + m)
    store = torch.randn((2, n_layers, t * hkv * d + layer_gap), generator=g).to(pc.TYPES[dtype])
    dev = store.cuda()
    rows = lambda x: x[:, :t * hkv * d].view(n_layers, t, hkv, d)
    k, v = rows(store[0]), rows(store[1])
    idx = torch.zeros((n_layers, hkv, ck[-1]), dtype=torch.int32)
    for layer in range(n_layers):
        for head in range(hkv):
            for r, (n, m) in enumerate(zip(lens, kept)):
                idx[layer, head, ck[r]:ck[r + 1]] = torch.randperm(n, generator=g)[:m].sort().values.to(torch.int32)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    (kp, vp, table, seq_lens), scale = c.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.purekv_compact_paged(rows(dev[0]), rows(dev[1]), idx.cuda(), types.SimpleNamespace(cu_seqlens=i32(cu)), types.SimpleNamespace(cu_kept=i32(ck)), kp, vp, table,
                           seq_lens, status=status, **scale)
    assert P.purekv_poll_status(status) == 0
    bits = lambda x: x.contiguous().view(torch.uint8)
    for got, was, x, sc in ((kp, c.k, k, c.k_scale), (vp, c.v, v, c.v_scale)):
        got, rest = got.cpu(), torch.ones(got.shape[1:3], dtype=torch.bool)
        for r in range(len(lens)):
            for i in range(0 if r in padding else kept[r]):
                at = (c.table[r, (prefix + i) // page], (prefix + i) % page)
                rest[at] = False
                for layer in range(n_layers):
                    src = cu[r] + idx[layer, :, ck[r] + i].long()
                    want = x[layer, src, torch.arange(hkv)]
                    have = got[(layer, *at)]
                    if kind != "e4m3":
                        assert torch.equal(have, want)
                    else:
                        value = (want.double() / sc[layer].double()[:, None]).clamp(-448, 448)
                        assert ((have.double() - value).abs() <= pc.stored_tolerance("e4m3", value, value.abs())).all()
        assert torch.equal(bits(got[:, rest]), bits(was[:, rest]))


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("hkv,d,page,layout", [(2, 128, 16, "nhd"), (4, 64, 7, "nhd"), (1, 128, 1, "hnd"), (3, 96, 64, "hnd"), (5, 16, 16, "nhd")])
def test_layouts(kind, hkv, d, page, layout):
    check(1, [50, 1, 33], [20, 1, 33], hkv, d, kind, page, layout)


def test_behind_a_shared_prefix():
    check(2, [40, 30], [11, 30], 2, 128, "bf16", prefix=21)


def test_requests_that_keep_nothing():
    check(3, [40, 0, 30, 5], [11, 0, 0, 5], 2, 64, "bf16")


def test_padding_stores_nothing():
    check(4, [40, 20, 30], [11, 4, 7], 2, 64, "e4m3", padding=(1,))


def test_layers_apart():
    check(5, [100], [37], 2, 64, "bf16", n_layers=5, layer_gap=64)


def test_many_rows():
    check(6, [900, 400, 1500], [300, 77, 510], 4, 64, "bf16", n_layers=3)


@pytest.mark.parametrize("index", [-1, 40, 2 ** 31 - 1, -2 ** 31])
def test_an_index_outside_its_request_is_left_out(index):
    k = torch.randn((1, 60, 1, 64), dtype=torch.bfloat16, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    idx = i32([[[3, index, 7]]])
    pool = torch.zeros((1, 2, 16, 1, 64), dtype=torch.bfloat16, device="cuda")
    v_pool, status = pool.clone(), i32([0])
    P.purekv_compact_paged(k, k, idx, types.SimpleNamespace(cu_seqlens=i32([0, 40])), types.SimpleNamespace(cu_kept=i32([0, 3])), pool, v_pool, i32([[1]]), i32([3]),
                           status=status)
    with pytest.raises(P.PureKVError) as e:
        P.purekv_poll_status(status)
    assert e.value.status == P.ERR_BAD_PAGE
    want = torch.zeros_like(pool)
    want[0, 1, 0], want[0, 1, 2] = k[0, 3], k[0, 7]
    assert torch.equal(pool, want) and torch.equal(v_pool, want)
