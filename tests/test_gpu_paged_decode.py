"""purekv_decode_paged against attention in 64 bits: types, heads, lengths, pages, strides, hints; rows it must not read; padding;
pages that do not exist; streams, captures and two calls at once."""
import pytest
import torch

from paper_2510_25600_b200 import binding as P
from tests import paged_common as pc

pytestmark = pytest.mark.gpu


def queries(seed, n, H, d, kind):
    return (1.5 * torch.randn((n, H, d), generator=torch.Generator().manual_seed(seed + 1000))).to(torch.float32 if kind == "fp32" else torch.bfloat16)


def compare(c, q, got, lse, scale=None, only=None, layer=None):
    kind, dtype = c.kind, "fp32" if c.kind == "fp32" else "bf16"
    got, lse = got.cpu().double(), lse.cpu().double()
    for r in range(len(c.lens)) if only is None else only:
        k, v = c.rows(r, "k", layer), c.rows(r, "v", layer)
        o, z, weight, size = pc.attention(q[r].double(), k, v, scale)
        if not k.shape[0]:
            assert (got[r] == 0).all() and torch.isneginf(lse[r]).all()
            continue
        assert ((got[r] - o).abs() <= pc.attention_tolerance(dtype, kind, o, weight, size, c.d)).all(), (r, float((got[r] - o).abs().max()))
        assert ((lse[r] - z).abs() <= pc.lse_tolerance(z, size, c.d)).all(), (r, float((lse[r] - z).abs().max()))


def check(seed, lens, H, hkv, d, kind="bf16", page=16, layout="nhd", max_len=None, scale=0.0, scales=True, strided=False):
    c = pc.Cache(seed, lens, hkv, d, kind, page, layout, scales=scales)
    q = queries(seed, len(lens), H, d, kind)
    (kp, vp, table, seq_lens), sc = c.cuda()
    dq = q.cuda()
    if strided:                                      # the q part of a projection's output
        whole = torch.full((len(lens), H + 2 * hkv, d), float("nan"), dtype=q.dtype, device="cuda")
        whole[:, :H] = dq
        dq = whole[:, :H]
    out, lse = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda"), torch.full((len(lens), H), float("nan"), device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for hint in ([0, 1, max(lens + [1])] if max_len is None else [max_len]):
        got = P.purekv_decode_paged(dq, kp, vp, table, seq_lens, max_len=hint, out=out.fill_(float("nan")), lse=lse.fill_(float("nan")), softmax_scale=scale, status=status, **sc)
        assert got is out and P.purekv_poll_status(status) == 0
        compare(c, q, out, lse, scale)


LENS = [0, 1, 5, 16, 17, 64, 130, 700, 1999, 3]


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("H,hkv,d", [(4, 4, 128), (8, 4, 64), (28, 4, 128), (32, 8, 64), (16, 1, 128), (12, 1, 64), (3, 1, 128), (7, 7, 64)])
def test_heads(kind, H, hkv, d):
    check(1, LENS, H, hkv, d, kind)


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("H,hkv", [(17, 1), (40, 2), (71, 1), (128, 2)])
def test_many_queries_per_kv_head(kind, H, hkv):
    check(2, [0, 33, 257], H, hkv, 128, kind)


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("page,layout", [(1, "nhd"), (2, "hnd"), (7, "nhd"), (16, "hnd"), (48, "nhd"), (100, "hnd"), (128, "nhd"), (5000, "nhd")])
def test_pages(kind, page, layout):
    check(3, [0, 1, 15, 99, 100, 101, 640], 6, 2, 64, kind, page, layout)


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [8, 16, 24, 32, 64])
def test_pages_of_a_few_rows(kind, d, page):
    check(3, [0, 7, 8, 9, 33, 100, 640, 1], 9, 3, d, kind, page, "nhd" if page % 16 else "hnd")
    check(3, [65, 2, 200], 16, 1, d, kind, page)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[9000], [5000, 3, 0, 2, 7000], [8191, 8192, 8193], [40] * 60 + [9001] + [0] * 9])
def test_long_requests(kind, lens):
    check(4, lens, 8, 2, 128, kind, 64)


def test_long_fp32_requests():
    check(4, [9000, 0, 3, 4097], 4, 2, 64, "fp32", 32)


def test_many_requests():
    g = torch.Generator().manual_seed(6)
    check(5, torch.randint(0, 60, (400,), generator=g).tolist(), 8, 2, 64, "bf16", 16)
    check(6, torch.randint(0, 300, (150,), generator=g).tolist(), 4, 4, 128, "e4m3", 16)


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("H,hkv,d,page", [(8, 2, 128, 16), (24, 2, 64, 7)])
def test_every_way_of_launching(kind, H, hkv, d, page):
    """What is expected to be the longest request sizes the launch, whatever the lengths are: few and many requests, each form of both."""
    g = torch.Generator().manual_seed(30)
    for lens in (torch.randint(0, 300, (80,), generator=g).tolist(), [700, 0, 3, 64], [129]):
        c = pc.Cache(30, lens, hkv, d, kind, page)
        q = queries(30, len(lens), H, d, kind)
        (kp, vp, table, seq_lens), sc = c.cuda()
        dq, lse = q.cuda(), torch.empty((len(lens), H), device="cuda")
        want = None
        for hint in (0, 1, 64, 65, 128, 129, 256, 257, 600, 2048, 2049, 9000, 1 << 17, (1 << 31) - 1):
            got = P.purekv_decode_paged(dq, kp, vp, table, seq_lens, max_len=hint, out=torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda"), lse=lse.fill_(float("nan")), **sc)
            if want is None:
                want = got.float()
                compare(c, q, got, lse)
            else:                                  # two results within the tolerance of the same: compared with twice the weights' bound
                assert ((got.float() - want).abs() <= 2.0 ** -6 * want.abs() + 2.0 ** -6).all(), hint
        compare(c, q, got, lse)


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("d,n", [(64, 40), (128, 3000)])
def test_many_keys_of_little_weight(kind, d, n):
    # one key has nearly all the weight, its values are 0: what comes out is the others', of 2^-26 of its weight each
    c = pc.Cache(31, [n, 1], 2, d, kind, scales=False)
    q = torch.ones((2, 8, d), dtype=torch.float32 if kind == "fp32" else torch.bfloat16)
    for s in range(n):
        c.k[c.table[0, s // c.page], s % c.page] = torch.tensor(2.25 if s == 7 else 0.0).to(c.k.dtype)
        c.v[c.table[0, s // c.page], s % c.page] = torch.tensor(0.0 if s == 7 else 448.0).to(c.v.dtype)
    (kp, vp, table, lens), sc = c.cuda()
    lse = torch.empty((2, 8), device="cuda")
    for hint in (0, 1, n, 9000):
        got = P.purekv_decode_paged(q.cuda(), kp, vp, table, lens, max_len=hint, lse=lse, softmax_scale=8.0 / d, **sc)
        compare(c, q, got, lse, 8.0 / d)


@pytest.mark.parametrize("n", [1, 2, 3, 5, 8, 13, 21, 40, 70, 110])
def test_lengths_one_by_one(n):
    check(7, list(range(n, n + 8)), 5, 1, 128, "bf16", 8, max_len=0)


@pytest.mark.parametrize("n_req,rows", [(1, 300), (1, 1700), (2, 900), (9, 400), (40, 250)])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "fp32"])
def test_even_batches(kind, n_req, rows):
    check(8, [rows - r for r in range(n_req)], 14, 2, 128, kind, 32)


def test_scale_of_the_softmax_and_no_scales():
    check(9, [50, 300], 8, 2, 128, "bf16", scale=0.03)
    check(10, [50, 300], 8, 2, 128, "e4m3", scale=0.2, scales=False)


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
def test_queries_out_of_a_projection(kind):
    check(11, [5, 300, 0, 77], 6, 2, 128, kind, strided=True)


@pytest.mark.parametrize("kind,size", [("bf16", 40.0), ("fp32", 40.0), ("e4m3", 40.0), ("e4m3", 1e-3), ("bf16", 1e-3)])
def test_extreme_logits(kind, size):
    c = pc.Cache(12, [900, 40], 2, 128, kind)
    q = (queries(12, 2, 8, 128, kind).float() * size).to(torch.float32 if kind == "fp32" else torch.bfloat16)
    (kp, vp, table, lens), sc = c.cuda()
    lse = torch.empty((2, 8), device="cuda")
    got = P.purekv_decode_paged(q.cuda(), kp, vp, table, lens, lse=lse, **sc)
    compare(c, q, got, lse)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_queries_of_a_wide_range(kind):
    # heads whose elements differ by powers of two far beyond what 16 bits of a fraction hold
    c = pc.Cache(13, [300, 20], 2, 128, kind)
    q = queries(13, 2, 8, 128, kind)
    q[:, :, ::7] *= 2.0 ** -30
    q[:, 1] *= 2.0 ** -60
    q[:, 2, 5] = 0
    q[:, 3] = 0
    (kp, vp, table, lens), sc = c.cuda()
    lse = torch.empty((2, 8), device="cuda")
    compare(c, q, P.purekv_decode_paged(q.cuda(), kp, vp, table, lens, lse=lse, **sc), lse)


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
def test_non_finite_rows(kind):
    """A NaN among a head's keys or values reaches that head's result and no other; a key of -inf logit weighs nothing."""
    c = pc.Cache(14, [200, 200, 200], 2, 64, kind, page=16, scales=False)
    at = lambda r, s: (c.table[r, s // 16], s % 16)
    c.k[(*at(0, 150), 0)] = torch.full((64,), float("nan")).to(c.k.dtype)
    c.v[(*at(1, 37), 1)] = torch.full((64,), float("nan")).to(c.v.dtype)
    q = queries(14, 3, 4, 64, kind)
    if kind != "e4m3":
        q[2, 0, 0] = 1.0
        c.k[(*at(2, 99), 0)] = torch.tensor([float("-inf")] + [0.0] * 63).to(c.k.dtype)
        q[2, 1, 0] = 2.0
    (kp, vp, table, lens), sc = c.cuda()
    lse = torch.empty((3, 4), device="cuda")
    got = P.purekv_decode_paged(q.cuda(), kp, vp, table, lens, lse=lse, **sc).cpu()
    assert torch.isnan(got[0, :2]).all() and torch.isnan(lse[0, :2]).all() and torch.isnan(got[1, 2:]).all()
    assert torch.isfinite(got[0, 2:]).all() and torch.isfinite(got[1, :2]).all() and torch.isfinite(lse[1]).all()
    compare(c, q, got, lse, only=[2])


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_pages_and_rows_that_do_not_exist_are_left_out(kind, d):
    c = pc.Cache(15, [100, 100, 60], 2, d, kind, page=16)
    q = queries(15, 3, 4, d, kind)
    (kp, vp, table, lens), sc = c.cuda()
    table[0, 2] = kp.shape[0]               # rows 32-47 of request 0
    table[1, 6] = -5                        # rows 96-99 of request 1
    lens[2] = 2 ** 31 - 1                   # request 2: more rows than its list holds
    table[2, 4:] = 2 ** 31 - 1
    status, lse = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty((3, 4), device="cuda")
    for hint in (0, 1, 1 << 20):
        status.zero_()
        got = P.purekv_decode_paged(q.cuda(), kp, vp, table, lens, max_len=hint, lse=lse, status=status, **sc)
        with pytest.raises(P.PureKVError) as e:
            P.purekv_poll_status(status)
        assert e.value.status == P.ERR_BAD_PAGE
        keep = {0: [s for s in range(100) if not 32 <= s < 48], 1: list(range(96)), 2: list(range(64))}
        c.lens[2] = 60
        for r, rows in keep.items():
            if r == 2:
                continue                     # its last page holds slots that nobody wrote (NaN here)
            o, z, weight, size = pc.attention(q[r].double(), c.rows(r, "k")[rows], c.rows(r, "v")[rows])
            dtype = "fp32" if kind == "fp32" else "bf16"
            assert ((got[r].cpu().double() - o).abs() <= pc.attention_tolerance(dtype, kind, o, weight, size, d)).all()
            assert ((lse[r].cpu().double() - z).abs() <= pc.lse_tolerance(z, size, d)).all()


def test_a_request_of_missing_pages_alone():
    c = pc.Cache(16, [40, 40], 1, 64, "bf16")
    (kp, vp, table, lens), _ = c.cuda()
    table[0] = -1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = queries(16, 2, 2, 64, "bf16")
    lse = torch.empty((2, 2), device="cuda")
    got = P.purekv_decode_paged(q.cuda(), kp, vp, table, lens, lse=lse, status=status)
    assert status.item() == P.ERR_BAD_PAGE
    compare(c, q, got, lse, only=[1])


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_rows_past_32_bits(kind):
    n_pages = 17000 if kind == "bf16" else 34000        # 2^32 bytes and more
    pool = [torch.empty((n_pages, 128, 8, 128), dtype=pc.TYPES[kind], device="cuda") for _ in "kv"]
    c = pc.Cache(17, [300, 200], 8, 128, kind, page=128)
    (kp, vp, table, lens), sc = c.cuda()
    far = n_pages - 1 - torch.arange(kp.shape[0], device="cuda")
    for big, small in zip(pool, (kp, vp)):
        big.view(torch.uint8)[far] = small.view(torch.uint8)
    moved = torch.where(table >= 0, n_pages - 1 - table, table)
    q = queries(17, 2, 16, 128, kind)
    lse = torch.empty((2, 16), device="cuda")
    compare(c, q, P.purekv_decode_paged(q.cuda(), *pool, moved, lens, lse=lse, **sc), lse)


def test_twice_the_same_to_the_bit():
    for kind, lens in (("bf16", [9000, 30, 4000, 0, 700]), ("e4m3", [200] * 50), ("fp32", [900, 4000])):
        c = pc.Cache(18, lens, 2, 128, kind)
        q = queries(18, len(lens), 8, 128, kind).cuda()
        (kp, vp, table, seq_lens), sc = c.cuda()
        a, b = (P.purekv_decode_paged(q, kp, vp, table, seq_lens, **sc) for _ in range(2))
        assert torch.equal(a, b)


def test_output_over_the_queries():
    c = pc.Cache(19, [300, 20, 0, 2500], 2, 128, "bf16")
    q = queries(19, 4, 8, 128, "bf16")
    (kp, vp, table, lens), _ = c.cuda()
    want = P.purekv_decode_paged(q.cuda(), kp, vp, table, lens)
    dq = q.cuda()
    for hint in (0, 2500):
        x = dq.clone()
        P.purekv_decode_paged(x, kp, vp, table, lens, max_len=hint, out=x)
        tol = 2.0 ** -7 * want.float().abs() + 2.0 ** -7          # two ways of splitting the work at most: each within its tolerance
        assert ((x.float() - want.float()).abs() <= tol).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "fp32"])
def test_captured_and_replayed_with_other_lengths(kind):
    """A captured step follows the lengths and the table that lie in device memory when it is replayed."""
    lens = [100, 3000, 1, 0]
    c = pc.Cache(20, lens, 2, 64, kind)
    q = queries(20, 4, 4, 64, kind)
    (kp, vp, table, seq_lens), sc = c.cuda()
    dq, lse, out = q.cuda(), torch.empty((4, 4), device="cuda"), torch.empty(q.shape, dtype=q.dtype, device="cuda")
    ws = torch.empty(max(16, P.purekv_decode_paged_ws_bytes(4, 0, 4, 2, 64, P.FP32 if kind == "fp32" else P.BF16)), dtype=torch.uint8, device="cuda")
    step = lambda: P.purekv_decode_paged(dq, kp, vp, table, seq_lens, out=out, lse=lse, ws=ws, **sc)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
        step()
    for other in (lens, [1, 17, 1, 0], [99, 2999, 0, 0], [0, 0, 0, 0]):
        seq_lens.copy_(torch.tensor(other, dtype=torch.int32))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        c.lens = list(other)
        compare(c, q, out, lse)


def test_two_streams_at_once():
    runs = []
    for seed, kind, lens in ((21, "bf16", [5000, 200, 0, 9000]), (22, "e4m3", [300] * 40)):
        c = pc.Cache(seed, lens, 4, 128, kind, 64)
        q = queries(seed, len(lens), 16, 128, kind)
        runs.append((c, q, q.cuda(), *c.cuda(), torch.cuda.Stream(), torch.empty((len(lens), 16), device="cuda")))
    torch.cuda.synchronize()
    outs = [None, None]
    for _ in range(20):
        for i, (c, q, dq, cache, sc, stream, lse) in enumerate(runs):
            with torch.cuda.stream(stream):
                outs[i] = P.purekv_decode_paged(dq, *cache, lse=lse, **sc)
    torch.cuda.synchronize()
    for (c, q, dq, cache, sc, stream, lse), out in zip(runs, outs):
        compare(c, q, out, lse)


def test_nothing_is_written_around_the_outputs():
    c = pc.Cache(23, [300, 20, 0], 2, 64, "bf16")
    q = queries(23, 3, 6, 64, "bf16").cuda()
    (kp, vp, table, lens), _ = c.cuda()
    guard = torch.full((3 * 6 * 64 + 128,), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((3 * 6 + 16,), 7.0, device="cuda")
    before = kp.clone(), vp.clone()
    for hint in (0, 300):
        P.purekv_decode_paged(q, kp, vp, table, lens, max_len=hint, out=guard[64:-64].view(3, 6, 64), lse=lse[8:-8].view(3, 6))
        assert (guard[:64] == 7).all() and (guard[-64:] == 7).all() and (lse[:8] == 7).all() and (lse[-8:] == 7).all()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, (kp, vp)))


def test_nothing_to_do():
    c = pc.Cache(24, [], 2, 64, "bf16", spare_pages=2)
    (kp, vp, table, lens), _ = c.cuda()
    empty = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    assert P.purekv_decode_paged(empty, kp, vp, table, lens).shape == (0, 4, 64)
    P.purekv_append_paged(empty[:, :2], empty[:, :2], kp, vp, table, lens)
    cu = torch.zeros(1, dtype=torch.int32, device="cuda")
    holder = type("H", (), dict(cu_seqlens=cu, cu_kept=cu))
    P.purekv_compact_paged(empty[None, :, :2], empty[None, :, :2], torch.zeros((1, 2, 0), dtype=torch.int32, device="cuda"), holder, holder, kp[None], vp[None], table, lens)
    assert P.purekv_poll_status(None) == 0


def test_a_list_without_pages():
    # no column in the table, and no page in the pool: every row is missing, nothing is read
    q = queries(25, 2, 4, 64, "bf16").cuda()
    lens = torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    for n_pages, columns in ((2, 0), (0, 2)):
        pool = torch.zeros((n_pages, 16, 2, 64), dtype=torch.bfloat16, device="cuda")
        for hint in (0, 3):
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            out = P.purekv_decode_paged(q, pool, pool, torch.zeros((2, columns), dtype=torch.int32, device="cuda"), lens, max_len=hint, status=status)
            assert status.item() == P.ERR_BAD_PAGE and (out[1] == 0).all()


def test_pools_that_lie_in_one_tensor():
    # K and V pages side by side, and a window of a larger pool
    c = pc.Cache(26, [700, 33, 0, 1500], 4, 128, "bf16", 16)
    q = queries(26, 4, 16, 128, "bf16")
    both = torch.full((c.k.shape[0], 2, 16, 6, 128), float("nan"), dtype=torch.bfloat16)
    both[:, 0, :, 1:5], both[:, 1, :, 1:5] = c.k, c.v
    both = both.cuda()
    (_, _, table, lens), _ = c.cuda()
    lse = torch.empty((4, 16), device="cuda")
    for hint in (0, 1500):
        compare(c, q, P.purekv_decode_paged(q.cuda(), both[:, 0, :, 1:5], both[:, 1, :, 1:5], table, lens, max_len=hint, lse=lse), lse)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "fp32"])
def test_uninitialised_workspaces(kind):
    c = pc.Cache(27, [3000, 1, 0, 900], 2, 64, kind, 16)
    q = queries(27, 4, 8, 64, kind)
    (kp, vp, table, lens), sc = c.cuda()
    need = P.purekv_decode_paged_ws_bytes(4, 0, 8, 2, 64, P.FP32 if kind == "fp32" else P.BF16)
    lse = torch.empty((4, 8), device="cuda")
    for fill in (0xff, 0x7f, 0x01):
        ws = torch.full((need + 64,), fill, dtype=torch.uint8, device="cuda")
        compare(c, q, P.purekv_decode_paged(q.cuda(), kp, vp, table, lens, lse=lse, ws=ws[:need], **sc), lse)
        assert (ws[need:] == fill).all()
    with pytest.raises(P.PureKVError) as e:
        P.purekv_decode_paged(q.cuda(), kp, vp, table, lens, ws=torch.empty(100, dtype=torch.uint8, device="cuda"), **sc)
    assert e.value.status == P.ERR_WORKSPACE


@pytest.mark.parametrize("hint", [0, 2000])
def test_two_graphs_that_share_a_workspace(hint):
    made = []
    ws = torch.empty(P.purekv_decode_paged_ws_bytes(4, 0, 8, 2, 128), dtype=torch.uint8, device="cuda")
    for seed, lens in ((28, [2000, 7, 0, 1000]), (29, [5, 1999, 300, 64])):
        c = pc.Cache(seed, lens, 2, 128, "bf16", 16)
        q = queries(seed, 4, 8, 128, "bf16")
        (kp, vp, table, seq), _ = c.cuda()
        dq, lse, out = q.cuda(), torch.empty((4, 8), device="cuda"), torch.empty(q.shape, dtype=q.dtype, device="cuda")
        call = lambda a=(dq, kp, vp, table, seq), o=out, z=lse: P.purekv_decode_paged(*a, max_len=hint, out=o, lse=z, ws=ws)
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        made.append((c, q, out, lse, graph, dq, kp, vp, table, seq))
    for _ in range(3):
        for m in made:
            m[2].fill_(float("nan"))
            m[4].replay()
    torch.cuda.synchronize()
    for m in made:
        compare(m[0], m[1], m[2], m[3])
