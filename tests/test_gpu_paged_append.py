"""purekv_append_paged against its definition in 64 bits: rotations, axes, layouts, types, ragged and padded batches; what it must not
touch; pages that do not exist."""
import pytest
import torch

from paper_2510_25600_b200 import binding as P
from tests import paged_common as pc

pytestmark = pytest.mark.gpu


def frequencies(rot, theta=10000.0):
    return theta ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))


def check(seed, lens, new, H, hkv, d, kind, page=16, layout="nhd", rot=None, sections=None, interleaved=False, far=0, one_each=False, with_q=True, scales=True,
          extra=0, head_major=False):
    """Requests of `lens` rows in the end, `new` of them new; `extra` tokens behind the last request's."""
    g = torch.Generator().manual_seed(seed)
    dtype = "fp32" if kind == "fp32" else "bf16"
    before = [max(0, n - m) for n, m in zip(lens, new)]
    c = pc.Cache(seed, before, hkv, d, kind, page, layout, room=max(new + [1]), scales=scales)
    c.seq_lens = torch.tensor(lens, dtype=torch.int32)
    t, rot = sum(new) + extra, d if rot is None else rot
    qkv = torch.randn((t, H + 2 * hkv, d), generator=g).to(pc.TYPES[dtype])
    if head_major:
        qkv = qkv.transpose(0, 1).contiguous().transpose(0, 1)
    dev = qkv.cuda() if not head_major else qkv.transpose(0, 1).contiguous().cuda().transpose(0, 1)
    q, k, v = dev[:, :H], dev[:, H:H + hkv], dev[:, H + hkv:]
    axes = sections or (rot // 2,)
    pos = torch.randint(0, 5000, (len(axes), t), generator=g, dtype=torch.int32) + far
    inv = frequencies(rot) if rot else None
    (kp, vp, table, seq_lens), scale = c.cuda()
    cu = torch.tensor([0] + list(torch.tensor(new).cumsum(0)), dtype=torch.int32)
    rope = dict(positions=(pos if sections else pos[0]).cuda(), inv_freq=inv.cuda(), sections=sections, interleaved=interleaved) if rot else {}
    k_out = torch.full((t, hkv, d), float("nan"), dtype=pc.TYPES[dtype], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = P.purekv_append_paged(k, v, kp, vp, table, seq_lens, None if one_each else cu.cuda(), q=q if with_q else None, k_out=k_out, status=status, **rope, **scale)
    assert P.purekv_poll_status(status) == 0
    angle = pc.angles(pos, inv, axes) if rot else torch.zeros((t, 0)).double()
    for got, x in ([(q_out, qkv[:, :H])] if with_q else []) + [(k_out, qkv[:, H:H + hkv])]:
        want, size = pc.rotate(x, angle, interleaved)
        got = got.cpu().double()
        if not rot:
            assert torch.equal(got, want)
        assert ((got - want).abs() <= pc.stored_tolerance(dtype, want, size)).all()
        assert torch.equal(got[..., rot:], want[..., rot:])
    # the pages: the new rows, and every other slot as it was, to the bit
    bits = lambda x: x.contiguous().view(torch.uint8)
    for got, was, x, sc, turned in ((kp, c.k, qkv[:, H:H + hkv], c.k_scale, True), (vp, c.v, qkv[:, H + hkv:], c.v_scale, False)):
        got = got.cpu()
        rest = torch.ones(got.shape[:2], dtype=torch.bool)
        want, size = pc.rotate(x, angle, interleaved) if turned else (x.double(), x.double().abs() * 0)
        for r, (n, m) in enumerate(zip(lens, new)):
            for i in range(m if n > 0 else 0):
                s, tok = n - m + i, int(cu[r]) + i
                at = (c.table[r, s // page], s % page)
                rest[at] = False
                value = want[tok] if sc is None else (want[tok] / sc.double()[:, None]).clamp(-448, 448)
                units = size[tok] if sc is None else size[tok] / sc.double()[:, None]
                tol = pc.stored_tolerance(kind, value, units)
                if not turned and kind != "e4m3":
                    assert torch.equal(got[at].double(), value)
                assert ((got[at].double() - value).abs() <= tol).all(), (r, i)
        assert torch.equal(bits(got[rest]), bits(was[rest]))


@pytest.mark.parametrize("kind", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("d,rot,interleaved", [(128, 128, False), (128, 128, True), (64, 64, False), (64, 32, False), (128, 48, True), (96, 96, False), (16, 16, True), (256, 64, False), (128, 0, False)])
def test_rotations(kind, d, rot, interleaved):
    check(1, [40, 7, 33], [9, 7, 1], 6, 2, d, kind, rot=rot, interleaved=interleaved)


@pytest.mark.parametrize("sections", [(16, 24, 24), (64,), (1, 62, 1), (0, 64), (16, 16, 16, 16)])
def test_axes_of_positions(sections):
    check(2, [20, 30], [20, 3], 4, 4, 128, "bf16", sections=sections)


@pytest.mark.parametrize("far", [-3000, 1 << 20, 1 << 24, (1 << 31) - 6000])
def test_far_positions_keep_their_fraction_of_a_turn(far):
    check(3, [5], [5], 2, 1, 64, "fp32", far=far)


@pytest.mark.parametrize("page,layout", [(1, "nhd"), (7, "nhd"), (16, "hnd"), (100, "hnd"), (128, "nhd")])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_pages(page, layout, kind):
    check(4, [130, 1, 64, 65], [61, 1, 64, 2], 5, 5, 64, kind, page=page, layout=layout)


@pytest.mark.parametrize("H,hkv", [(1, 1), (28, 4), (32, 8), (71, 1), (3, 3)])
def test_heads(H, hkv):
    check(5, [12, 3], [5, 3], H, hkv, 128, "bf16")


@pytest.mark.parametrize("n_req", [1, 2, 33, 300])
def test_one_token_each(n_req):
    check(6, [1 + (7 * r) % 50 for r in range(n_req)], [1] * n_req, 4, 2, 64, "bf16", one_each=True)


def test_padding_of_a_batch_is_rotated_and_stored_nowhere():
    check(7, [9, 0, 4, 0, 0], [1] * 5, 4, 2, 128, "e4m3", one_each=True)
    check(8, [9, 0, 4, 0], [2, 3, 1, 0], 4, 2, 128, "bf16", extra=5)      # and tokens past the last request's


def test_requests_without_new_tokens():
    check(9, [9, 8, 0, 7], [0, 3, 0, 0], 4, 2, 128, "bf16")


def test_prompts_of_many_tokens():
    check(10, [700, 1200], [700, 900], 4, 2, 64, "bf16")                  # the form of several tokens a block, one of them short
    check(11, [1190], [1187], 2, 1, 64, "fp32", interleaved=True)


def test_layouts_of_the_projection():
    check(12, [40], [40], 4, 2, 64, "bf16", head_major=True)
    check(13, [40], [40], 4, 2, 64, "bf16", with_q=False)


def test_no_scales_mean_one():
    check(14, [40], [40], 4, 2, 64, "e4m3", scales=False)


def test_in_place():
    x = torch.randn((7, 4, 64), dtype=torch.bfloat16, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    pos, inv = torch.arange(7, dtype=torch.int32, device="cuda"), frequencies(64).cuda()
    want = P.purekv_append_paged(None, None, None, None, None, None, q=x, positions=pos, inv_freq=inv)
    k = x.clone()
    P.purekv_append_paged(k, None, None, None, None, None, q=x, q_out=x, k_out=k, positions=pos, inv_freq=inv)
    assert torch.equal(x, want) and torch.equal(k, want)


def test_values_at_the_ends_of_the_eight_bit_range():
    # values beyond +-448 scales, infinities and NaN; ties go to even: 17 and 19 lie between 16, 18 and 20
    x = torch.tensor([448.0, -448.0, 449.0, 1e30, float("inf"), float("-inf"), float("nan"), 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 0.0], dtype=torch.bfloat16)
    want = torch.tensor([448.0, -448.0, 448.0, 448.0, 448.0, -448.0, float("nan"), 16.0, 20.0, 0.0, 2.0 ** -8, 0.0])
    k = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    k[0, 0, :12] = x
    c = pc.Cache(1, [0], 1, 64, "e4m3", room=1, scales=False)
    c.seq_lens = torch.tensor([1], dtype=torch.int32)
    (kp, vp, table, lens), _ = c.cuda()
    P.purekv_append_paged(k.cuda(), k.cuda(), kp, vp, table, lens)
    for pool in (kp, vp):
        assert torch.allclose(pool.cpu()[c.table[0, 0], 0, 0, :12].float(), want, rtol=0, atol=0, equal_nan=True)


@pytest.mark.parametrize("table,lens", [([[9, 1]], [16]), ([[-1, 1]], [16]), ([[0, 1]], [33]), ([[0, 1]], [2]), ([[0, 2 ** 31 - 1]], [18])])
def test_rows_that_have_no_place(table, lens):
    """A page outside the pool, or more rows than the list holds, or fewer rows than there are new ones: they are left out and the
    status word says so; the others are stored."""
    n_pages, page, new = 4, 16, 4
    pool = torch.zeros((n_pages, page, 1, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.randn((new, 1, 64), dtype=torch.bfloat16, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    v_pool = pool.clone()
    P.purekv_append_paged(k, k, pool, v_pool, torch.tensor(table, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                          torch.tensor([0, new], dtype=torch.int32, device="cuda"), status=status)
    with pytest.raises(P.PureKVError) as e:
        P.purekv_poll_status(status)
    assert e.value.status == P.ERR_BAD_PAGE
    want = torch.zeros_like(pool)
    for i in range(new):
        s = lens[0] - new + i
        if 0 <= s < 2 * page and 0 <= table[0][s // page] < n_pages:
            want[table[0][s // page], s % page] = k[i]
    assert torch.equal(pool, want) and torch.equal(v_pool, want)


def test_the_library_keeps_a_word_of_its_own():
    pool = torch.zeros((1, 16, 1, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    one = torch.ones((1, 1), dtype=torch.int32, device="cuda")
    P.purekv_append_paged(k, k, pool, pool, one, one[0])            # page 1 of one
    with pytest.raises(P.PureKVError):
        P.purekv_poll_status(None)
    assert P.purekv_poll_status(None) == 0                            # read once, cleared


def test_rows_past_32_bits():
    n_pages = 17000                                                    # 2^31 elements are 16384 pages of 128 x 8 x 128
    pool = torch.empty((n_pages, 128, 8, 128), dtype=torch.bfloat16, device="cuda")
    v_pool = torch.empty_like(pool)
    k = torch.randn((2, 16, 128), dtype=torch.bfloat16, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    table = torch.tensor([[n_pages - 1], [3]], dtype=torch.int32, device="cuda")
    P.purekv_append_paged(k[:, :8], k[:, 8:], pool, v_pool, table, torch.tensor([128, 5], dtype=torch.int32, device="cuda"))
    assert P.purekv_poll_status(None) == 0
    for x, y in ((pool, k[:, :8]), (v_pool, k[:, 8:])):
        assert torch.equal(x[n_pages - 1, 127], y[0]) and torch.equal(x[3, 4], y[1])
