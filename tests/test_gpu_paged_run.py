"""The paged cache as it is used: rotation, prefill, scores, selection, compaction into pages, then steps of append and attention; checked
stage by stage against 64 bits on what the stage before left."""
import numpy as np
import pytest
import torch

from paper_2510_25600_b200 import binding as P
from paper_2510_25600_b200 import inputs
from paper_2510_25600_b200.paged import PagedCache
from paper_2510_25600_b200.pipeline import PureKVPipeline
from tests import paged_common as pc

pytestmark = pytest.mark.gpu

THETA = 10000.0


def conversation(kind, d, H, hkv, sections, seed=0):
    """A prompt of three requests through the pipeline into pages.  Returns the cache and what was kept, layer by layer."""
    dtype = torch.float32 if kind == "fp32" else torch.bfloat16
    g = torch.Generator("cuda").manual_seed(seed)
    batch = inputs.make_batch([5, 0, 9], [3, 2, 4], [20, 33, 7], 6, 7)
    layers, t = 3, batch.total_tokens
    rows = lambda heads: torch.randn((layers, t, heads, d), generator=g, device="cuda").to(dtype)
    q, k, v = rows(H), rows(hkv), rows(hkv)
    pos = torch.randint(0, 400, (len(sections), t), generator=g, device="cuda", dtype=torch.int32)
    inv = (THETA ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).cuda()
    for layer in range(layers):
        P.purekv_append_paged(k[layer], None, None, None, None, None, q=q[layer], q_out=q[layer], k_out=k[layer], positions=pos, inv_freq=inv, sections=sections)
    pipe = PureKVPipeline(batch.seq_lens, batch.n_prefix, batch.n_frames, inputs.STMask(6, 7, tile=16 if kind == "fp32" else 64), layers, H, hkv, d, dtype, (0,), (1, 2), 16, 0.3)
    scale = None
    if kind == "e4m3":
        scale = [(0.01 + 0.01 * torch.rand((2, hkv), generator=g, device="cuda")) for _ in "kv"]
    cache = PagedCache(2, 80, 8, hkv, d, pc.TYPES[kind], 5, 200, *(scale or (None, None)))
    cache.set_rows([0, 3, 0])                              # request 1 has three rows of its own before
    for x in (cache.k, cache.v):
        x.view(torch.uint8)[:] = 0x11
    pipe.run_device(q, k, v, pages=cache)
    pipe.check_status()
    cache.check_status()
    return cache, pipe, k, v, inv, g, dtype


def held(cache, pool, r, layer):
    n = int(cache.h_lens[r])
    x = torch.stack([pool[layer, cache.block_table[r, s // 8].item(), s % 8].double() for s in range(n)]).cpu() if n else torch.zeros((0, *pool.shape[3:])).double()
    scale = cache.k_scale if pool is cache.k else cache.v_scale
    return x if scale is None else x * scale[layer].cpu().double()[:, None]


@pytest.mark.parametrize("kind,d,H,hkv,sections", [("bf16", 128, 8, 2, (16, 24, 24)), ("bf16", 64, 7, 1, (32,)), ("fp32", 64, 4, 2, (32,)), ("e4m3", 128, 6, 2, (64,))])
def test_from_a_prompt_to_its_tokens(kind, d, H, hkv, sections):
    cache, pipe, k, v, inv, g, dtype = conversation(kind, d, H, hkv, sections)
    batch, kept = pipe.batch, np.diff(pipe.budget.h_cu_kept)
    assert cache.h_lens[:3].tolist() == [kept[0], kept[1] + 3, kept[2]]
    name = "fp32" if kind == "fp32" else "bf16"
    # the survivors lie in their rows
    for r in range(3):
        for layer in range(2):
            idx = pipe.idx[layer, :, pipe.budget.h_cu_kept[r]:pipe.budget.h_cu_kept[r + 1]].long() + int(batch.h_cu[r])
            for pool, x, sc in ((cache.k, k, cache.k_scale), (cache.v, v, cache.v_scale)):
                want = torch.stack([x[layer + 1, idx[head], head] for head in range(hkv)], dim=1).cpu().double()
                got = held(cache, pool, r, layer)[3 if r == 1 else 0:]
                if kind != "e4m3":
                    assert torch.equal(got, want)
                else:
                    units = sc[layer].cpu().double()[:, None]
                    value = (want / units).clamp(-448, 448)
                    assert ((got / units - value).abs() <= pc.stored_tolerance("e4m3", value, value.abs()) + 1e-6 * value.abs()).all()
    # three steps, the second without request 2; conversations 3 and 4 are padding all the while
    for step in range(3):
        new = [1, 1, 0 if step == 1 else 1, 0, 0]
        before = cache.h_lens.copy()
        cache.advance(new)
        active = torch.tensor(new)
        qkv = torch.randn((5, H + 2 * hkv, d), generator=g, device="cuda").to(dtype)
        pos = torch.randint(300, 500, (len(sections), 5), generator=g, device="cuda", dtype=torch.int32)
        cu = torch.tensor([0, 1, 2, 2 + new[2], 2 + new[2], 2 + new[2]], dtype=torch.int32, device="cuda")
        n_tok = int(cu[-1])
        for layer in range(2):
            q = cache.append(layer, qkv[:n_tok, :H], qkv[:n_tok, H:H + hkv], qkv[:n_tok, H + hkv:], positions=pos[:, :n_tok].contiguous(), inv_freq=inv, sections=sections, cu_new=cu)
            cache.check_status()
            angle = pc.angles(pos[:, :n_tok].cpu(), inv.cpu(), sections)
            want, size = pc.rotate(qkv[:n_tok, :H].cpu(), angle, False)
            assert ((q.cpu().double() - want).abs() <= pc.stored_tolerance(name, want, size)).all()
            k_new, k_size = pc.rotate(qkv[:n_tok, H:H + hkv].cpu(), angle, False)
            rows = [r for r in range(5) if active[r]]
            for i, r in enumerate(rows):
                assert cache.h_lens[r] == before[r] + 1
                got = held(cache, cache.k, r, layer)[-1]
                units = torch.ones(hkv, 1).double() if cache.k_scale is None else cache.k_scale[layer].cpu().double()[:, None]
                value = (k_new[i] / units).clamp(-448, 448) if kind == "e4m3" else k_new[i] / units
                assert ((got / units - value).abs() <= pc.stored_tolerance(kind, value, k_size[i] / units) + 1e-6 * value.abs()).all()
            full = torch.zeros((5, H, d), dtype=dtype, device="cuda")
            full[rows] = q
            lse = torch.empty((5, H), device="cuda")
            o = cache.attend(layer, full, lse=lse)
            cache.check_status()
            for r in range(5):
                ref, z, weight, size = pc.attention(full[r].cpu().double(), held(cache, cache.k, r, layer), held(cache, cache.v, r, layer))
                if cache.h_lens[r] == 0:
                    assert (o[r] == 0).all() and torch.isneginf(lse[r]).all()
                    continue
                assert ((o[r].cpu().double() - ref).abs() <= pc.attention_tolerance(name, kind, ref, weight, size, d)).all()
                assert ((lse[r].cpu().double() - z).abs() <= pc.lse_tolerance(z, size, d)).all()
    cache.release(0)
    assert cache.h_lens[0] == 0 and cache.free_pages == 80 - sum(-(-int(n) // 8) for n in cache.h_lens)


def test_a_captured_step_goes_on():
    """Append and attention of two layers in one graph, replayed token after token while lengths and pages change in device memory."""
    H, hkv, d, n = 8, 2, 128, 3
    g = torch.Generator("cuda").manual_seed(5)
    inv = (THETA ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).cuda()
    caches = [PagedCache(2, 60, 16, hkv, d, torch.bfloat16, n, 300) for _ in range(2)]      # replayed; eager
    for c in caches:
        c.set_rows([20, 0, 290])
        for x in (c.k, c.v):
            x.copy_(torch.randn(x.shape, generator=torch.Generator("cuda").manual_seed(6), device="cuda"))
    assert [p for p in caches[0]._pages] == [p for p in caches[1]._pages]
    qkv, pos = torch.zeros((2, n, H + 2 * hkv, d), dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    out = [torch.empty((n, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ws = torch.empty(max(16, P.purekv_decode_paged_ws_bytes(n, 300, H, hkv, d)), dtype=torch.uint8, device="cuda")

    def step(c, outs):
        for layer in range(2):
            q = c.append(layer, qkv[layer, :, :H], qkv[layer, :, H:H + hkv], qkv[layer, :, H + hkv:], positions=pos, inv_freq=inv)
            c.attend(layer, q, out=outs[layer], ws=ws, max_len=300)

    for c in caches:                      # once outside the capture; it overwrites the last rows that are there
        step(c, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], out)
    for token in range(9):
        for c in caches:
            c.advance([1, 1 if token >= 4 else 0, 1])
        qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda"))
        pos.copy_(torch.randint(0, 1000, (n,), generator=g, device="cuda", dtype=torch.int32))
        graph.replay()
        want = [torch.empty_like(out[0]) for _ in range(2)]
        step(caches[1], want)
        for a, b in zip(out, want):
            assert torch.equal(a, b)
        live = caches[0].h_lens > 0
        assert torch.isfinite(out[0][torch.from_numpy(live).cuda()]).all()
    for c in caches:
        c.check_status()


def test_the_packed_cache_and_the_pages_agree():
    """The same prompt into the packed cache and into pages: purekv_decode_attention and purekv_decode_paged of the same query."""
    cache, pipe, k, v, inv, g, dtype = conversation("bf16", 128, 8, 2, (64,), seed=3)
    q = torch.randn((3, 8, 128), generator=g, device="cuda").to(dtype)
    P.purekv_compact_kv(k[1:3], v[1:3], pipe.idx, pipe.batch, pipe.budget, k_out=pipe.k_c, v_out=pipe.v_c)
    for layer in range(2):
        a = P.purekv_decode_attention(q, pipe.k_c[layer], pipe.v_c[layer], pipe.budget)
        b = cache.attend(layer, q)
        for r in (0, 2):                   # request 1 has rows of its own in the pages
            assert (a[r].float() - b[r].float()).abs().max() <= 2.0 ** -6      # two bf16 results of values below 4: each within 2^-7


def test_rows_are_not_set_in_a_capture():
    cache = PagedCache(1, 8, 16, 2, 64, torch.bfloat16, 2, 40)
    cache.set_rows([3, 17])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        torch.zeros(4, device="cuda")
        with pytest.raises(RuntimeError):
            cache.advance()
    assert cache.h_lens.tolist() == [3, 17] and cache.free_pages == 5
    cache.advance()
    torch.cuda.synchronize()
    assert cache.seq_lens.tolist() == [4, 18]
