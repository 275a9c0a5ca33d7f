"""Waits of the paged decode step that run out: the call returns, says so in the status word, and the next one is right.  The limit is
set to no time at all, so that every copy under way is late; nothing is withheld, so all of them land."""
import time

import pytest
import torch

from paper_2510_25600_b200 import binding as P
from tests import paged_common as pc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [16, 12])     # the copy engine's loads, and the threads' (which wait for runs alone)
@pytest.mark.parametrize("kind,H,hkv,d", [("bf16", 8, 4, 128), ("bf16", 36, 4, 64), ("e4m3", 8, 8, 128), ("e4m3", 24, 2, 64), ("fp32", 4, 4, 128), ("fp32", 16, 2, 64)])
def test_late_copies_and_runs(kind, H, hkv, d, page):
    lens = [3000, 1, 0, 900, 5000, 64] + [40] * 200
    c = pc.Cache(50, lens, hkv, d, kind, page)
    q = torch.randn((len(lens), H, d), generator=torch.Generator().manual_seed(50)).to(torch.float32 if kind == "fp32" else torch.bfloat16)
    cache, scales = c.cuda()
    dq, lse, out = q.cuda(), torch.empty((len(lens), H), device="cuda"), torch.empty(q.shape, dtype=q.dtype, device="cuda")
    pools = [x.clone() for x in cache[:2]]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.zeros(P.purekv_decode_paged_ws_bytes(len(lens), 0, H, hkv, d, P.FP32 if kind == "fp32" else P.BF16), dtype=torch.uint8, device="cuda")
    step = lambda word: P.purekv_decode_paged(dq, *cache, out=out, lse=lse, ws=ws, status=word, **scales)
    step(None)
    want, want_lse = out.clone(), lse.clone()
    P.purekv_poll_status(None)
    P.purekv_set_wait_limit_ns(1)
    try:
        start = time.monotonic()
        for _ in range(5):
            step(status)
        if page == 16:
            with pytest.raises(P.PureKVError) as e:
                P.purekv_poll_status(status)
            assert e.value.status == P.ERR_TIMEOUT
        torch.cuda.synchronize()
        assert time.monotonic() - start < 1.0, "what is in flight lands at once: no CTA should have waited for something that never comes"
    finally:
        P.purekv_set_wait_limit_ns(0)
    status.zero_()
    step(status)
    assert P.purekv_poll_status(status) == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(pools, cache[:2]))
