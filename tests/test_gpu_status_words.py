"""Calls made without a status word: what a paged call reports stops no prefill, and each report is read once."""
import numpy as np
import pytest
import torch

from paper_2510_25600_b200 import inputs
from tests import gpu_common as gc

pytestmark = pytest.mark.gpu


def store_into_a_missing_page(P):
    pool = torch.zeros((2, 16, 1, 64), dtype=torch.bfloat16, device="cuda")
    row = torch.ones((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    P.purekv_append_paged(row, row, pool, pool.clone(), ints([[5]]), ints([1]))


def polled(P):
    with pytest.raises(P.PureKVError) as e:
        P.purekv_poll_status(None)
    return e.value.status


def test_a_missing_page_stops_no_prefill():
    P = gc.pk()
    assert P.purekv_poll_status(None) == 0
    batch = inputs.make_batch([20, 0], [5, 3], [70, 150], 12, 12)
    wl = inputs.Workload("status words", 77, "bf16", 8, 2, 128, 1, (0,), (0,), batch, inputs.STMask(12, 12, tile=64), 16, 0.25)
    x, db = inputs.make_qkv(wl, 0), gc.device_batch(wl)
    q, k, v = (gc.upload(x, n, "bf16") for n in "qkv")
    buf, info = P.purekv_plan_build_host(db, P.st_params(wl.mask), P.BF16, wl.head_dim, wl.n_q_heads, wl.n_kv_heads)
    prefill = lambda plan: P.purekv_st_sparse_prefill(q, k, v, db, P.Plan(torch.from_numpy(plan).cuda(), info), out=torch.full_like(q, 7.0))
    plan = np.array(buf, copy=True)
    want = prefill(plan)
    store_into_a_missing_page(P)
    assert torch.equal(prefill(plan), want)
    assert polled(P) == P.ERR_BAD_PAGE and P.purekv_poll_status(None) == 0
    # both at once: one after the other
    wrong = plan.copy()
    P.PlanHeaderView.from_buffer(wrong).magic ^= 0x10
    store_into_a_missing_page(P)
    prefill(wrong)
    assert {polled(P), polled(P)} == {P.ERR_BAD_PLAN, P.ERR_BAD_PAGE} and P.purekv_poll_status(None) == 0
    assert torch.equal(prefill(plan), want)
