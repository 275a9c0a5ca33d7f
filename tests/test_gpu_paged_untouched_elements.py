"""Elements of a row behind those that turn go through purekv_append_paged as they are, to the bit."""
import pytest
import torch

from paper_2510_25600_b200 import binding as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,d,rot", [(torch.bfloat16, 64, 32), (torch.bfloat16, 96, 48), (torch.float32, 64, 16), (torch.bfloat16, 128, 112)])
@pytest.mark.parametrize("n", [5, 700])
def test_every_bit_pattern(dtype, d, rot, interleaved, n):
    g = torch.Generator("cuda").manual_seed(100)
    whole = torch.int16 if dtype is torch.bfloat16 else torch.int32
    bits = torch.randint(-(1 << 31), 1 << 31, (n, 6, d), generator=g, device="cuda").to(whole)
    bits[:, :, rot::3] |= 0x7f80 if whole is torch.int16 else 0x7f800000          # infinities and NaN of every kind
    x = bits.view(dtype)
    pools = [torch.zeros((-(-n // 16), 16, 2, d), dtype=dtype, device="cuda") for _ in "kv"]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    k_out = torch.empty((n, 2, d), dtype=dtype, device="cuda")
    q_out = P.purekv_append_paged(x[:, 2:4], x[:, 4:], *pools, ints([list(range(pools[0].shape[0]))]), ints([n]), ints([0, n]), q=x[:, :2], k_out=k_out,
                                  positions=torch.arange(n, dtype=torch.int32, device="cuda"), inv_freq=torch.ones(rot // 2, dtype=torch.float64, device="cuda"),
                                  interleaved=interleaved)
    rows = lambda pool: pool.view(-1, 2, d)[:n].view(whole)
    assert torch.equal(q_out.view(whole)[..., rot:], bits[:, :2, rot:]) and torch.equal(k_out.view(whole)[..., rot:], bits[:, 2:4, rot:])
    assert torch.equal(rows(pools[0])[..., rot:], bits[:, 2:4, rot:]) and torch.equal(rows(pools[1]), bits[:, 4:])
