"""Rows next to the largest numbers: codes and scales as defined; what rounds to 2^128 is infinite in both types, its neighbours are what they are."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import kv_util as ku  # noqa: E402


@pytest.mark.parametrize("x", [torch.float32, torch.bfloat16])
def test_rows_next_to_the_largest_numbers(x):
    from paper_2605_03109_amd import gsi

    top = torch.finfo(x).max
    half = 3.5 * 2.0 ** 126                                       # a tie: to the even code, 4
    row = torch.tensor([half, -half, 0.96875 * half, -0.96875 * half, 2.0 ** 127, 1.5 * 2.0 ** 126, 0.0, -2.0 ** 100] * 4, device="cuda")
    K = torch.stack([row, torch.where(row == half, top, row), row.clamp(-0.96875 * half, 0.96875 * half)]).to(x).view(3, 1, 32)
    cache = gsi.KvCache.empty(1, 1, 32, 16)
    slots = torch.tensor([0, 5, 15], dtype=torch.int32, device="cuda")
    gsi.kv_append(cache, K, -K, slots)
    at = slots.long()
    for held, codes, scales in ((K, cache.K, cache.K_scale), (-K, cache.V, cache.V_scale)):
        code, byte, _ = ku.hold(held)
        assert torch.equal(codes[0, :, at].transpose(0, 1), ku.pack(code)) and torch.equal(scales[0, 0, 0, at], byte.flatten())
    for dt in (torch.float32, torch.bfloat16):
        for got, held in zip(gsi.kv_expand(cache, slots, dt), (K, -K)):
            assert torch.equal(got.double(), ku.hold(held)[2].to(dt).double())
            assert bool(torch.isinf(got[:2]).any()) and not torch.isinf(got[2]).any()
