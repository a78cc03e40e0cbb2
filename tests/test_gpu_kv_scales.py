"""Attention with scales at the ends of their range: 0 and next to it, and the largest."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import kv_util as ku  # noqa: E402

from test_gpu_kv_attention import DT  # noqa: E402


# (fp32 queries of 1e-36 reach below 2^-133 with their third terms, whose bits a scale of 2e38 would show)
@pytest.mark.parametrize("x,size,scale", [(x, *s) for x in ("f32", "bf16") for s in ((1e35, 0.0), (1e35, -0.0), (1e35, 1e-39), (1e35, 3e-37), (1e-30, 1e30))]
                         + [("bf16", 1e-36, 2.2e38), ("bf16", 1e-36, -2.2e38)])
@pytest.mark.parametrize("n_new", [1, 80])
def test_scales_that_are_tiny_or_huge(size, scale, n_new, x):
    """Scores in front of the scale reach 10^37, behind it a few units at most."""
    from paper_2605_03109_amd import gsi

    cache, Q, q_start, kv_len, table = ku.layout(gsi, [200, 90], [n_new, n_new], 4, 2, 64, 16, DT[x], 7, True)
    Q = (Q.float() * size).to(Q.dtype)
    scale = float(torch.tensor(scale, dtype=torch.float32))           # as the call takes it
    O, lse = gsi.kv_attention(cache, Q, q_start, kv_len, table, max_q=n_new, scale=scale, lse=True)
    ku.check(O, lse, ku.attention(cache, Q, q_start, kv_len, table, scale), f"queries of {size}, scale {scale}")


@pytest.mark.parametrize("scale", [2.4e38, -2.4e38, 3.4e38])
def test_scales_whose_exponents_are_no_numbers(scale):
    """scale * log2(e) has to be one."""
    from paper_2605_03109_amd import gsi

    cache, Q, q_start, kv_len, table = ku.layout(gsi, [20], [1], 4, 2, 64, 16, torch.float32, 7, True)
    with pytest.raises(gsi.GsiError):
        gsi.kv_attention(cache, Q, q_start, kv_len, table, max_q=1, scale=scale)
