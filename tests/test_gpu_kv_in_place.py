"""Attention whose output takes the place of its queries, row for row: the same bits, in every kernel and division of the work."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import kv_util as ku  # noqa: E402

from test_gpu_kv_attention import DT  # noqa: E402


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lens,n_new,heads,kv_heads", [([300, 7, 0], [1, 1, 1], 4, 2), ([9000, 40], [1, 1], 8, 2), ([2900, 2500], [16, 9], 8, 2),
                                                       ([300, 150], [200, 75], 4, 2), ([4800, 300, 2100], [300, 150, 40], 4, 1),
                                                       ([3 + 20 * b for b in range(30)] + [600], [1] * 30 + [200], 4, 4)])
def test_in_place(lens, n_new, heads, kv_heads, dim, x):
    from paper_2605_03109_amd import gsi

    print(f"case in place lens={str(lens)[:40]} new={str(n_new)[:40]} {heads}/{kv_heads} dim={dim} {x}", flush=True)
    cache, Q, q_start, kv_len, table = ku.layout(gsi, lens, n_new, heads, kv_heads, dim, 32, DT[x], 4, True)
    want = gsi.kv_attention(cache, Q, q_start, kv_len, table, max_q=max(n_new), max_len=max(lens))
    both = Q.clone()
    assert gsi.kv_attention(cache, both, q_start, kv_len, table, max_q=max(n_new), max_len=max(lens), O=both) is both
    assert torch.equal(both, want)


def test_over_the_queries_of_a_fused_projection():
    """A row of O begins where the one before ends, not where the next row of Q begins: refused."""
    from paper_2605_03109_amd import gsi

    cache, Q, q_start, kv_len, table = ku.layout(gsi, [50, 20], [3, 2], 4, 2, 64, 16, torch.float32, 4, True)
    flat = torch.zeros(5, 3 * 4 * 64, device="cuda")
    q = flat[:, :256].unflatten(1, (4, 64))
    with pytest.raises(gsi.GsiError, match="lies over"):
        gsi.kv_attention(cache, q, q_start, kv_len, table, max_q=3, O=flat.view(-1)[:5 * 256].view(5, 4, 64))
