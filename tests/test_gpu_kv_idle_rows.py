"""Tokens of the call that no request has, in front of the first and behind the last: O = 0 and lse = -inf, whatever lay there."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import kv_util as ku  # noqa: E402

from test_gpu_kv_attention import DT  # noqa: E402


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("front,back", [(3, 0), (7, 4), (0, 5)])
@pytest.mark.parametrize("lens,n_new,heads,kv_heads,max_len", [([50, 120], [1, 1], 4, 2, None), ([4000, 40], [1, 1], 4, 2, 4000), ([150, 90], [120, 77], 4, 2, 150),
                                                               ([2800, 300], [300, 150], 4, 1, 4200), ([9 * b for b in range(30)] + [300], [1] * 30 + [200], 4, 4, 300)])
def test_rows_of_no_request(lens, n_new, heads, kv_heads, max_len, front, back, x):
    from paper_2605_03109_amd import gsi

    print(f"case idle rows {front} {back} lens={str(lens)[:40]} {x}", flush=True)
    cache, Q, q_start, kv_len, table = ku.layout(gsi, lens, n_new, heads, kv_heads, 64, 16, DT[x], 4, True)
    T = Q.shape[0]
    want = ku.attention(cache, Q, q_start, kv_len, table)
    more = torch.full((front + T + back,) + Q.shape[1:], math.nan, dtype=Q.dtype, device="cuda")
    more[front:front + T] = Q
    O, lse = torch.full_like(more, 7.0), torch.full(more.shape[:2], 7.0, device="cuda")
    gsi.kv_attention(cache, more, q_start + front, kv_len, table, max_q=max(n_new), max_len=max_len, O=O, lse=lse)
    ku.check(O[front:front + T], lse[front:front + T], want, "between")
    for part, l in ((O[:front], lse[:front]), (O[front + T:], lse[front + T:])):
        assert not part.any() and bool((l == -math.inf).all())


@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_no_request_has_a_token(x):
    from paper_2605_03109_amd import gsi

    cache, Q, q_start, kv_len, table = ku.layout(gsi, [50, 120], [4, 3], 4, 2, 64, 16, DT[x], 4, True)
    O, lse = torch.full_like(Q, 7.0), torch.full(Q.shape[:2], 7.0, device="cuda")
    for at in (0, 3, 7):
        gsi.kv_attention(cache, Q, torch.full_like(q_start, at), kv_len, table, max_q=4, O=O.fill_(7.0), lse=lse.fill_(7.0))
        assert not O.any() and bool((lse == -math.inf).all())
