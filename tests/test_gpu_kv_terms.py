"""bf16 attention in a launch for up to four rows of a head of keys: weights in two bf16 terms, so that an output is what its exact value rounds to, or next to it
where that value lies by a boundary.

The bound: a bf16 number has 8 significant bits, so a rounding is off by at most 2^-8 of what is rounded, and a weight in two terms by 2^-16.  The weighted mean
is then off by at most 2^-16 sum_j w_j |v_j|, taken twice, beside ku.attention's bound for fp32 arithmetic; rounding keeps order, so the output lies
between what the two ends of that interval round to.  (A weight of one term is off by up to 2^-8: 256 times as much.)  ku.attention's bound for bf16 is its bound for
fp32 + 2^-8 (sum_j w_j |v_j| + |O|), which gives the sum."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import kv_util as ku  # noqa: E402


def outside(O, want):
    """Elements that two terms cannot give."""
    exact, _, fine, coarse, _ = want
    e = fine + 2.0 ** -15 * (256 * (coarse - fine) - exact.abs())
    return int(((O < (exact - e).bfloat16()) | (O > (exact + e).bfloat16())).sum())


@pytest.mark.parametrize("dim", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("lens,n_new,heads,kv_heads", [([300, 77, 5], [1, 1, 1], 4, 4), ([300, 900], [1, 1], 8, 2), ([500, 40], [4, 2], 2, 2),
                                                       ([9000, 4000], [1, 1], 12, 3)])
def test_up_to_four_rows(lens, n_new, heads, kv_heads, dim):
    from paper_2605_03109_amd import gsi

    print(f"case two terms lens={lens} new={n_new} {heads}/{kv_heads} dim={dim}", flush=True)
    cache, Q, q_start, kv_len, table = ku.layout(gsi, lens, n_new, heads, kv_heads, dim, 32, torch.bfloat16, 3, True)
    want = ku.attention(cache, Q, q_start, kv_len, table)
    O, lse = gsi.kv_attention(cache, Q, q_start, kv_len, table, max_q=max(n_new), lse=True)
    ku.check(O, lse, want, "terms")
    assert outside(O, want) == 0
