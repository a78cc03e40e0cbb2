"""Requests with more keys than their rows of the table have places: token i of n sees the keys j <= kv_len - n + i that lie on a page, against the
definition in 64 bits over the same table with entries that name no page behind its end."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import kv_util as ku  # noqa: E402

from test_gpu_kv_attention import DT  # noqa: E402


def cut(gsi, lens, n_new, heads, kv_heads, dim, page, x, width, seed=5):
    """A layout whose table ends after `width` places, and the same table as wide as the longest request with no pages there."""
    cache, Q, q_start, kv_len, table = ku.layout(gsi, lens, n_new, heads, kv_heads, dim, page, DT[x], seed, poison=True)
    wide = table.clone()
    wide[:, width:] = -1
    return cache, Q, q_start, kv_len, table[:, :width].contiguous(), wide


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("lens,n_new,heads,kv_heads,dim,page,width", [
    ([80, 40, 64], [10, 3, 1], 4, 2, 64, 64, 1),                        # few rows, whole tiles
    ([300, 64, 65], [2, 2, 1], 2, 2, 64, 16, 4),
    ([2700, 2550, 2570], [16, 9, 16], 8, 4, 64, 32, 80),                # few rows, shares
    ([80], [80], 4, 4, 64, 64, 1),                                      # prompts, whole tiles
    ([300, 90, 257], [200, 90, 257], 4, 2, 64, 16, 16),
    ([150, 700], [60, 500], 8, 2, 128, 64, 2),                          # more new tokens than places
    ([2800, 300, 2561], [300, 150, 40], 4, 1, 128, 64, 40),             # prompts, shares
    ([1 + 9 * b for b in range(30)] + [300], [1] * 30 + [200], 4, 4, 128, 16, 16),  # both kernels
])
def test_tokens_past_the_last_place(lens, n_new, heads, kv_heads, dim, page, width, x):
    from paper_2605_03109_amd import gsi

    print(f"case past the table lens={str(lens)[:40]} new={str(n_new)[:40]} {heads}/{kv_heads} dim={dim} page={page} width={width} {x}", flush=True)
    cache, Q, q_start, kv_len, table, wide = cut(gsi, lens, n_new, heads, kv_heads, dim, page, x, width)
    want = ku.attention(cache, Q, q_start, kv_len, wide)
    for max_len in (None, 4200):
        O, lse = gsi.kv_attention(cache, Q, q_start, kv_len, table, max_q=max(n_new), max_len=max_len, lse=True)
        ku.check(O, lse, want, f"max_len {max_len}")


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("n_new", [5, 70])
def test_the_longest_length(n_new, x):
    """All tokens lie behind the table's last place: each sees every key there is."""
    from paper_2605_03109_amd import gsi

    cache, Q, q_start, kv_len, table, wide = cut(gsi, [160 + n_new, 96], [n_new] * 2, 4, 2, 64, 16, x, 10)
    long = kv_len.clone()
    long[0] = 2 ** 31 - 1
    O, lse = gsi.kv_attention(cache, Q, q_start, long, table, max_q=n_new, lse=True)
    ku.check(O, lse, ku.attention(cache, Q, q_start, kv_len, wide), "2^31 - 1 keys")


@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_a_prompt_longer_than_its_row(x):
    """The tables' own outputs: of 80 tokens 64 have a place, and token i sees the first min(i + 1, 64) keys."""
    from paper_2605_03109_amd import gsi

    i32 = dict(dtype=torch.int32, device="cuda")
    heads, dim, page, T = 4, 64, 64, 80
    g = torch.Generator(device="cuda").manual_seed(2)
    K, V, Q = (torch.randn(T, heads, dim, generator=g, device="cuda").to(DT[x]) for _ in range(3))
    cache = ku.random_cache(gsi, 3, heads, dim, page, 4, poison=True)
    table = torch.full((1, 1), -1, **i32)
    kv_len, q_start, slots, _, status = gsi.kv_tables(torch.zeros(1, **i32), torch.full((1,), T, **i32), torch.tensor([2, 0], **i32),
                                                      torch.full((1,), 2, **i32), table, T, page)
    assert status.tolist() == [1, 1] and kv_len.tolist() == [80] and slots.tolist() == list(range(128, 192)) + [-1] * 16
    gsi.kv_append(cache, K, V, slots)
    O, lse = gsi.kv_attention(cache, Q, q_start, kv_len, table, max_q=T, lse=True)
    ku.check(O, lse, ku.attention(cache, Q, q_start, kv_len, torch.cat([table, table * 0 - 1], 1)), "a prompt of 80, 64 places")
