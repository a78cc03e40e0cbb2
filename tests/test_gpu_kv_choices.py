"""Attention over the 4-bit cache against its definition in 64 bits where the choice of kernels and the division of the work change:
many requests, whole tiles and shares of both kernels, calls that take both, other streams."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import kv_util as ku  # noqa: E402

from test_gpu_kv_attention import DT, case  # noqa: E402


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("B,kv_heads", [(256, 1), (257, 1), (300, 2), (700, 1)])
def test_many_single_tokens(B, kv_heads, x):
    """Requests are looked up 256 at a time; up to 512 tiles are whole, more are shares."""
    case([(7 * b) % 90 for b in range(B)], [1] * B, 2 * kv_heads, kv_heads, 32, 16, x)


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("long", [130, 4200])
def test_many_prompts(long, x):
    """Prompts of 300 requests, some with more new tokens than keys or none; one long context makes them shares."""
    lens = [(11 * b) % 100 for b in range(299)] + [long]
    n_new = [max(0, n - (5 * b) % 60) + (b % 17 == 0) for b, n in enumerate(lens[:-1])] + [90]
    case(lens, n_new, 4, 1, 64, 16, x)


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [96, 128, 160, 256])
def test_prompts_in_shares(dim, x):
    """Fewer tiles than workgroups, contexts long enough that they are cut."""
    case([2800, 300, 2100], [300, 150, 40], 4, 1, dim, 64, x, max_len=4200)


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,n_new", [(8, 2, [16, 9]), (4, 4, [12, 7]), (32, 2, [4, 3])])
@pytest.mark.parametrize("dim", [64, 256])
def test_few_rows_in_shares(heads, kv_heads, n_new, dim, x):
    """Several tiles of 8 and 16 rows a request, cut by workgroups and waves."""
    case([2900, 2500], n_new, heads, kv_heads, dim, 32, x)


@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_few_rows_shares_of_many_short_tiles(x):
    """More tiles than workgroups: a wave ends some, begins others."""
    case([1 + (37 * b) % 200 for b in range(80)], [1 + b % 2 if b % 5 else 0 for b in range(80)], 16, 8, 64, 16, x)


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("long", [900, 3000])
def test_single_tokens_beside_a_prompt(long, x):
    """Both kernels in one call, each with its requests; tokens of no request at the end are cleared once."""
    from paper_2605_03109_amd import gsi

    lens, n_new = [(53 * b) % 700 + 1 for b in range(30)] + [long, 0], [1] * 30 + [200, 0]
    cache, Q, q_start, kv_len, table = ku.layout(gsi, lens, n_new, 4, 4, 128, 16, DT[x], 6, True)
    more = torch.cat([Q, Q[:3]])
    O, lse = gsi.kv_attention(cache, more, q_start, kv_len, table, max_q=200, lse=True)
    ku.check(O[:-3], lse[:-3], ku.attention(cache, Q, q_start, kv_len, table), "both kernels")
    assert not O[-3:].any() and bool((lse[-3:] == -float("inf")).all())


@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_lengths_past_the_table(x):
    """A request has no more keys than its row of the table has places."""
    from paper_2605_03109_amd import gsi

    for n_new in (1, 70):
        cache, Q, q_start, kv_len, table = ku.layout(gsi, [160, 96], [n_new] * 2, 4, 2, 64, 16, DT[x], 4, True, width=10)
        long = kv_len + torch.tensor([2 ** 31 - 1 - 160, 0], dtype=torch.int32, device="cuda")
        assert torch.equal(gsi.kv_attention(cache, Q, q_start, long, table, max_q=n_new), gsi.kv_attention(cache, Q, q_start, kv_len, table, max_q=n_new))


def test_every_call_on_another_stream():
    """Outputs that the calls allocate are the named stream's; the current one is busy meanwhile."""
    from paper_2605_03109_amd import gsi

    lens, n_new, heads, dim, page = [40, 0, 17], [1, 33, 5], 4, 64, 16
    i32 = dict(dtype=torch.int32, device="cuda")
    T = sum(n_new)
    K, V, Q = (torch.randn(T, heads, dim, device="cuda") for _ in range(3))

    def step(stream):
        cache = ku.random_cache(gsi, 16, heads, dim, page, 3)
        table = torch.full((3, 5), -1, **i32)
        table[0, :3], table[2, :2] = torch.tensor([3, 9, 4], **i32), torch.tensor([0, 7], **i32)
        free, n_free = torch.tensor([1, 2, 5, 6, 8, 10], **i32), torch.tensor([6], **i32)
        before, new = torch.tensor(lens, **i32), torch.tensor(n_new, **i32)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
            busy = torch.randn(2048, 2048, device="cuda")
            for _ in range(8):
                busy = busy @ busy * 1e-3
        length, start, slots, positions, status = gsi.kv_tables(before, new, free, n_free, table, T, page, stream=stream)
        gsi.kv_append(cache, K, V, slots, stream=stream)
        k, v = gsi.kv_expand(cache, slots, torch.bfloat16, stream=stream)
        O, lse = gsi.kv_attention(cache, Q, start, length, table, max_q=33, lse=True, stream=stream)
        nothing = gsi.kv_tables(before[:0], new[:0], free, n_free, table[:0], 4, page, stream=stream)
        torch.cuda.synchronize()
        return [length, start, slots, positions, status, k, v, O, lse, table, cache.K, cache.V_scale, *nothing]

    for a, b in zip(step(None), step(torch.cuda.Stream())):
        assert torch.equal(a, b)


def test_the_binding_refuses_what_it_can_see():
    from paper_2605_03109_amd import gsi

    cache = gsi.KvCache.empty(4, 2, 64, 16)
    i32 = dict(dtype=torch.int32, device="cuda")
    Q, start, lens, table = torch.zeros(3, 4, 64, device="cuda"), torch.tensor([0, 3], **i32), torch.tensor([5], **i32), torch.zeros(1, 2, **i32)
    slots = torch.zeros(3, **i32)
    for bad in (dict(Q=Q[..., :32]), dict(table=table[0]), dict(q_start=start[:1]), dict(kv_len=lens.long()), dict(Q=Q.transpose(0, 1)),
                dict(O=torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")), dict(lse=torch.zeros(3, 2, device="cuda")), dict(Q=Q.half())):
        with pytest.raises((ValueError, TypeError)):
            gsi.kv_attention(**{**dict(cache=cache, Q=Q, q_start=start, kv_len=lens, table=table), **bad})
    for K, V, s in ((Q[:, :2], Q[:, :2].bfloat16(), slots), (Q, Q, slots), (Q[:, :2], Q[:2, :2], slots), (Q[:, :2], Q[:, :2], slots[:2])):
        with pytest.raises(ValueError):
            gsi.kv_append(cache, K, V, s)
    with pytest.raises(ValueError):
        gsi.kv_expand(cache, slots, torch.float32, K=torch.zeros(3, 2, 32, device="cuda"))
    with pytest.raises(ValueError):
        gsi.kv_tables(lens, lens, slots, lens, table[0], 3, 16)
    with pytest.raises(gsi.GsiError):
        gsi.kv_attention(cache, Q, None, lens, table)  # three tokens, one request
