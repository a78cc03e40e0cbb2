"""Tables of a paged cache built on the device, against a loop over requests."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def loop(kv_len, n_new, free, n_free, table, T, page):
    """What gsi_kv_tables returns, token by token; `table` is changed in place."""
    width = table.shape[1]
    n_free = max(0, min(n_free, len(free)))
    lens, start, slots, pos_, taken, missing = [], [0], [], [], 0, 0
    for b, (a, n) in enumerate(zip(kv_len, n_new)):
        a, n = max(a, 0), min(max(n, 0), T - start[-1])
        for j in range(-(-a // page), -(-(a + n) // page)):
            if j >= width:
                missing += 1
                continue
            table[b, j] = free[taken] if taken < n_free else -1
            if taken < n_free:
                taken += 1
            else:
                missing += 1
        for p in range(a, a + n):
            e = table[b, p // page] if p // page < width else -1
            slots.append(e * page + p % page if e >= 0 else -1)
            pos_.append(p)
        start.append(start[-1] + n)
        lens.append(a + n)
    pad = [-1] * (T - len(slots))
    return lens, start, slots + pad, pos_ + pad, [taken, missing]


def run(kv_len, n_new, page, width, T, n_free, seed, free_cap=None):
    from paper_2605_03109_amd import gsi

    rng = np.random.default_rng(seed)
    B = len(kv_len)
    have = [min(-(-max(a, 0) // page), width) for a in kv_len]
    cap = n_free if free_cap is None else free_cap
    ids = rng.permutation(sum(have) + cap).astype(np.int32)
    table = np.full((B, width), -7, np.int32)
    at = 0
    for b, n in enumerate(have):
        table[b, :n] = ids[at:at + n]
        at += n
    free = ids[at:]
    dev = lambda a: torch.tensor(np.asarray(a, np.int32).reshape(np.shape(a)), device="cuda")  # noqa: E731
    d_table = dev(table)
    inputs = [dev(kv_len), dev(n_new), dev(free), dev([n_free])]
    kept = [t.clone() for t in inputs]
    for _ in range(2):  # the same call again gives the same results
        got = gsi.kv_tables(*inputs, d_table, T, page)
        want_table = table.copy()
        want = loop(kv_len, n_new, free.tolist(), n_free, want_table, T, page)
        for name, g, w in zip(("kv_len", "q_start", "slots", "positions", "status"), got, want):
            assert g.tolist() == list(map(int, w)), name
        assert np.array_equal(d_table.cpu().numpy(), want_table)
    assert all(torch.equal(a, b) for a, b in zip(inputs, kept))


@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 511, 512, 513, 1500])
@pytest.mark.parametrize("page", [16, 128])
def test_ragged(B, page):
    print(f"case tables B={B} page={page}", flush=True)
    rng = np.random.default_rng(B + page)
    kv_len = rng.integers(0, 400, B).tolist()
    n_new = rng.integers(0, 40, B).tolist()
    need = sum(-(-(a + n) // page) - -(-a // page) for a, n in zip(kv_len, n_new))
    run(kv_len, n_new, page, 440 // page + 2, sum(n_new) + 5, need + 3, B)


def test_page_edges_and_idle_requests():
    kv_len = [0, 0, 15, 16, 17, 31, 32, 0, 16]
    n_new = [0, 1, 1, 1, 1, 1, 16, 33, 0]
    run(kv_len, n_new, 16, 8, sum(n_new), 40, 3)


def test_free_list_runs_out():
    run([0, 5, 40, 100], [64, 64, 64, 64], 16, 20, 256, 7, 4)
    run([0, 5], [64, 64], 16, 20, 128, 0, 5)
    run([0, 5], [64, 64], 16, 20, 128, 50, 6, free_cap=3)  # a counter past the list's end


def test_narrow_table_and_small_step():
    run([0, 30, 60], [80, 80, 80], 16, 4, 240, 40, 7)   # the table ends before the tokens
    run([0, 30, 60], [80, 80, 80], 16, 12, 100, 40, 8)  # the step ends inside the second request
    run([3, 30, 60], [80, 80, 80], 16, 12, 0, 40, 9)    # a step of no tokens


def test_negative_lengths_count_as_none():
    run([-5, 20, -1], [3, -4, 0], 16, 6, 10, 10, 10)


def test_long_prompts():
    run([0, 100000, 7], [70000, 1, 9000], 64, 2000, 79001, 1400, 11)


def test_no_requests():
    from paper_2605_03109_amd import gsi

    z = torch.zeros(0, dtype=torch.int32, device="cuda")
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens, start, slots, pos, status = gsi.kv_tables(z, z, one, one, torch.zeros((0, 4), dtype=torch.int32, device="cuda"), 3, 16)
    assert lens.numel() == 0 and start.tolist() == [0] and slots.tolist() == [-1] * 3 == pos.tolist() and status.tolist() == [0, 0]
