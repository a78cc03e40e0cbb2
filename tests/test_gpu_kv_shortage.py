"""Tables where pages run out: status[1] says in every step whether a token of it has no place, in the step that lacked the page and in those after."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def step(lens, n_new, free, n_free, table, T, page):
    from paper_2605_03109_amd import gsi

    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    out = gsi.kv_tables(dev(lens), dev(n_new), dev(free), dev([n_free]), table, T, page)
    return [t.tolist() for t in out]


def lost(lens, n_new, slots, page):
    """Pages that a token of the step lies on without a slot."""
    at, pages = 0, set()
    for b, (a, n) in enumerate(zip(lens, n_new)):
        for p in range(max(a, 0), max(a, 0) + n):
            if at < len(slots) and slots[at] < 0:
                pages.add((b, p // page))
            at += 1
    return len(pages)


def test_a_list_that_runs_out_inside_a_page():
    table = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    lens, _, slots, _, status = step([0, 3], [20, 2], [5], 1, table, 24, 16)
    assert lens == [20, 5] and status == [1, 2]                # the second page of the one, and the one that the other began without a page
    # pages come back: tokens of a page that is not there have no slot, and the step says so
    lens2, _, slots, _, status = step(lens, [1, 1], [7, 8, 9], 3, table, 2, 16)
    assert slots == [-1, -1] and status == [0, 2]
    # from the next page on the request has places again; what lies before stays a hole
    lens3, _, slots, _, status = step(lens2, [14, 0], [7, 8, 9], 3, table, 14, 16)
    assert slots == [-1] * 11 + [7 * 16, 7 * 16 + 1, 7 * 16 + 2] and status == [1, 1]
    assert table[0].tolist() == [5, -1, 7, -1]


def test_the_step_again_from_its_first_lengths():
    """Nothing was lost yet: the same lengths with pages that came back."""
    table = torch.full((1, 4), -1, dtype=torch.int32, device="cuda")
    _, _, slots, _, status = step([10], [40], [], 0, table, 40, 16)
    assert status == [0, 4] and slots == [-1] * 40
    table[0, 0] = 3
    _, _, slots, _, status = step([10], [40], [6, 2, 1], 3, table, 40, 16)
    assert status == [3, 0] and min(slots) >= 0 and table[0].tolist() == [3, 6, 2, 1]


def test_single_tokens_past_a_table_of_one_place():
    table = torch.full((1, 1), -1, dtype=torch.int32, device="cuda")
    lens = [15]
    table[0, 0] = 2
    for n in range(20):
        lens, _, slots, _, status = step(lens, [1], [9, 4], 2, table, 1, 16)
        assert (slots, status) == (([2 * 16 + 15], [0, 0]) if n == 0 else ([-1], [0, 1]))


@pytest.mark.parametrize("seed", range(6))
def test_every_loss_is_counted(seed):
    rng = np.random.default_rng(seed)
    B, page, width = [3, 40, 600, 9, 130, 1][seed], 16, 5
    lens = rng.integers(-2, 100, B).tolist()
    table = torch.tensor(rng.permutation(B * width).reshape(B, width), dtype=torch.int32, device="cuda")
    table[torch.tensor(rng.random((B, width)) < 0.3, device="cuda")] = -1
    table[0, 0] = 2 ** 31 - 1                                     # a page whose slots are no int32
    for _ in range(3):
        n_new = (rng.integers(0, 30, B) * (rng.random(B) < 0.7)).tolist()
        T = max(1, sum(n_new) - (seed == 3))                     # (seed 3: the last token does not fit into the step)
        before = lens
        lens, start, slots, _, status = step(lens, n_new, list(range(9000, 9000 + B)), B, table, T, page)
        n = [b - a for a, b in zip(start, start[1:])]
        assert status[1] == lost(before, n, slots, page)
