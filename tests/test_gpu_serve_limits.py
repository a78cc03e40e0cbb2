"""The attention half of a block at its limits: pages that run out, requests past their length, steps of many sizes."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def block_of(n_pages, max_len, requests=2, heads=4, dim=64, page=16, k=64):
    from paper_2605_03109_amd import serve

    d = heads * dim
    g = torch.Generator(device="cuda").manual_seed(3)
    W = {n: (torch.randn(d, d, generator=g, device="cuda") / d ** 0.5).to(torch.bfloat16) for n in "qkvo"}
    U = [torch.linalg.qr(torch.randn(d, k, generator=g, device="cuda"))[0].to(torch.bfloat16).contiguous() for _ in range(2)]
    block = serve.AttentionBlock(W, U[0], U[1], heads, heads, requests, n_pages, max_len, page)

    def step(*n_new):
        X = torch.randn(sum(n_new), d, generator=g, device="cuda")
        return block.step(X, torch.tensor(n_new, dtype=torch.int32, device="cuda"), max(n_new))

    return block, step


def test_pages_that_run_out_are_reported():
    block, step = block_of(n_pages=3, max_len=160)
    step(30, 10)
    assert block.status.tolist() == [3, 0] and int(block.missing) == 0 and int(block.n_free) == 0
    step(1, 1)                                                    # both still fit into their last pages
    assert block.status.tolist() == [0, 0] and int(block.missing) == 0
    step(1, 9)
    assert block.status.tolist() == [0, 1] and int(block.missing) == 1
    step(0, 1)                                                    # on a page that was not there
    assert block.status.tolist() == [0, 1] and int(block.missing) == 2 and int(block.n_free) == 0


def test_a_block_set_back():
    """Lengths, free list and their count as they were: the same step again gives the same."""
    block, step = block_of(n_pages=12, max_len=160)
    step(30, 10)
    state, table = (block.kv_len, block.free, block.n_free), block.table.clone()
    X, n_new = torch.randn(21, 256, device="cuda"), torch.tensor([20, 1], dtype=torch.int32, device="cuda")
    first = block.step(X, n_new, 20).clone()
    block.kv_len, block.free, block.n_free = state
    block.table.copy_(table)
    assert torch.equal(block.step(X, n_new, 20), first)
    assert int(block.n_free) == 12 - 4 - 1 and int(block.missing) == 0


def test_requests_past_their_length_are_reported():
    block, step = block_of(n_pages=20, max_len=32)
    step(32, 5)
    assert int(block.missing) == 0
    for n in range(1, 4):
        step(1, 1)
        assert int(block.missing) == n and int(block.n_free) == 17


def test_steps_of_many_sizes_keep_few_buffers():
    """Ragged prompts make steps of as many sizes as there are tokens: what a block holds does not grow with them."""
    block, step = block_of(n_pages=400, max_len=6000)

    def held_after(sizes):
        for n in sizes:
            step(n, n % 7)
        torch.cuda.synchronize()
        return torch.cuda.memory_allocated()

    held_after([100])
    before = held_after(range(60, 68))
    held_after(range(1, 100))
    # a size of 50 tokens takes 14 rows of 256 in fp32 a token, 0.7 MB, and its workspaces
    assert held_after(range(60, 68)) - before <= 8 << 20


def test_a_size_that_was_given_up_gives_the_same():
    a, step_a = block_of(n_pages=40, max_len=160)
    b, step_b = block_of(n_pages=40, max_len=160)
    b.KEPT = 1
    for n_new in ([20, 3], [1, 1], [20, 3], [1, 1], [5, 1], [1, 1]):
        assert torch.equal(step_a(*n_new), step_b(*n_new))
