"""The attention half of a block over prompts and decode steps, against a plain one in 64 bits that keeps its own rows."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import kv_util as ku  # noqa: E402


@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 2)])
def test_prompts_then_tokens(heads, kv_heads):
    """Every token fires, so that a map is W x up to the image's rounding.  The rounding of a row to 4 bits is not continuous: the plain block
    takes the cache's rows as they are and checks that they are within half a code step of its own keys and values."""
    from paper_2605_03109_amd import gsi, serve

    print(f"case serve heads={heads}/{kv_heads}", flush=True)
    dev, dim, k, page = "cuda", 64, 64, 16
    d = heads * dim
    g = torch.Generator(device=dev).manual_seed(11)
    W = {n: (torch.randn(m, d, generator=g, device=dev) / d ** 0.5).to(torch.bfloat16) for n, m in
         (("q", d), ("k", kv_heads * dim), ("v", kv_heads * dim), ("o", d))}
    U = [torch.linalg.qr(torch.randn(d, k, generator=g, device=dev))[0].to(torch.bfloat16).contiguous() for _ in range(2)]
    block = serve.AttentionBlock(W, U[0], U[1], heads, kv_heads, 3, 40, 160, page, eps=0.0)
    past = [0, 0, 0]
    for n_new in ([70, 5, 0], [1, 1, 33], [1, 1, 1], [0, 90, 2], [1, 1, 1]):
        T = sum(n_new)
        X = torch.randn(T, d, generator=g, device=dev)
        got = block.step(X, torch.tensor(n_new, dtype=torch.int32, device=dev), max(n_new)).double()
        x = X.double()
        want_rows = {n: x @ W[n].double().t() for n in "kvq"}
        lens = [a + b for a, b in zip(past, n_new)]
        assert block.kv_len.tolist() == lens
        out = torch.zeros(T, heads, dim, dtype=torch.float64, device=dev)
        t0 = 0
        for b, n in enumerate(n_new):
            for h in range(kv_heads if n else 0):
                kk, vv, real = ku.keys_of(block.cache, block.table[b, :-(-lens[b] // page)].tolist(), h, lens[b])
                assert bool(real.all())
                for held, name in ((kk, "k"), (vv, "v")):
                    mine = want_rows[name][t0:t0 + n].view(n, kv_heads, dim)[:, h]
                    top = mine.view(n, -1, 32).abs().amax(-1, keepdim=True).expand(n, dim // 32, 32).reshape(n, dim)
                    # a step between codes is at most 2 of 6, so half of one is a sixth of what the scale is chosen for: below 1/3 of the largest
                    assert bool(((held[-n:] - mine).abs() <= top / 3 + 1e-2).all())
                q = want_rows["q"][t0:t0 + n].view(n, kv_heads, -1, dim)[:, h]
                s = torch.einsum("tgd,kd->tgk", q, kk) / math.sqrt(dim)
                later = torch.arange(lens[b], device=dev)[None] > lens[b] - n + torch.arange(n, device=dev)[:, None]
                p = torch.softmax(s.masked_fill(later[:, None], -math.inf), -1)
                out[t0:t0 + n].view(n, kv_heads, -1, dim)[:, h] = p @ vv
            t0 += n
        want = out.view(T, -1) @ W["o"].double().t()
        # images are rounded to bf16 (2^-9 relative of a map's fast part); queries' errors enter through scores of a few units
        err = (got - want).norm() / want.norm()
        assert float(err) <= 1e-2, f"step {n_new}: {float(err):.2e}"
        past = lens
    assert int(block.n_free) == 40 - sum(-(-n // page) for n in past)
    held = block.table[block.table >= 0]
    assert held.unique().numel() == held.numel() == sum(-(-n // page) for n in past)  # no page twice


def test_the_command(capsys, monkeypatch):
    import json
    import sys

    from paper_2605_03109_amd import serve

    monkeypatch.setattr(sys, "argv", ["serve", "--d", "512", "--heads", "8", "--kv-heads", "4", "--k", "64", "--requests", "3", "--prompt", "100", "--steps", "3"])
    assert serve.main() == 0
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["prompt_tokens"] > 100 and line["decode_us_per_step"] > 0
